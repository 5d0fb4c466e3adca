"""What the speculative and bounded-cache operators of the KV pool are measured on.

Three kinds of pass:

tree     decode_attention_tree: attention of a tree of drafted tokens over a trace's cache.
weights  decode_attention_weights: decode attention that also adds every cached position's attention weight to a
         running sum per KV head.
bounded  the cache's side of a decode step with a bounded cache: append_kv_path stores the accepted drafts, evict_positions
         brings every trace back to its budget by weight, and the next token attends to what is left.

Head layouts and lengths are those of the repository's configurations (32/8 and 64/8 heads of 128 in bf16, 4/1 heads of 64
in fp32; prompts of 512, suffixes of 1k to 32k tokens).
"""
import math

import torch

own = False

PAGE = 16
HEADS = {"8b": (32, 8, 128, "bf16"), "gqa8": (64, 8, 128, "bf16"), "gqa5": (40, 8, 128, "bf16"),
         "tiny": (4, 1, 64, "fp32"), "half": (8, 2, 64, "bf16")}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one trace, one drafted token, a short prompt: the smallest call, latency counts
        dict(name="tree-one", kind="tree", heads="8b", n=1, nodes=1, lo=100, hi=100),
        # fp32 pool, ragged trees, some caches empty or one token long
        dict(name="tree-fp32", kind="tree", heads="tiny", n=8, nodes=13, lo=0, hi=256),
        # 64 sampled traces of one problem, each verifying a 16-token draft tree
        dict(name="tree-64x16", kind="tree", heads="8b", n=64, nodes=16, lo=4608, hi=16896),
        # wide trees over 8 query heads a KV head: 512 query rows for each key
        dict(name="tree-wide", kind="tree", heads="gqa8", n=32, nodes=64, lo=2048, hi=25600),
        # one trace
        dict(name="weights-one", kind="weights", heads="8b", n=1, lo=500, hi=500),
        # fp32 pool
        dict(name="weights-fp32", kind="weights", heads="tiny", n=8, lo=0, hi=256),
        # 64 traces in the middle of their reasoning
        dict(name="weights-64", kind="weights", heads="8b", n=64, lo=4608, hi=16896),
        # few traces with very long caches
        dict(name="weights-long", kind="weights", heads="gqa8", n=4, lo=98304, hi=131072),
        # small fp32 pool of two layers
        dict(name="bounded-fp32", kind="bounded", heads="tiny", n=8, layers=2, budget=129, recent=17, over=60, path=5),
        # 64 traces, drafts of up to 8 accepted tokens
        dict(name="bounded-64", kind="bounded", heads="8b", n=64, layers=4, budget=4096, recent=256, over=40, path=8),
        # all 36 layers of the 8B layout
        dict(name="bounded-36", kind="bounded", heads="8b", n=16, layers=36, budget=2048, recent=128, over=64, path=8),
        # a whole reasoning step is taken over at once, then the cache goes back to its budget
        dict(name="bounded-burst", kind="bounded", heads="8b", n=32, layers=2, budget=4096, recent=512, over=500, path=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("tree", "weights", "bounded"))
    heads = rng.choice(("8b", "8b", "gqa8", "gqa5", "tiny", "half"))
    small = heads in ("tiny", "half")
    n = _log(rng, 1, 8 if small else 64)
    if kind == "bounded":
        layers = rng.randint(1, 4)
        budget = _log(rng, 32, 512 if small else 4096)
        return dict(kind=kind, heads=heads, n=n, layers=layers, budget=budget, recent=rng.randint(1, budget),
                    over=rng.randint(0, budget // 4 + 1), path=_log(rng, 1, 64))
    hi = _log(rng, 8, 512 if small else (8192 if n > 16 else 20480))
    case = dict(kind=kind, heads=heads, n=n, lo=rng.randint(0, hi), hi=hi)
    if kind == "tree":
        case["nodes"] = _log(rng, 1, 64)
    return case


def _ints(gen, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=gen)


def _normal(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(dtype)


class State:
    pass


def _draw_inputs(c, seed):
    """Every input of a case, from the seed alone; lengths and trees are made on the host."""
    Hq, Hkv, d, dt = HEADS[c["heads"]]
    t, L, n = TYPES[dt], c.get("layers", 1), c["n"]
    host, gen = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
    s = State()
    s.c, s.dtype = c, t
    if c["kind"] == "bounded":
        s.lens = c["budget"] + _ints(host, 0, c["over"], (n,))
        T, s.budget = c["path"], c["budget"]
        s.cap = c["budget"] + c["over"] + T + 1
        s.path_len = _ints(host, 0, T, (n,)).int().cuda()
        s.weights = torch.exp(1.5 * torch.randn((L, n, Hkv, s.cap), generator=gen, device="cuda"))
        s.weights[torch.rand(s.weights.shape, generator=gen, device="cuda") < 0.1] = 0.0     # positions nothing looked at yet
        s.weights_out = torch.empty_like(s.weights)
        s.kept = torch.full((L, n, Hkv, c["budget"]), -1, dtype=torch.int32, device="cuda")
        # the accepted nodes: ascending indices into a draft twice as long (at most 64 wide trees, or a plain run)
        D = min(2 * T, T + 64)
        s.path = torch.rand((n, D), generator=host).argsort(1)[:, :T].sort(1).values.int().cuda()
        s.k_draft, s.v_draft = (_normal(gen, (n, D, L, Hkv, d), t) for _ in range(2))
        s.nodes = 1
        s.k_next, s.v_next = (_normal(gen, (n, 1, L, Hkv, d), t) for _ in range(2))
    else:
        s.lens = _ints(host, c["lo"], c["hi"], (n,))
        s.cap = max(1, c["hi"])
        if c["kind"] == "weights":
            s.weight_sum = torch.rand((n, Hkv, s.cap), generator=gen, device="cuda") * 0.05
        s.nodes = c.get("nodes", 1)
        s.k_next, s.v_next = (_normal(gen, (n, s.nodes, L, Hkv, d), t) for _ in range(2))
    T = s.nodes
    s.n_nodes = _ints(host, (T + 1) // 2, T, (n,)).int().cuda()
    up = (torch.rand((n, T), generator=host) * (torch.arange(T) + 1)).long()      # 0 .. u
    s.parents = (torch.maximum(up, torch.arange(T) - 5).clamp(max=63) - 1).clamp(min=-1)
    s.parents = torch.minimum(s.parents, torch.arange(T) - 1).int().cuda()
    s.q = _normal(gen, (n, T, Hq, d), t, 1.5)
    s.k, s.v = (_normal(gen, (n, s.cap, L, Hkv, d), t) for _ in range(2))
    return s


def prepare(case, seed):
    s = _draw_inputs(case, seed)
    if own:
        from paper_2601_09093_b200 import binding as B

        Hq, Hkv, d, dt = HEADS[case["heads"]]
        n, L = case["n"], case.get("layers", 1)
        pages = -(-s.cap // PAGE)
        s.pool = B.KVPool(L, Hq, Hkv, d, PAGE, num_blocks=n * pages + 8, max_traces=n, max_pages_per_trace=pages,
                          dtype=B.STEP_BF16 if dt == "bf16" else B.STEP_FP32)
        s.pool.fork_prefix(n, 0, None, None)
        order, done = s.lens.argsort(), 0
        for k in range(n):                    # traces grow together until each has its length
            upto = int(s.lens[order[k]])
            for a in range(done, upto, 4096):
                b, rows = min(upto, a + 4096), order[k:].sort().values.cuda()
                s.pool.append_kv(rows.int(), b - a, s.k[rows, a:b].contiguous(), s.v[rows, a:b].contiguous())
            done = max(done, upto)
        s.ids = torch.arange(n, dtype=torch.int32, device="cuda")
        s.views = s.pool.views()
        del s.k, s.v
    s.lens = s.lens.cuda()
    return s


def _ancestors(parents, n_nodes):
    """[n, T, T] bool: node u attends to node w (w is u or one of its ancestors); rows behind a tree's end are empty."""
    n, T = parents.shape
    at = torch.arange(T, device=parents.device)
    step = (parents[:, :, None] == at) | (at[:, None] == at)
    reach = step.float()
    for _ in range(max(1, (T - 1).bit_length())):          # paths of doubled length each time
        reach = (reach @ reach > 0).float()
    valid = at[None] < n_nodes[:, None]
    return (reach > 0) & valid[:, :, None] & valid[:, None, :]


def _attend(q, k, v, kd, vd, tree, lens):
    """q [n, T, Hq, d]; k, v [n, S, Hkv, d]; kd, vd [n, T, Hkv, d]; tree [n, T, T] -> out, weights of the cached positions."""
    n, T, Hq, d = q.shape
    S, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    rows = q.view(n, T, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * T, d) * d ** -0.5
    sc = torch.cat((rows @ k.permute(0, 2, 3, 1), rows @ kd.permute(0, 2, 3, 1)), -1)          # [n, Hkv, G T, S + T]
    sc.view(n, Hkv, G, T, S + T)[..., :S].masked_fill_((torch.arange(S, device=q.device) >= lens[:, None])[:, None, None, None], -math.inf)
    sc.view(n, Hkv, G, T, S + T)[..., S:].masked_fill_(~tree[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = sc.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, 1.0, total))
    out = p[..., :S] @ v.permute(0, 2, 1, 3) + p[..., S:] @ vd.permute(0, 2, 1, 3)
    return out.view(n, Hkv, G, T, d).permute(0, 3, 1, 2, 4).reshape(n, T, Hq, d), p[..., :S]


def _tree_plain(s, f, lens, k, v):
    seen = torch.arange(s.nodes, device="cuda")[None] < s.n_nodes[:, None]
    out, _ = _attend(s.q.to(f), k[:, :, 0].to(f), v[:, :, 0].to(f), s.k_next[:, :, 0].to(f), s.v_next[:, :, 0].to(f),
                     _ancestors(s.parents, s.n_nodes), lens)
    return torch.where(seen[:, :, None, None], out, 0.0)


def _weights_plain(s, f):
    none = s.k_next[:, :, 0].to(f)
    tree = torch.zeros((len(s.lens), 1, 1), dtype=torch.bool, device="cuda")
    out, p = _attend(s.q.to(f), s.k[:, :, 0].to(f), s.v[:, :, 0].to(f), none, none, tree, s.lens)
    return out[:, 0], p.sum(2)


def _commit(s):
    """The accepted nodes go behind every trace's cache."""
    T = s.path.shape[1]
    at = torch.arange(T, device="cuda")
    row, col = torch.nonzero(at < s.path_len[:, None], as_tuple=True)
    node, pos = s.path[row, col].long(), s.lens[row] + col
    s.k[row, pos], s.v[row, pos] = s.k_draft[row, node], s.v_draft[row, node]
    s.lens = s.lens + s.path_len


def _evict(s):
    """Every trace longer than its budget keeps its last `recent` positions, as the last slots of the budget, and those of
    the largest weight before them: where such a position lies below those slots it stays, the free slots there take
    the others in order."""
    b, m, pos = s.budget, s.budget - s.c["recent"], torch.arange(s.cap, device="cuda")
    S = s.lens[:, None]
    first = (S - s.c["recent"])[None, :, None]
    old = pos < first
    key = torch.where(old, s.weights, -math.inf)
    best = key.sort(dim=-1, descending=True, stable=True).indices[..., :m]
    chosen = torch.zeros_like(old.expand_as(key)).scatter(-1, best, True)
    free, come = ~chosen[..., :m], chosen & (pos >= m)
    nth = come.cumsum(-1) - 1                                        # the how-manieth of those that move in
    source = torch.zeros_like(key, dtype=torch.int64).scatter_add(
        -1, torch.where(come, nth, s.cap - 1), torch.where(come, pos, 0))
    low = torch.where(free, source.gather(-1, (free.cumsum(-1) - 1).clamp(min=0)), pos[:m])
    last = (first + torch.arange(s.c["recent"], device="cuda")).expand(*low.shape[:-1], -1)
    kept = torch.cat((low, last), -1)                                # [L, n, Hkv, b]: the old place of every slot
    cut = (s.lens > b)[None, :, None, None]
    kept = torch.where(cut, kept, pos[:b])
    moved = torch.zeros_like(s.weights)
    moved[..., :b] = s.weights.gather(-1, kept)
    s.weights_out = torch.where(cut, moved, s.weights)
    at = kept.permute(1, 3, 0, 2)[..., None].expand(-1, -1, -1, -1, s.k.shape[-1])                # [n, b, L, Hkv, d]
    s.k[:, :b], s.v[:, :b] = s.k.gather(1, at), s.v.gather(1, at)
    s.kept = torch.where(cut, kept.int(), s.kept)
    s.lens = s.lens.clamp(max=b)


def run(state):
    s, kind = state, state.c["kind"]
    if own:
        v = s.views
        if kind == "tree":
            return s.pool.decode_attention_tree(0, s.q, s.k_next, s.v_next, s.parents, v["block_table"], v["seq_lens"],
                                                n_nodes=s.n_nodes)
        if kind == "weights":
            out = s.pool.decode_attention_weights(0, s.q[:, 0], v["block_table"], v["seq_lens"], s.weight_sum)
            return out, s.weight_sum
        s.pool.append_kv_path(s.ids, s.k_draft, s.v_draft, s.path, s.path_len)
        s.pool.evict_positions(s.ids, s.weights, s.budget, s.c["recent"], weights_out=s.weights_out, kept_out=s.kept)
        out = s.pool.decode_attention_tree(0, s.q, s.k_next, s.v_next, s.parents, v["block_table"], v["seq_lens"])
        return out, s.kept, s.weights_out, v["seq_lens"]
    if kind == "tree":
        return _tree_plain(s, torch.float32, s.lens, s.k, s.v).to(s.dtype)
    if kind == "weights":
        out, w = _weights_plain(s, torch.float32)
        s.weight_sum += w
        return out, s.weight_sum
    _commit(s)
    _evict(s)
    out = _tree_plain(s, torch.float32, s.lens, s.k[:, :s.budget], s.v[:, :s.budget]).to(s.dtype)
    return out, s.kept, s.weights_out, s.lens.int()


def work(case):
    Hq, Hkv, d, dt = HEADS[case["heads"]]
    n, L, e = case["n"], case.get("layers", 1), 2 if dt == "bf16" else 4
    row = 2 * Hkv * d * e                                         # K and V of one position of one layer
    if case["kind"] == "bounded":
        b, p = case["budget"], case["path"] / 2                   # accepted tokens, on average
        gone = p + case["over"] / 8                               # the first pass also cuts what is over
        moved = n * L * row * 2 * (p + case["recent"] + min(gone, b - case["recent"]))   # drafts in, the last ones along, holes filled
        lists = n * L * Hkv * 4 * (3 * b + p)
        return {"bytes": moved + lists + n * (b * row + 2 * Hq * d * e), "flops": 4.0 * n * Hq * d * b}
    S = (case["lo"] + case["hi"]) / 2
    T = 0.75 * case["nodes"] if case["kind"] == "tree" else 1
    if case["kind"] == "tree":
        return {"bytes": n * (S * row + T * row + 2 * T * Hq * d * e), "flops": 4.0 * n * T * Hq * d * (S + T / 2)}
    return {"bytes": n * (S * (row + 8 * Hkv) + Hq * d * (e + 4)), "flops": 4.0 * n * Hq * d * S}


def exact(case, seed):
    """From the definitions in 64 bits, one trace and one KV head at a time."""
    s = _draw_inputs(case, seed)
    Hq, Hkv, d, _ = HEADS[case["heads"]]
    G, n, T = Hq // Hkv, case["n"], s.nodes
    lens, kind = s.lens.tolist(), case["kind"]
    nodes = [1] * n if kind != "tree" else s.n_nodes.tolist()
    parents = s.parents.tolist()
    out = torch.zeros((n, T, Hq, d), dtype=torch.float64, device="cuda")
    sums = s.weight_sum.double() if kind == "weights" else None
    for i in range(n):
        keep = None
        K, V = s.k[i, :lens[i]], s.v[i, :lens[i]]
        if kind == "bounded":
            take = s.path[i, :int(s.path_len[i])].long()
            K, V = torch.cat((K, s.k_draft[i, take])), torch.cat((V, s.v_draft[i, take]))
            if len(K) > s.budget:
                first = len(K) - case["recent"]
                w = s.weights[0, i, :, :first].double().cpu()
                keep = [sorted(sorted(range(first), key=lambda j, r=r: (-r[j], j))[:s.budget - case["recent"]])
                        + list(range(first, len(K))) for r in w.tolist()]
        sees = torch.zeros((T, T), dtype=torch.bool)
        for u in range(nodes[i] if kind != "weights" else 0):
            w = u
            while w >= 0:
                sees[u, w] = True
                w = parents[i][w]
        live = nodes[i]
        for h in range(Hkv):
            k, v = K[:, 0, h].double(), V[:, 0, h].double()
            if keep is not None:
                k, v = k[keep[h]], v[keep[h]]
            q = s.q[i, :live, h * G:(h + 1) * G].double().reshape(live * G, d)
            a = q @ k.T / math.sqrt(d)
            if kind != "weights":
                a = torch.cat((a, (q @ s.k_next[i, :live, 0, h].double().T / math.sqrt(d)).masked_fill(
                    ~sees[:live, :live].repeat_interleave(G, 0).cuda(), -math.inf)), 1)
                v = torch.cat((v, s.v_next[i, :live, 0, h].double()))
            if a.shape[1] == 0:
                continue
            p = torch.softmax(a, 1)
            out[i, :live, h * G:(h + 1) * G] = (p @ v).view(live, G, d)
            if kind == "weights":
                sums[i, h, :lens[i]] += p.sum(0)
    if kind == "tree":
        return out
    if kind == "weights":
        return out[:, 0], sums
    return out, None, None, None
