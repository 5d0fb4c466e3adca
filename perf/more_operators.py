"""What the rotary-position and fork-group operators of the KV pool are measured on.

Four kinds of pass:

rotate   rotate_positions: the rotary position of queries or keys, both directions (the transposed one is the gradient).
store    store_kv_rotated: keys are rotated on their way into the paged cache, values go along, the queries of the same
         tokens are rotated in the same launch; then the last token attends to what the last layer's cache now holds.
groups   decode_attention_groups: decode attention of traces that were forked from several prompts, each prompt's pages
         read once for all of its traces.
step     a decode step layer by layer, as a model runs it: store_kv_rotated and decode_attention_groups of every layer.

Head layouts and lengths are those of the repository's configurations (32/8 and 64/8 heads of 128 in bf16, 4/1 heads of 64
in fp32; prompts of 512 and of 8k to 32k tokens, 64 traces, decode steps of one token and bulk appends of 32).
"""
import math

import torch

own = False

PAGE = 16
HEADS = {"8b": (32, 8, 128, "bf16"), "gqa8": (64, 8, 128, "bf16"), "gqa5": (40, 8, 128, "bf16"),
         "tiny": (4, 1, 64, "fp32"), "half": (8, 2, 64, "bf16")}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

# what part of a head is rotated, the layout of a pair, and how the angles are stretched for contexts longer than trained on
ROTARY = {
    "halves": dict(part=1.0, base=1e6, interleaved=False),
    "pairs": dict(part=1.0, base=1e4, interleaved=True),
    "part": dict(part=0.5, base=1e4, interleaved=False),
    "quarter": dict(part=0.25, base=1e4, interleaved=True),
    "linear": dict(part=1.0, base=1e4, interleaved=False, scaling="linear", factor=8.0),
    "yarn": dict(part=1.0, base=1e6, interleaved=False, scaling="yarn", factor=4.0, original_positions=32768),
    "bands": dict(part=1.0, base=5e5, interleaved=False, scaling="bands", factor=8.0, original_positions=8192),
}


def listed():
    return [
        # one token's queries: the smallest call, latency counts
        dict(name="rotate-one", kind="rotate", heads="8b", what="q", batch=1, rows=1, far=2000, rotary="halves", back=False),
        # queries and keys of a prompt inside the packed output of a projection, a long context
        dict(name="rotate-prompt", kind="rotate", heads="8b", what="qk", batch=1, rows=8191, far=131072, rotary="yarn", back=False),
        # the gradient of the rotation, fp32, a part of each head, ragged row count
        dict(name="rotate-back", kind="rotate", heads="tiny", what="qk", batch=33, rows=1021, far=4096, rotary="part", back=True),
        # 64 reasoning steps of 1k tokens at once, neighbouring pairs
        dict(name="rotate-bulk", kind="rotate", heads="gqa8", what="q", batch=64, rows=1024, far=32768, rotary="pairs", back=False),
        # one trace, one token, one layer
        dict(name="store-one", kind="store", heads="8b", n=1, tokens=1, layers=1, base=100, shift=0, rotary="halves"),
        # the cache write of a decode step for 64 traces, four layers at once, positions ahead of a bounded cache's slots
        dict(name="store-64", kind="store", heads="8b", n=64, tokens=1, layers=4, base=300, shift=9000, rotary="bands"),
        # 32 tokens for 64 traces, all 36 layers
        dict(name="store-bulk", kind="store", heads="8b", n=64, tokens=32, layers=36, base=17, shift=0, rotary="halves"),
        # a few traces of one short prompt
        dict(name="groups-one", kind="groups", heads="8b", problems=1, per=4, prompt_lo=512, prompt_hi=512, lo=1, hi=100, ended=0.0),
        # 64 traces of one problem with a long prompt
        dict(name="groups-64", kind="groups", heads="8b", problems=1, per=64, prompt_lo=32768, prompt_hi=32768, lo=1, hi=1024, ended=0.0),
        # eight problems in one pool, ragged prompts, a quarter of the traces has ended
        dict(name="groups-8x12", kind="groups", heads="gqa8", problems=8, per=12, prompt_lo=1000, prompt_hi=16000, lo=0, hi=3000, ended=0.25),
        # fp32 pool, prompts of any length, some traces without a token of their own
        dict(name="groups-fp32", kind="groups", heads="tiny", problems=3, per=4, prompt_lo=5, prompt_hi=500, lo=0, hi=60, ended=0.1),
        # a decode step of four layers, two problems of 32 traces
        dict(name="step-2x32", kind="step", heads="8b", problems=2, per=32, layers=4, prompt_lo=8192, prompt_hi=8192, lo=1, hi=2048, rotary="halves"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotate", "store", "groups", "step"))
    heads = rng.choice(("8b", "8b", "gqa8", "gqa5", "tiny", "half"))
    small = heads in ("tiny", "half")
    rotary = rng.choice(sorted(ROTARY))
    if kind == "rotate":
        batch = _log(rng, 1, 64)
        return dict(kind=kind, heads=heads, what=rng.choice(("q", "qk")), batch=batch, rows=_log(rng, 1, 1000),
                    far=_log(rng, 1100, 1 << 20), rotary=rotary, back=rng.random() < 0.5)
    if kind == "store":
        return dict(kind=kind, heads=heads, n=_log(rng, 1, 64), tokens=_log(rng, 1, 32), layers=_log(rng, 1, 36),
                    base=rng.randint(0, 400), shift=rng.choice((0, rng.randint(1, 200000))), rotary=rotary)
    per = rng.randint(1, 32)
    case = dict(kind=kind, heads=heads, problems=rng.randint(1, min(16, 64 // per)), per=per)
    hi = _log(rng, 16, 700 if small else 16000 if kind == "groups" else 4000)
    case["prompt_lo"], case["prompt_hi"] = rng.randint(0, hi), hi
    most = 100 if small else 2000 if kind == "groups" else 500
    case["lo"], case["hi"] = sorted((_log(rng, 1, most), _log(rng, 1, most)))
    if kind == "step":
        return dict(case, layers=rng.randint(1, 4), rotary=rotary)
    return dict(case, lo=0, ended=rng.choice((0.0, rng.uniform(0.0, 0.9))))


def _frequencies(name, d):
    """Angle per position of every pair, in 64 bits, and the factor on the rotated values."""
    c = ROTARY[name]
    D = int(d * c["part"])
    theta = c["base"] ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    kind, s = c.get("scaling"), c.get("factor", 1.0)
    if kind == "linear":
        return D, theta / s, 1.0
    if kind == "yarn":
        at = [D * math.log(c["original_positions"] / (turns * 2 * math.pi)) / (2 * math.log(c["base"])) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), D - 1)
        slow = ((torch.arange(D // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return D, theta * (1 - slow) + theta / s * slow, 0.1 * math.log(s) + 1.0
    if kind == "bands":
        turns = c["original_positions"] * theta / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return D, theta * keep + theta / s * (1 - keep), 1.0
    return D, theta, 1.0


def _ints(gen, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=gen)


def _normal(gen, shape, dtype, std=1.0):
    out = torch.empty(shape, device="cuda", dtype=dtype)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 27):
        flat[a:a + (1 << 27)] = torch.randn(min(1 << 27, flat.numel() - a), generator=gen, device="cuda") * std
    return out


class State:
    pass


def _draw_inputs(c, seed):
    """Every input of a case, from the seed alone; lengths are made on the host."""
    Hq, Hkv, d, dt = HEADS[c["heads"]]
    t = TYPES[dt]
    host, gen = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
    s = State()
    s.c, s.dtype = c, t
    if c["kind"] == "rotate":
        packed = _normal(gen, (c["batch"], c["rows"], Hq + 2 * Hkv, d), t)
        s.x = packed[:, :, :Hq] if c["what"] == "q" else packed[:, :, :Hq + Hkv]
        first = _ints(host, 0, c["far"] - c["rows"], (c["batch"], 1))
        s.positions = (first + torch.arange(c["rows"])).int().cuda()
        return s
    if c["kind"] == "store":
        s.problems, s.per, s.L, s.T = 1, c["n"], c["layers"], c["tokens"]
        s.prompt = torch.zeros(1, dtype=torch.int64)
        s.own = _ints(host, 0, c["base"], (c["n"],))
        s.ended = torch.zeros(c["n"], dtype=torch.bool)
        shift = c["shift"]
    else:
        s.problems, s.per, s.L, s.T = c["problems"], c["per"], c.get("layers", 1), int(c["kind"] == "step")
        s.prompt = _ints(host, c["prompt_lo"], c["prompt_hi"], (s.problems,))
        s.own = _ints(host, c["lo"], c["hi"], (s.problems * s.per,))
        s.ended = torch.rand(s.problems * s.per, generator=host) < c.get("ended", 0.0)
        shift = 0
    n = s.n = s.problems * s.per
    s.cap = int(s.own.max()) + s.T                                 # own positions, the new tokens' among them
    s.kp, s.vp = (_normal(gen, (s.problems, max(1, int(s.prompt.max())), s.L, Hkv, d), t) for _ in range(2))
    s.k, s.v = (_normal(gen, (n, max(1, s.cap), s.L, Hkv, d), t) for _ in range(2))
    if c["kind"] == "groups":
        s.q = _normal(gen, (n, Hq, d), t, 1.5)
        return s
    s.q = _normal(gen, (s.L, n, s.T, Hq, d), t, 1.5)
    s.k_new, s.v_new = (_normal(gen, (n, s.T, s.L, Hkv, d), t) for _ in range(2))
    s.first = (s.prompt.repeat_interleave(s.per) + s.own + shift).int().cuda()       # position of the first new token
    s.positions = s.first if shift else None
    return s


def prepare(case, seed):
    s = _draw_inputs(case, seed)
    Hq, Hkv, d, dt = HEADS[case["heads"]]
    if "rotary" in case:
        s.D, s.theta, s.scale = _frequencies(case["rotary"], d)
        s.theta = s.theta.cuda()
        s.interleaved = ROTARY[case["rotary"]]["interleaved"]
    if own:
        from paper_2601_09093_b200 import binding as B

        if "rotary" in case:
            r = dict(ROTARY[case["rotary"]])
            s.rotary = B.Rotary(int(d * r.pop("part")), **r)
    if case["kind"] == "rotate":
        return s
    if own:
        pages = -(-(int(s.prompt.max()) + s.cap) // PAGE)
        blocks = sum(int(p) // PAGE for p in s.prompt) + s.n * (-(-s.cap // PAGE) + 1) + 8
        s.pool = B.KVPool(s.L, Hq, Hkv, d, PAGE, num_blocks=blocks, max_traces=s.n, max_pages_per_trace=max(1, pages),
                          dtype=B.STEP_BF16 if dt == "bf16" else B.STEP_FP32)
        for g in range(s.problems):
            P = int(s.prompt[g])
            s.pool.fork_prefix(s.per, P, *(x[g, :P].permute(1, 2, 0, 3).contiguous() for x in (s.kp, s.vp)))
        order, done = s.own.argsort(), 0
        for i in range(s.n):                    # traces grow together until each has its length
            upto = int(s.own[order[i]])
            for a in range(done, upto, 4096):
                b, rows = min(upto, a + 4096), order[i:].sort().values.cuda()
                s.pool.append_kv(rows.int(), b - a, s.k[rows, a:b].contiguous(), s.v[rows, a:b].contiguous())
            done = max(done, upto)
        if s.ended.any():
            s.pool.release_traces(s.ended.nonzero()[:, 0].int().cuda())
        s.ids = torch.arange(s.n, dtype=torch.int32, device="cuda")
        s.views = s.pool.views()
        s.group_rows = torch.arange(0, s.n + 1, s.per, dtype=torch.int32, device="cuda")
        s.group_pages = (s.prompt // PAGE).int().cuda()
        if case["kind"] != "groups":
            s.start = s.pool.extend(s.ids, s.T)
            s.q_out = torch.empty_like(s.q)
        del s.k, s.v, s.kp, s.vp
    s.prompt_dev = s.prompt.cuda()
    s.own_dev = s.own.cuda()
    s.live = (~s.ended).cuda()
    return s


def _turn(s, x, positions, back=False):
    """x [..., heads, d] rotated by positions [...]: 32 bits, angles in 64."""
    angle = positions.double()[..., None] * s.theta
    cos, sin = (angle.cos() * s.scale).float()[..., None, :], (angle.sin() * s.scale).float()[..., None, :]
    if back:
        sin = -sin
    x = x.float()
    y = x.clone()
    D = s.D
    a, b = (slice(0, D, 2), slice(1, D, 2)) if s.interleaved else (slice(0, D // 2), slice(D // 2, D))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _attend(s, q, layer, own_lens):
    """q [n, Hq, d] over each trace's prompt and its own positions, softmax over both together."""
    n, Hq, d = q.shape
    N, per, Hkv = s.problems, s.per, s.kp.shape[3]
    G = Hq // Hkv
    f = torch.float32
    rows = q.to(f).view(N, per, Hkv, G, d) * d ** -0.5
    kp, vp, k, v = (x[:, :, layer].to(f) for x in (s.kp, s.vp, s.k, s.v))
    P, S = kp.shape[1], k.shape[1]
    grouped = rows.permute(0, 2, 1, 3, 4).reshape(N, Hkv, per * G, d)
    sp = grouped @ kp.permute(0, 2, 3, 1)                                           # [N, Hkv, per G, P]
    sp.masked_fill_((torch.arange(P, device=q.device) >= s.prompt_dev[:, None])[:, None, None], -math.inf)
    sp = sp.view(N, Hkv, per, G, P).permute(0, 2, 1, 3, 4).reshape(n, Hkv, G, P)
    so = rows.view(n, Hkv, G, d) @ k.permute(0, 2, 3, 1)
    so.masked_fill_((torch.arange(S, device=q.device) >= own_lens[:, None])[:, None, None], -math.inf)
    top = torch.maximum(sp.amax(-1), so.amax(-1))[..., None]
    top = torch.where(top.isinf(), 0.0, top)
    pp, po = sp.sub_(top).exp_(), so.sub_(top).exp_()
    total = pp.sum(-1, keepdim=True) + po.sum(-1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    out = pp.view(N, per, Hkv, G, P).permute(0, 2, 1, 3, 4).reshape(N, Hkv, per * G, P) @ vp.permute(0, 2, 1, 3)
    out = out.view(N, Hkv, per, G, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, G, d) + po @ v.permute(0, 2, 1, 3)
    return torch.where(s.live[:, None, None], (out / total).reshape(n, Hq, d), 0.0).to(s.dtype)


def _store(s, layers):
    """The new tokens of the given layers into the dense cache behind every trace's own positions; their rotated queries."""
    at = torch.arange(s.T, device="cuda")
    pos = s.first[:, None] + at
    row, col = torch.arange(s.n, device="cuda")[:, None], s.own_dev[:, None] + at
    for l in layers:
        s.k[row, col, l] = _turn(s, s.k_new[:, :, l], pos).to(s.dtype)
        s.v[row, col, l] = s.v_new[:, :, l]
    return torch.stack([_turn(s, s.q[l], pos).to(s.dtype) for l in layers])


def run(state):
    s, c = state, state.c
    kind = c["kind"]
    if kind == "rotate":
        if own:
            from paper_2601_09093_b200 import binding as B

            return B.rotate_positions(s.x, s.rotary, s.positions, transpose=c["back"])
        return _turn(s, s.x, s.positions, c["back"]).to(s.dtype)
    if own:
        table, lens = s.views["block_table"], s.views["seq_lens"]
        attend = lambda l, q: s.pool.decode_attention_groups(l, q, table, lens, s.group_rows, s.group_pages)   # noqa: E731
        if kind == "groups":
            return attend(0, s.q)
        if kind == "store":
            s.pool.store_kv_rotated(0, s.ids, s.start, s.k_new, s.v_new, s.rotary, q=s.q, q_out=s.q_out, positions=s.positions)
            return s.q_out, attend(s.L - 1, s.q_out[-1, :, -1].contiguous())
        outs = []
        for l in range(s.L):
            s.pool.store_kv_rotated(l, s.ids, s.start, s.k_new[:, :, l:l + 1], s.v_new[:, :, l:l + 1], s.rotary, q=s.q[l:l + 1],
                                    q_out=s.q_out[l:l + 1], positions=s.positions)
            outs.append(attend(l, s.q_out[l, :, 0]))
        return s.q_out, outs
    if kind == "groups":
        return _attend(s, s.q, 0, s.own_dev)
    if kind == "store":
        q = _store(s, range(s.L))
        return q, _attend(s, q[-1, :, -1], s.L - 1, s.own_dev + s.T)
    qs, outs = [], []
    for l in range(s.L):
        qs.append(_store(s, [l]))
        outs.append(_attend(s, qs[-1][0, :, 0], l, s.own_dev + 1))
    return torch.cat(qs), outs


def work(case):
    Hq, Hkv, d, dt = HEADS[case["heads"]]
    e = 2 if dt == "bf16" else 4
    if case["kind"] == "rotate":
        rows, heads = case["batch"] * case["rows"], Hq + (Hkv if case["what"] == "qk" else 0)
        return {"bytes": rows * (heads * d * 2 * e + 4), "flops": 3.0 * rows * heads * d}
    row = 2 * Hkv * d * e                                         # K and V of one position of one layer
    if case["kind"] == "store":
        n, T, L = case["n"], case["tokens"], case["layers"]
        S = case["base"] / 2 + T
        return {"bytes": n * (T * L * (2 * row + 2 * Hq * d * e) + S * row + Hq * d * e),
                "flops": n * (3.0 * T * L * (Hq + Hkv) * d + 4.0 * Hq * d * S)}
    n, L = case["problems"] * case["per"], case.get("layers", 1)
    live, P, S = 1 - case.get("ended", 0.0), (case["prompt_lo"] + case["prompt_hi"]) / 2, (case["lo"] + case["hi"]) / 2
    one = case["problems"] * P * row + n * live * S * row + 2 * n * Hq * d * e
    flops = 4.0 * n * live * Hq * d * (P + S)
    if case["kind"] == "step":
        one, flops = one + n * (2 * row + 2 * Hq * d * e), flops + 3.0 * n * (Hq + Hkv) * d
    return {"bytes": L * one, "flops": L * flops}


def _exact_frequencies(name, d):
    """Pair by pair: a rotation slower than the trained length allows is slowed down by the factor."""
    c = ROTARY[name]
    D, s, kind, trained = round(d * c["part"]), c.get("factor", 1.0), c.get("scaling"), c.get("original_positions", 0)
    out, log_base = [], math.log(c["base"])
    for i in range(D // 2):
        f = math.exp(-2 * i / D * log_base)
        slowed = 0.0
        if kind == "linear":
            slowed = 1.0
        elif kind == "yarn":                                       # by the pair's index, between 32 turns and one
            first = max(0, math.floor(D / 2 * math.log(trained / (64 * math.pi)) / log_base))
            last = min(D - 1, math.ceil(D / 2 * math.log(trained / (2 * math.pi)) / log_base))
            slowed = min(1.0, max(0.0, (i - first) / (last - first)))
        elif kind == "bands":                                      # by its turns over the trained length, between 4 and one
            slowed = min(1.0, max(0.0, (4.0 - trained * f / (2 * math.pi)) / 3.0))
        out.append(f * (1.0 - slowed) + f * slowed / s)
    return D, torch.tensor(out, dtype=torch.float64), 1.0 + 0.1 * math.log(s) if kind == "yarn" else 1.0


def _exact_turn(case, x, positions):
    """x [..., heads, d] as pairs in the complex plane, times exp(i position theta)."""
    D, theta, scale = _exact_frequencies(case["rotary"], x.shape[-1])
    phase = torch.polar(torch.full((), scale, dtype=torch.float64, device=x.device),
                        positions.double()[..., None, None] * theta.to(x.device))
    if case.get("back"):
        phase = phase.conj()
    y = x.double().clone()
    if ROTARY[case["rotary"]]["interleaved"]:
        z = torch.view_as_complex(y[..., :D].unflatten(-1, (D // 2, 2)).contiguous()) * phase
        y[..., :D] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(y[..., :D // 2], y[..., D // 2:D].contiguous()) * phase
        y[..., :D] = torch.cat((z.real, z.imag), -1)
    return y


def exact(case, seed):
    """From the definitions in 64 bits, one trace and one KV head at a time."""
    s = _draw_inputs(case, seed)
    if case["kind"] == "rotate":
        return torch.cat([_exact_turn(case, x[None], p[None]) for x, p in zip(s.x, s.positions)])
    Hq, Hkv, d, _ = HEADS[case["heads"]]
    G = Hq // Hkv
    queries = [s.q.double()]
    if case["kind"] != "groups":
        pos = s.first[:, None] + torch.arange(s.T, device="cuda")
        turned = [_exact_turn(case, s.q[l], pos) for l in range(s.L)]
        layers = range(s.L) if case["kind"] == "step" else [s.L - 1]
        queries = [turned[l][:, -1].to(s.dtype).double() for l in layers]      # the cache and its readers hold rounded rows
    else:
        layers = [0]
    outs = []
    for l, q in zip(layers, queries):
        out = torch.zeros((s.n, Hq, d), dtype=torch.float64, device="cuda")
        if s.T:
            fresh = _exact_turn(case, s.k_new[:, :, l], pos).to(s.dtype)
        for i in range(s.n):
            P, S = int(s.prompt[i // s.per]), int(s.own[i])
            if s.ended[i] or P + S + s.T == 0:
                continue
            K, V = [s.kp[i // s.per, :P, l], s.k[i, :S, l]], [s.vp[i // s.per, :P, l], s.v[i, :S, l]]
            if s.T:
                K, V = K + [fresh[i]], V + [s.v_new[i, :, l]]
            K, V = torch.cat(K).double(), torch.cat(V).double()
            for h in range(Hkv):
                p = torch.softmax(q[i, h * G:(h + 1) * G] @ K[:, h].T / math.sqrt(d), 1)
                out[i, h * G:(h + 1) * G] = p @ V[:, h]
        outs.append(out)
    if case["kind"] == "groups":
        return outs[0]
    if case["kind"] == "store":
        return torch.stack(turned), outs[0]
    return torch.stack(turned), outs
