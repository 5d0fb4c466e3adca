"""Pins of the oracle's draft trees and position eviction by hand-worked cases and identities."""
import numpy as np

from oracle import attention as OA
from oracle import bounded as OB
from oracle import drafts as OD
from oracle.kv_pool import KVPoolOracle


def test_a_chain_is_ordinary_decoding_one_token_after_another():
    rng = np.random.default_rng(1)
    S, T, Hq, Hkv, d = 5, 4, 4, 2, 8
    K, V = rng.standard_normal((2, S, Hkv, d))
    kd, vd = rng.standard_normal((2, T, Hkv, d))
    q = rng.standard_normal((T, Hq, d))
    got, _ = OD.tree_attention(q, K, V, kd, vd, [-1, 0, 1, 2], T)
    for u in range(T):
        want = OA.dense_decode_attention(q[u], np.concatenate([K, kd[:u + 1]]), np.concatenate([V, vd[:u + 1]]))
        np.testing.assert_allclose(got[u], want, atol=1e-12)


def test_paths_to_the_root():
    parents = [-1, 0, 0, 2, -1, 9, 5]                   # node 5's parent does not come before it: none
    assert OD.path_to_root(parents, 3) == [3, 2, 0]
    assert OD.path_to_root(parents, 4) == [4]
    assert OD.path_to_root(parents, 6) == [6, 5]


def test_slots_by_hand():
    #           0    1    2    3    4    5    6    7    8
    w = np.array([0.1, 0.9, 0.5, 0.5, 0.0, 0.8, 0.5, 0.2, 0.3])
    # budget 5, recent 2: of positions 0..6 the three largest are 1, 5 and (tie of 2, 3, 6) 2
    assert OB.slots(w, 9, 5, 2) == [5, 1, 2, 7, 8]
    assert OB.slots(w, 9, 5, 0) == [5, 1, 2, 3, 6]
    assert OB.slots(w, 9, 5, 5) == [4, 5, 6, 7, 8]
    nan = np.array([np.nan, -1.0, np.nan, -np.inf, 0.0, -0.0])
    assert OB.slots(nan, 6, 4, 0) == [4, 1, 5, 3]
    assert OB.slots(nan, 6, 5, 0) == [0, 1, 4, 3, 5] or OB.slots(nan, 6, 5, 0) == [0, 1, 5, 3, 4]


def test_evict_keeps_the_bookkeeping_consistent_and_unshares_pages():
    pool = KVPoolOracle(2, 2, 4, 4, 40, 4, 10)
    rng = np.random.default_rng(2)
    kp, vp = rng.standard_normal((2, 2, 2, 12, 4))
    ids = pool.fork_prefix(3, 12, kp, vp)
    kn, vn = rng.standard_normal((2, 3, 9, 2, 2, 4))
    pool.append_kv(ids, 9, kn, vn)
    w = rng.random((2, 2, 2, 24))
    before = [OA.gather_trace_kv(pool.k_pages[1], pool.v_pages[1], pool.block_table[2], 21)[0]]
    after, kept = OB.evict(pool, ids[:2], w, 10, 3)
    pool.check_invariants()
    assert list(pool.seq_lens[:3]) == [10, 10, 21] and pool.status == 0
    assert pool.refcount[pool.block_table[2, 0]] == 1   # the others have pages of their own now
    np.testing.assert_array_equal(OA.gather_trace_kv(pool.k_pages[1], pool.v_pages[1], pool.block_table[2], 21)[0], before[0])
    np.testing.assert_array_equal(kept[1, 0, 1, 7:], [18, 19, 20])
    K = OA.gather_trace_kv(pool.k_pages[1], pool.v_pages[1], pool.block_table[1], 10)[0]
    whole = np.concatenate([kp[1].swapaxes(0, 1), kn[1, :, 1]])
    np.testing.assert_array_equal(K[:, 1], whole[kept[1, 1, 1], 1])
    assert np.all(after[..., 10:] == 0)


def test_append_path_is_append_of_the_named_rows():
    rng = np.random.default_rng(3)
    a, b = (KVPoolOracle(1, 1, 4, 4, 20, 2, 6) for _ in range(2))
    kd, vd = rng.standard_normal((2, 2, 5, 1, 1, 4))
    for p in (a, b):
        p.fork_prefix(2, 0)
    path = np.array([[0, 2, 4], [1, 1, 0]])
    OD.append_path(a, [0, 1], 5, path, [3, 2], kd, vd)
    b.append_kv([0], 3, kd[:1, path[0]], vd[:1, path[0]])
    b.append_kv([1], 2, kd[1:, path[1, :2]], vd[1:, path[1, :2]])
    np.testing.assert_array_equal(a.k_pages, b.k_pages)
    assert list(a.seq_lens) == [3, 2] and a.status == 0
    OD.append_path(a, [1, 1, 0], 5, np.array([[0], [0], [7]]), [1, 1, 1], np.concatenate([kd, kd[:1]]), np.concatenate([vd, vd[:1]]))
    assert a.status == (1 << 3) | (1 << 1) and list(a.seq_lens) == [3, 3]


def test_slots_of_subnormal_weights_and_of_nan_by_hand():
    w = np.array([1e-40, 2e-40, 5e-39, 0.0, -0.0, -1e-45, 1e-45], dtype=np.float32)
    assert OB.slots(w, 7, 1, 0) == [2]
    assert OB.slots(w, 7, 4, 0) == [0, 1, 2, 6]
    assert OB.slots(w, 7, 6, 0) == [0, 1, 2, 3, 4, 6]
    # 0, 1, 3 and 4 stay where they are, and the free slot takes 5
    nan = np.array([np.nan, -1.0, np.nan, -np.inf, 0.0, -0.0])
    assert OB.slots(nan, 6, 5, 0) == [0, 1, 5, 3, 4]
