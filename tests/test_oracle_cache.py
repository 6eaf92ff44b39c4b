"""The 64-bit definitions of a bounded cache pinned by closed forms, hand-worked examples and the C oracle (CPU only)."""
import numpy as np

from oracle import cache_oracle as K
from oracle import s4c_oracle as O


def inputs(seed, B=2, N=6, Hq=4, Hkv=2, D=64, n=(9, 4)):
    r = np.random.default_rng(seed)
    f = lambda *s: r.standard_normal(s).astype(np.float32).astype(np.float64)
    parent = np.array([[-1, 0, 0, 1, 1, 3], [-1, 0, 1, 2, 3, 4]], dtype=np.int32)
    return f(B, N, Hq, D), f(B, N, Hkv, D), f(B, N, Hkv, D), f(B, Hkv, 16, D), f(B, Hkv, 16, D), np.array(n, dtype=np.int32), parent


def test_unchanged_scores_are_tree_attention():
    q, kt, vt, kc, vc, n, parent = inputs(1)
    f = lambda a: a.astype(np.float32)
    want, status = O.tree_attn(f(q), f(kt), f(vt), f(kc), f(vc), n, parent)[:2]
    assert not status.any()
    out, lse, mean, _, _, _ = K.tree_attn_scored(q, kt, vt, kc, vc, n, parent)
    assert np.abs(out - want).max() < 1e-12
    assert (np.abs(out) <= mean + 1e-15).all()
    # equal keys: the log-sum-exp is the score plus the log of their number
    kt[:], kc[:] = kt[0, 0, 0], kt[0, 0, 0]
    _, lse, _, _, _, _ = K.tree_attn_scored(q, kt, vt, kc, vc, n, parent)
    depth = [0, 1, 1, 2, 2, 3]
    for i in range(6):
        assert np.allclose(lse[0, i], kt[0, 0, 0] @ q[0, i].T / 8.0 + np.log(9 + depth[i] + 1))


def test_a_row_constant_changes_lse_alone():
    """Distances from the root instead of the node: the output is the same, lse differs by slope times depth."""
    q, kt, vt, kc, vc, n, parent = inputs(2)
    slopes = np.array([0.5, 0.25, 0.125, 2.0])
    out, lse, _, _, _, _ = K.tree_attn_scored(q, kt, vt, kc, vc, n, parent, cap=3.0, slopes=slopes)
    for b, i, h in np.ndindex(2, 6, 4):
        seen = K.ancestors_or_self(parent[b])[i]
        k = np.concatenate([kc[b, h // 2, :n[b]], kt[b, seen, h // 2]])
        v = np.concatenate([vc[b, h // 2, :n[b]], vt[b, seen, h // 2]])
        depth = len(seen) - 1
        x = 3.0 * np.tanh(k @ q[b, i, h] / 8.0 / 3.0) - slopes[h] * (n[b] + depth - np.concatenate([np.arange(n[b]), n[b] + np.arange(depth + 1)]))
        p = np.exp(x)
        assert np.allclose(out[b, i, h], p @ v / p.sum())
        assert np.allclose(lse[b, i, h], np.log(p.sum()) + slopes[h] * depth)


def test_positions_by_row_are_the_default():
    q, kt, vt, kc, vc, n, parent = inputs(3)
    slopes = np.array([0.5, 0.25, 0.125, 1.0])
    pos = np.tile(np.arange(16, dtype=np.int32) + 1000, (2, 2, 1))
    a = K.tree_attn_scored(q, kt, vt, kc, vc, n, parent, slopes=slopes)
    b = K.tree_attn_scored(q, kt, vt, kc, vc, n, parent, slopes=slopes, key_pos=pos, root_pos=n + 1000)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_weights_of_a_row_add_up_to_one():
    """Each query row gives away a weight of one, to keys up to its own."""
    q, kt, vt, kc, vc, n, parent = inputs(4)
    path = np.array([[0, 1, 3, -1], [0, 1, 2, 3]], dtype=np.int32)
    L = np.array([2, 3], dtype=np.int32)
    kw = dict(cap=2.0, slopes=np.array([0.1, 0.2, 0.3, 0.4]))
    _, lse, _, _, _, _ = K.tree_attn_scored(q, kt, vt, kc, vc, n, parent, **kw)
    for b in range(2):
        kc[b, :, n[b]:n[b] + L[b] + 1] = kt[b, path[b, :L[b] + 1]].transpose(1, 0, 2)
    before = np.full((2, 2, 16), 5.0)
    w, _, added = K.kv_weigh(q, kc, lse, n + L + 1, path, L, before, **kw)
    assert np.allclose(added.sum(-1), 2 * (L + 1)[:, None])
    for b in range(2):
        assert np.allclose(w[b, :, :n[b]], 5.0 + added[b, :, :n[b]])
        assert np.allclose(w[b, :, n[b]:n[b] + L[b] + 1], added[b, :, n[b]:n[b] + L[b] + 1])
        assert (w[b, :, n[b] + L[b] + 1:] == 5.0).all()


def test_eviction_by_hand():
    weight = np.array([[[[3.0, 1.0, 4.0, 1.0, 5.0, 9.0, 2.0, 6.0]]]])
    pos = np.arange(8, dtype=np.int32).reshape(1, 1, 1, 8)
    kept = lambda **kw: K.kv_evict(weight, kw.get("pos", pos), np.array([kw.get("n", 8)]), np.array([8]), kw["budget"], kw["recent"])
    k, n = kept(budget=4, recent=0)               # 4, 5, 9, 6 stay: rows 2, 4, 5, 7; places 0, 1, 3
    assert k[0, 0, 0].tolist() == [4, 5, 2, 7] and n.tolist() == [4]
    k, _ = kept(budget=4, recent=2)               # rows 6 and 7 are new; 9 and 5
    assert k[0, 0, 0].tolist() == [4, 5, 6, 7]
    k, _ = kept(budget=7, recent=0)               # of the two ones the first stays
    assert k[0, 0, 0].tolist() == [0, 1, 2, 7, 4, 5, 6]
    k, n = kept(budget=10, recent=3)              # nothing to do
    assert k[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, -1, -1] and n.tolist() == [8]
    k, _ = kept(budget=3, recent=3, pos=pos[..., ::-1].copy())        # the first rows are the new ones
    assert k[0, 0, 0].tolist() == [0, 1, 2]
    k, n = kept(budget=3, recent=0, n=0)
    assert k[0, 0, 0].tolist() == [-1, -1, -1] and n.tolist() == [0]


def test_gathered_pages():
    pool = np.arange(3 * 2 * 4 * 1).reshape(3, 2, 4, 1)
    got = K.gather_pages(pool, np.array([[2, 0]]))
    assert got[0, 1, :, 0].tolist() == [20, 21, 22, 23, 4, 5, 6, 7]
