"""What the entry points of a bounded cache refuse before they touch the device (no GPU), and how mistakes reach Python."""
import ctypes as C

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2506_14158_amd import binding as B
from paper_2506_14158_amd.verify import TreeVerifier

ONE = C.c_void_p(256)          # never dereferenced: every call here fails before a launch


def shape(**kw):
    d = dict(B=2, Hq=8, Hkv=2, D=128, N=64, S_cap=64 * 128, dtype=B.S4C_BF16)
    d.update(kw)
    return B.AttnShape(**d)


def score(cap=0.0, slopes=None, key_pos=None, root_pos=None):
    return C.byref(B._Score(cap, slopes, key_pos, root_pos))


def test_scored_attention():
    L = B.lib()
    at = lambda sh=shape(), sc=score(), q=ONE, lse=ONE, m=4096, ws=ONE, wsb=1 << 30, scale=0.0: L.s4c_tree_attn_scored(
        C.byref(sh), sc, q, ONE, ONE, ONE, ONE, ONE, ONE, m, scale, ONE, lse, None, ws, wsb, None)
    assert at(q=None) == -1 and at(sh=shape(N=129)) == -3 and at(sh=shape(Hq=7)) == -2 and at(m=1 << 20) == -2
    assert at(q=C.c_void_p(264)) == -2
    assert B.s4c_tree_attn_workspace_size(shape(), 4096) > 0 and at(ws=None) == -4 and at(wsb=8) == -4
    for cap in (-1.0, float("nan"), float("inf"), -float("inf"), 3.3e38, 1e-40, 1e28, 1e-28):
        assert at(sc=score(cap)) == -2, cap
    assert at(sc=score(0.0, ONE, ONE, None)) == -1
    for scale in (1e-19, 1e19):
        assert at(sc=score(0.0, ONE), scale=scale) == -2, scale
    pg = lambda sh=shape(), bt=ONE, mb=64, ps=128, npg=200, pool=ONE: L.s4c_tree_attn_scored_paged(
        C.byref(sh), score(), ONE, ONE, ONE, pool, ONE, bt, mb, ps, npg, ONE, ONE, 4096, 0.0, ONE, None, None, ONE, 1 << 30, None)
    assert pg(bt=None) == -1 and pg(pool=None) == -1 and pg(ps=96) == -3 and pg(mb=0) == -2 and pg(npg=0) == -2 and pg(mb=63) == -2


def test_weights():
    L = B.lib()
    w = lambda sh=shape(), sc=score(), q=ONE, k=ONE, lse=ONE, mp=4, m=4096, win=ONE, out=ONE: L.s4c_kv_weigh(
        C.byref(sh), sc, q, k, lse, ONE, ONE, ONE, mp, m, 0.0, win, out, None, None)
    for kw in (dict(q=None), dict(k=None), dict(lse=None), dict(win=None), dict(out=None), dict(sc=score(0.0, None, ONE, None))):
        assert w(**kw) == -1, kw
    assert w(sh=shape(D=96)) == -3 and w(sh=shape(N=200)) == -3 and w(sh=shape(dtype=9)) == -3
    assert w(mp=0) == -2 and w(m=0) == -2 and w(m=1 << 20) == -2 and w(k=C.c_void_p(8)) == -2 and w(sc=score(-1.0)) == -2
    assert w(mp=1 << 28) == -3 and w(sh=shape(S_cap=(1 << 30) + 1)) == -3
    pg = lambda bt=ONE, mb=64, ps=128, npg=200: L.s4c_kv_weigh_paged(C.byref(shape()), score(), ONE, ONE, bt, mb, ps, npg, ONE, ONE, ONE, ONE, 4,
                                                                     4096, 0.0, ONE, ONE, None, None)
    assert pg(bt=None) == -1 and pg(ps=32) == -3 and pg(mb=0) == -2 and pg(mb=65) == -2 and pg(npg=-1) == -2


def test_eviction():
    L = B.lib()
    size = B.s4c_kv_evict_workspace_size
    assert size(1, 2, 2, 100, 8192) >= 4 * (8 + 2 * 100 * 4) and size(1, 2, 2, 100, 8192) % 256 == 0
    assert size(1, 2, 2, 8000, 8192) < size(1, 2, 2, 4096, 8192) and size(1, 2, 2, 9000, 8192) == 256
    for bad in ((0, 2, 2, 8, 64), (1, 0, 2, 8, 64), (1, 2, 0, 8, 64), (1, 2, 2, 0, 64), (1, 2, 2, 8, 0), (65535, 2, 2, 8, 64)):
        assert size(*bad) == 0
    ev = lambda sh=shape(), layers=1, k=ONE, win=ONE, pin=ONE, nxt=ONE, budget=100, recent=10, w=ONE, ws=ONE, wsb=1 << 20: L.s4c_kv_evict(
        C.byref(sh), layers, k, ONE, win, pin, ONE, nxt, budget, recent, w, ONE, ONE, None, None, ws, wsb, None)
    for kw in (dict(k=None), dict(win=None), dict(pin=None), dict(nxt=None), dict(w=None)):
        assert ev(**kw) == -1, kw
    for kw in (dict(layers=0), dict(layers=70000), dict(budget=0), dict(recent=-1), dict(recent=101), dict(k=C.c_void_p(24)), dict(sh=shape(B=0)),
               dict(sh=shape(S_cap=0))):
        assert ev(**kw) == -2, kw
    assert ev(sh=shape(D=80)) == -3 and ev(sh=shape(dtype=5)) == -3 and ev(sh=shape(S_cap=(1 << 30) + 1)) == -3
    assert ev(ws=None) == -4 and ev(wsb=size(1, 2, 2, 100, 8192) - 1) == -4 and ev(ws=C.c_void_p(128)) == -4
    pg = lambda bt=ONE, mb=64, ps=128, npg=200: L.s4c_kv_evict_paged(C.byref(shape()), 1, ONE, ONE, bt, mb, ps, npg, ONE, ONE, ONE, ONE, 100, 10,
                                                                     ONE, ONE, ONE, None, None, ONE, 1 << 20, None)
    assert pg(bt=None) == -1 and pg(ps=100) == -3 and pg(mb=1) == -2 and pg(npg=0) == -2


Bn, N, Hq, Hkv, D, S, PAGE, LY = 2, 8, 4, 2, 64, 128, 64, 3


def fakes():
    t = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")
    i = lambda *s: t(*s, dt=torch.int32)
    f = lambda *s: t(*s, dt=torch.float32)
    return dict(q=t(Bn, N, Hq, D), tree=t(Bn, N, Hkv, D), cache=t(Bn, Hkv, S, D), pool=t(4, Hkv, PAGE, D), table=i(Bn, S // PAGE), n=i(Bn),
                parent=i(Bn, N), caches=t(LY, Bn, Hkv, S, D), pools=t(LY, 4, Hkv, PAGE, D), lse=f(Bn, N, Hq), w=f(Bn, Hkv, S),
                ws=f(LY, Bn, Hkv, S), pos=i(Bn, Hkv, S), poss=i(LY, Bn, Hkv, S), slopes=f(Hq), path=i(Bn, 4))


CALLS = {
    "attention": lambda v, x: v.tree_attn_scored(x.q, x.tree, x.tree, x.cache, x.cache, x.n, x.parent, x.score),
    "step": lambda v, x: v.step(x.q, x.tree, x.tree, x.cache, x.cache, x.n, x.parent, x.w, x.parent, B.S4C_GREEDY, score=x.score),
    "attention, paged": lambda v, x: B.s4c_tree_attn_scored_paged(x.q, x.tree, x.tree, x.pool, x.pool, x.table, x.n, x.parent, S, x.score, v.out,
                                                                  x.lse, 0.0, v.attn_status, v.attn_ws),
    "weights": lambda v, x: v.kv_weigh(x.q, x.cache, x.n, x.score, x.w),
    "weights, paged": lambda v, x: B.s4c_kv_weigh_paged(x.q, x.pool, x.table, x.lse, x.n, x.path, x.n, S, x.score, x.w, x.w),
    "eviction": lambda v, x: v.kv_evict(x.caches, x.caches, x.ws, x.poss, x.n, x.n),
    "eviction, paged": lambda v, x: B.s4c_kv_evict_paged(x.pools, x.pools, x.table, x.ws, x.poss, x.n, x.n, 50, 5, x.ws, x.poss, x.n, v.evict_ws),
}
# one argument that is not as it has to be
WRONG = [("q", lambda t: t.float(), TypeError), ("tree", lambda t: t[:, :7].contiguous(), TypeError), ("n", lambda t: t.long(), TypeError),
         ("n", lambda t: t[:1], Exception), ("parent", lambda t: t[:, :7].contiguous(), TypeError), ("cache", lambda t: t[:1], ValueError),
         ("caches", lambda t: t[:, :1].contiguous(), ValueError), ("lse", lambda t: t.half(), TypeError), ("w", lambda t: t[:, :, :5].contiguous(), TypeError),
         ("ws", lambda t: t.double(), TypeError), ("poss", lambda t: t.long(), TypeError), ("table", lambda t: t.long(), TypeError),
         ("table", lambda t: t[:1], TypeError), ("table", lambda t: None, TypeError), ("pool", lambda t: t[0], ValueError)]
USES = {"attention": "q tree n parent cache", "step": "q tree n parent cache", "attention, paged": "q tree n parent table pool lse",
        "weights": "q n cache w", "weights, paged": "q n table pool lse w", "eviction": "n caches ws poss", "eviction, paged": "n ws poss table"}


@pytest.mark.skipif(torch.cuda.is_available(), reason="the stream lookup does not throw where there is a device")
@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
@pytest.mark.parametrize("name", CALLS)
def test_mistakes_reach_python(name):
    from types import SimpleNamespace
    with FakeTensorMode():
        x = fakes()
        x["score"] = B.Score(3.0, x["slopes"], x["pos"], x["n"])
        v = TreeVerifier(Bn, N, Hq, Hkv, D, S, 500, torch.bfloat16, 4, S, layers=LY, budget=50, recent=5)
        # nothing wrong but that there is no GPU
        with pytest.raises(RuntimeError, match="No HIP GPUs"):
            CALLS[name](v, SimpleNamespace(**x))
        for what, change, error in WRONG:
            if what in USES[name].split():
                with pytest.raises(error):
                    CALLS[name](v, SimpleNamespace(**{**x, what: change(x[what])}))
        for bad in (x["score"]._replace(slopes=x["slopes"][:3].contiguous()), x["score"]._replace(key_pos=x["poss"]),
                    x["score"]._replace(root_pos=x["lse"])):
            if "eviction" not in name:
                with pytest.raises(TypeError):
                    CALLS[name](v, SimpleNamespace(**{**x, "score": bad}))
