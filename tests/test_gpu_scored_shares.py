"""Attention with changed scores whose units are divided into balanced shares: parts and whole units, their outputs and log-sum-exp,
against the 64-bit definition.  tests/test_scored_division.py checks that the cases are divided so."""
import copy

import pytest
import torch

from paper_2506_14158_amd import binding as B
from tests.test_gpu_division import Case as Sizes
from tests.test_gpu_scored import Case

pytestmark = pytest.mark.gpu

# Lengths repeat over the batch.  Of one tile or a few under a large max_cache_len: shares of a tile, and teams without one; long ones: shares
# that end inside units, with whole units between.
SHARES = [
    Sizes("rows256", "balanced", 7, 8, 4, 128, 47, "bf16", 8192, (5, 900, 0, 64, 129, 1100, 8193)),
    Sizes("rows256-long", "balanced", 7, 8, 4, 128, 47, "f16", 8192, (2300, 0, 1900, -1, 2111)),
    Sizes("rows256-two-tiles-of-rows", "balanced", 13, 2, 4, 128, 75, "bf16", 5003, (700, 1, 64, 0, 301)),
    Sizes("rows256-d64", "balanced", 7, 8, 4, 64, 47, "bf16", 8192, (2000, 63, 0, 1500, 640)),
    Sizes("rows128", "balanced", 7, 8, 4, 128, 20, "bf16", 8192, (1900, 5, 0, 1333, 64)),
    Sizes("rows128-d64", "balanced", 13, 8, 4, 64, 20, "f16", 8192, (1000, 0, 1, 64, 777, 8193)),
    Sizes("rows128-70-sequences", "balanced", 70, 2, 4, 128, 20, "bf16", 3000, (300, 0, 64, 5, 400)),
    Sizes("rows64", "balanced", 3, 32, 1, 128, 37, "bf16", 24000, (2000, 0, 1111)),
    Sizes("rows32-d64", "balanced", 13, 16, 1, 64, 20, "f16", 3000, (32, 0, 1, 500, 3001)),
    Sizes("rows32-long", "balanced", 13, 16, 2, 64, 1, "bf16", 3000, (3000, 2901)),
    Sizes("rows32-deep", "balanced", 33, 8, 1, 128, 20, "f16", 7960, (500, 0, 33, 7961, 64)),
    Sizes("rows64-f32", "balanced", 3, 30, 2, 64, 40, "f32", 3000, (2, 50, 1333)),
    Sizes("rows64-f32-d128", "balanced", 7, 20, 2, 128, 13, "f32", 2500, (900, 0, 331, 64)),
]
# every kind: the log-sum-exp alone, a cap, a bias, both
SCORES = [(0.0, "none"), (20.0, "none"), (0.0, "rows"), (0.0, "kept"), (15.0, "kept")]


def wide(c, S_cap):
    """The case in caches of S_cap rows a sequence; rows behind its own are zeros (contiguous), or page 0 (paged)."""
    w, n = copy.copy(c), c.shape.S_cap
    w.shape = copy.copy(c.shape)
    w.shape.S_cap = S_cap
    Bn, Hkv, D = c.shape.B, c.shape.Hkv, c.shape.D
    w.pos = torch.zeros(Bn, Hkv, S_cap, dtype=torch.int32, device="cuda")
    w.pos[:, :, :n] = c.pos
    if c.page:
        w.table = torch.zeros(Bn, S_cap // c.page, dtype=torch.int32, device="cuda")
        w.table[:, :n // c.page] = c.table
    else:
        w.kc, w.vc = (torch.zeros(Bn, Hkv, S_cap, D, dtype=t.dtype, device="cuda") for t in (c.kc, c.vc))
        w.kc[:, :, :n], w.vc[:, :, :n] = c.kc, c.vc
    return w


def of_heads(c, kv):
    """The case of some of its KV heads, results included."""
    s, G = copy.copy(c), c.shape.Hq // c.shape.Hkv
    heads = [h for g in kv for h in range(g * G, (g + 1) * G)]
    s.shape = copy.copy(c.shape)
    s.shape.Hkv, s.shape.Hq = len(kv), len(heads)
    s.q, s.out, s.lse, s.slopes = c.q[:, :, heads], c.out[:, :, heads], c.lse[:, :, heads], c.slopes[heads]
    s.kt, s.vt, s.pos = c.kt[:, :, kv], c.vt[:, :, kv], c.pos[:, kv]
    s.kc, s.vc = c.kc[:, kv], c.vc[:, kv]
    return s


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("sizes", SHARES, ids=lambda s: s.name)
def test_balanced_shares_against_the_definition(sizes, page):
    z, page = sizes, page and (64 if sizes.D == 128 else 128)
    lens = [z.lens[b % len(z.lens)] for b in range(z.B)]
    flagged = [not 0 <= n <= z.max_len for n in lens]
    short = [0 if f else n for n, f in zip(lens, flagged)]
    rows = -(-max(short) // 128) * 128
    c = Case(sum(map(ord, z.name)), z.B, z.N, z.Hkv * z.G, z.Hkv, z.D, z.dtype, short, rows, page)
    w = wide(c, -(-z.max_len // 128) * 128)
    for i, (cap, bias) in enumerate(SCORES):
        w.out.fill_(7.0)
        w.lse.fill_(7.0)
        w.len.copy_(torch.tensor(short, dtype=torch.int32))
        w.call(w.score(cap, bias), max_len=z.max_len)
        assert not w.status.any()
        for k in range(2):                       # of the first, a middle and the last KV head two
            s = of_heads(c, [(0, z.Hkv // 2, z.Hkv - 1)[(i + k) % 3]])
            s.check(s.score(cap, bias))
        if any(flagged):
            out, lse = w.out.clone(), w.lse.clone()
            w.len.copy_(torch.tensor(lens, dtype=torch.int32))
            w.call(w.score(cap, bias), max_len=z.max_len)
            assert w.status.tolist() == [B.S4C_SEQ_BAD_LEN if f else 0 for f in flagged]
            bad = torch.tensor(flagged)
            assert not w.out[bad].any() and (w.lse[bad] == float("inf")).all()
            assert torch.equal(w.out[~bad], out[~bad]) and torch.equal(w.lse[~bad], lse[~bad])


def test_balanced_shares_replayed():
    """A captured call, replayed with other lengths (other shares) between eager ones."""
    z = SHARES[4]
    c = Case(30, z.B, z.N, z.Hkv * z.G, z.Hkv, z.D, z.dtype, [1900] * z.B, 1920)
    w = wide(c, 8192)
    s = w.score(25.0, "kept")
    ws = B.alloc_workspace(B.s4c_tree_attn_workspace_size(w.shape, z.max_len))
    lengths = [(1900, 5, 0, 1333, 64, 1900, 1), (0, 0, 1, 0, 0, 0, 0), (700, 1800, 1900, 1024, 64, 63, 1777)]
    want = []
    for n in lengths:
        w.len.copy_(torch.tensor(n, dtype=torch.int32))
        w.call(s, max_len=z.max_len, ws=ws)
        want.append((w.out.clone(), w.lse.clone()))
    graph = torch.cuda.CUDAGraph()
    run = lambda: B.s4c_tree_attn_scored(w.q, w.kt, w.vt, w.kc, w.vc, w.len, w.parent, z.max_len, s, w.out, w.lse, 0.0, w.status, ws)
    with torch.cuda.graph(graph):
        run()
    for i in (0, 1, 2, 0, 2, 1):
        w.len.copy_(torch.tensor(lengths[i], dtype=torch.int32))
        w.out.fill_(3.0)
        w.lse.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w.out, want[i][0]) and torch.equal(w.lse, want[i][1])
        run()
        assert torch.equal(w.out, want[i][0]) and torch.equal(w.lse, want[i][1])
