"""Weights and eviction where there are many (sequence, KV head)s or long ones: runs of several steps, selection and moving in one launch."""
import copy

import numpy as np
import pytest
import torch

from oracle import cache_oracle as K
from paper_2506_14158_amd import binding as B
from tests.test_gpu_bounded_cache import Evict, Weigh, f64, host
from tests.test_gpu_scored import DT

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def long_weigh(seed, B_, Hkv, G, D, dtype, lengths, accepted, S_cap, page):
    """A Weigh with a cache of S_cap rows, drawn on the GPU."""
    c = Weigh(seed, B_, 8, Hkv * G, Hkv, D, dtype, lengths, accepted, page or 64, page, max_path=5)
    g = torch.Generator("cuda").manual_seed(seed)
    r = np.random.default_rng(seed)
    blocks = S_cap // page if page else 0
    c.kc = torch.empty(*((B_ * blocks + 1, Hkv, page, D) if page else (B_, Hkv, S_cap, D)), dtype=DT[dtype], device="cuda").normal_(generator=g)
    if page:
        c.table = torch.from_numpy(r.permutation(B_ * blocks + 1)[:B_ * blocks].reshape(B_, blocks).astype(np.int32)).cuda()
    c.S_cap = S_cap
    c.pos = torch.argsort(torch.rand(B_, Hkv, S_cap, generator=g, device="cuda"), -1).to(torch.int32)
    c.root = torch.full((B_,), S_cap, **I32)
    c.win = torch.rand(B_, Hkv, S_cap, generator=g, device="cuda")
    c.w = torch.full_like(c.win, 7.0)
    c.slopes = c.slopes / 64                    # distances of thousands of rows
    return c


def of_heads(c, kv):
    s = copy.copy(c)
    heads = [h for g in kv for h in range(g * c.G, (g + 1) * c.G)]
    s.q, s.lse, s.slopes = c.q[:, :, heads], c.lse[:, :, heads], c.slopes[heads]
    s.kc, s.win, s.pos = c.kc[:, kv], c.win[:, kv], c.pos[:, kv]
    return s


# B, Hkv, G, lengths (repeated), S_cap: on 256 CUs half tiles in runs of several steps (600 units of up to 12), whole tiles (more than 4096 steps in all)
STEPS = {
    "half tiles": (20, 30, 1, (1536, 1, 1291, 700, 129), 1536),
    "whole tiles": (8, 32, 4, (5001, 4096, 37, 2900, 5119), 5120),
    "whole tiles, one head": (8, 32, 1, (4999, 5120, 256, 257, 1025), 5120),
}


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", STEPS)
def test_weights_of_few_query_rows_over_several_steps(name, D, dtype, page):
    B_, Hkv, G, lengths, S_cap = STEPS[name]
    lengths = [lengths[b % len(lengths)] for b in range(B_)]
    accepted = [min(b % 5, n - 1) for b, n in enumerate(lengths)]
    c = long_weigh(sum(map(ord, name)) + D, B_, Hkv, G, D, dtype, lengths, accepted, S_cap, page)
    for i, (cap, bias) in enumerate(((0.0, "none"), (20.0, "kept"), (0.0, "rows"))):
        s = c.score(cap, bias)
        kv = [0, Hkv - 1, 7 + i]
        part = of_heads(c, kv)
        ps = part.score(cap, bias)
        want = part.want(ps)
        before = c.w.fill_(7.0).clone()
        c.call(s)
        assert not c.status.any()
        got_pos = None if s.key_pos is None else B.Score(cap, part.slopes, c.pos[:, kv], c.root)
        part.check(got_pos or ps, want, c.w[:, kv], before[:, kv])
    # in place: the same bits
    before = c.win.clone()
    c.call(s, in_place=True)
    for b, n in enumerate(lengths):
        assert torch.equal(c.win[b, :, :n], c.w[b, :, :n]) and torch.equal(c.win[b, :, n:], before[b, :, n:])


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("S_cap,budget,recent,weights", [(1408, 1024, 256, "spread"), (1408, 200, 64, "ties"), (5056, 2100, 333, "ties")])
def test_eviction_of_many_units(S_cap, budget, recent, weights, page):
    """As many units as two for every CU: who selects a unit's rows moves them too."""
    layers, Bn, Hkv = 16, 2, 16
    new = lambda: Evict(S_cap + budget, layers, Bn, Hkv, 64, "bf16", (S_cap - 7, S_cap // 2 + 55), S_cap, page, weights)
    c = new()
    c.check(budget, recent)
    apart = [c.rows(c.kc), c.rows(c.vc), c.w2, c.pos2, c.len2]
    c = new()
    c.run(budget, recent, in_place=True, kept=False)
    assert not c.status.any()
    n = c.len.tolist()
    for got, want in zip([c.rows(c.kc), c.rows(c.vc)], apart):
        assert torch.equal(got, want)
    for b in range(Bn):
        assert torch.equal(c.w[:, b, :, :n[b]], apart[2][:, b, :, :n[b]]) and torch.equal(c.pos[:, b, :, :n[b]], apart[3][:, b, :, :n[b]])
    assert torch.equal(c.len, apart[4])
