"""Changed scores at the ends of what the interface promises: the cap's tanh for both signs, values of V of any size."""
import numpy as np
import pytest
import torch

from paper_2506_14158_amd import binding as B
from tests.test_gpu_scored import DT, Case, f64

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def roots(dtype, N, Hq, Hkv, scores, cap, prefix):
    """The log-sum-exp of the roots, whose scores (of the one key that a root sees, or of `prefix` equal ones and itself) are given: [B][Hq]"""
    Bn, D = scores.shape[0], 64
    q = torch.zeros(Bn, N, Hq, D, dtype=dtype, device="cuda")
    q[:, 0, :, 0] = scores
    kt, vt = (torch.zeros(Bn, N, Hkv, D, dtype=dtype, device="cuda") for _ in range(2))
    kt[:, 0, :, 0] = 1.0
    kc, vc = (torch.zeros(Bn, Hkv, max(prefix, 1), D, dtype=dtype, device="cuda") for _ in range(2))
    kc[..., 0] = 1.0
    n = torch.full((Bn,), prefix, **I32)
    parent = torch.tensor([[-1] + [0] * (N - 1)] * Bn, **I32)
    shape = B.AttnShape(Bn, Hq, Hkv, D, N, max(prefix, 1), {torch.float32: B.S4C_F32, torch.bfloat16: B.S4C_BF16}[dtype])
    out, lse, status = torch.empty_like(q), torch.empty(Bn, N, Hq, device="cuda"), torch.ones(Bn, **I32)
    ws = B.alloc_workspace(max(256, B.s4c_tree_attn_workspace_size(shape, prefix)))
    B.s4c_tree_attn_scored(q, kt, vt, kc, vc, n, parent, prefix, B.Score(cap), out, lse, 1.0, status, ws)
    assert not status.any()
    return lse[:, 0]


def ladder(dtype, cap):
    """4096 different scores, from 2^-9 to 24 caps, most of them between 0.55 and 1.3, of either sign: [64][64]"""
    y = np.concatenate([np.linspace(0.55, 1.3, 1536), np.exp(np.linspace(np.log(2.0 ** -9), np.log(24.0), 512))])
    s = torch.from_numpy(np.concatenate([y, -y]) * cap).to(dtype).cuda()
    return s.view(64, 64)


@pytest.mark.parametrize("dtype,N", [("f32", 1), ("bf16", 70)])
@pytest.mark.parametrize("prefix", [0, 128])
def test_a_cap_is_odd_and_within_its_bound(dtype, N, prefix):
    """scale / cap is a power of two and a score one product, so that the cap's argument is exact.  One key: the log-sum-exp is the capped
    score, off by its tanh's 2^-22, by the rounding of the product that makes it natural (2^-24), and by those of log2(e) and ln 2 (1.4e-8 and 3e-9,
    relative).  129 equal keys (full tiles, whose scores are capped apart from the tree's): by the logarithm of their number beside it, with
    the sum's and the logarithm's own steps (2^-21 of the larger of the sum's terms)."""
    cap = 16.0
    s = ladder(DT[dtype], cap)
    got = f64(roots(DT[dtype], N, 64, 64, s, cap, prefix))
    x = cap * np.tanh(f64(s) / cap)
    bound = (2.0 ** -22 + 2.0 ** -24 + 1.7e-8) * np.abs(x)
    more = np.log(1.0 + prefix)
    err = np.abs(got - x - more)
    if prefix:
        bound = bound + 2.0 ** -21 * (np.abs(x) + more + 16.0)
    assert (err <= bound).all(), ((err / bound).max(), f64(s).flat[(err / bound).argmax()] / cap, (err / np.abs(x)).max())
    if not prefix:
        assert np.array_equal(got[:32], -got[32:])


@pytest.mark.parametrize("bias", ["rows", "kept"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("dtype,N", [("bf16", 80), ("bf16", 7), ("f32", 20)])
def test_values_of_any_size(dtype, N, cap, bias):
    """|V| up to 2^106, 448 keys: sums of them under steep slopes are as finite as without."""
    c = Case(31, 2, N, 4, 2, 128, dtype, (400, 129), 448)
    for t in (c.vt, c.vc):
        t.mul_(2.0 ** 104)
    if bias == "kept":
        c.pos = (1 << 30) + torch.arange(448, **I32).expand(2, 2, 448).contiguous()      # in order: the largest score is the last one's
        c.root = (1 << 30) + c.len
    c.call(c.score(cap, bias))
    assert bool(torch.isfinite(c.out).all())
    c.check(c.score(cap, bias))


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("bias", ["rows", "kept"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("dtype,N", [("bf16", 80), ("f16", 80), ("bf16", 7), ("f32", 20)])
def test_a_bias_that_decides_alone(dtype, N, cap, bias, sign):
    """Products with distances up to 2^22.6 (s4c.h: 2^23): a row's output is the value of its last key (its own), or of the first one.  Its exponential may be as far
    from 1 as a product's rounding, and is rounded to the storage type, as the output is (half a step each)."""
    c = Case(32, 2, N, 4, 2, 128, dtype, (300, 129), 320)
    c.slopes = torch.full((4,), sign * 2.0 ** 14, device="cuda")
    if bias == "kept":
        c.pos = (1 << 30) + torch.arange(320, **I32).expand(2, 2, 320).contiguous()
        c.root = (1 << 30) + c.len
    c.call(c.score(cap, bias))
    want = (c.vt if sign > 0 else c.vc[:, :, :1].transpose(1, 2).expand(2, N, 2, 128)).repeat_interleave(2, 2).double()
    step = torch.finfo(DT[dtype]).eps / 2
    assert bool(((c.out.double() - want).abs() <= 2.01 * step * want.abs()).all())
    if sign > 0 and bias == "kept":
        c.call(c.score(cap, "rows"))              # the same positions
        assert bool(((c.out.double() - want).abs() <= 2.01 * step * want.abs()).all())
