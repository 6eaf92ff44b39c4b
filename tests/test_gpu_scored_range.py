"""Changed scores at the ends of what the interface promises."""
import pytest
import torch

from tests.test_gpu_scored import Case

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


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
