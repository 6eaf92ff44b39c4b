"""Attention kernels with changed scores keep what they hold in registers, as the unchanged ones do (no GPU)."""
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_resources import resources

# (a minute of compiling each, eight at a time: without the log-sum-exp's fp16 unit, and of the few-row ones that of most registers)
MANY = ["tree_attn_mfma_lse_bf16.hip"] + ["tree_attn_mfma_%s_%s.hip" % (kind, t) for kind in ("slopes", "cap", "cap_slopes") for t in ("bf16", "f16")]
FEW = ["tree_attn_smallm_scored_bf16.hip"]


@pytest.fixture(scope="module")
def found():
    with ThreadPoolExecutor(8) as pool:
        return dict(zip(FEW + MANY, pool.map(resources, FEW + MANY)))


@pytest.mark.parametrize("source", FEW + MANY)
def test_nothing_is_kept_in_scratch_memory(found, source):
    kernels = {k: v for k, v in found[source].items() if "tree_attn_" in k}
    assert kernels
    for name, r in kernels.items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize"] == 0, (name, r)


@pytest.mark.parametrize("source", MANY)
def test_many_row_kernels_are_as_lean_as_the_unchanged_ones(found, source):
    """The bounds of tests/test_resources.py: waves on a SIMD; scalar registers where one unit is walked (parts::kWhole, 0) or shares (kShares, 1)."""
    kernels = {k: v for k, v in found[source].items() if "tree_attn_mfma_kernel" in k}
    for name, r in kernels.items():
        assert r["Occupancy"] >= (1 if "kernelILi4E" in name and "ELi128E" in name else 2), (name, r)
    for merge, paged, most in ((0, False, 0), (0, True, 0), (1, False, 2), (1, True, 8)):
        lean = {k: v for k, v in kernels.items() if "5MergeE%dE" % merge in k and ("Lb1ELb%d" % source.endswith("_f16.hip") in k) == paged}
        assert len(lean) == 4, sorted(kernels)                # rows, head sizes
        for name, r in lean.items():
            assert r["SGPRs Spill"] <= most, (name, r)
