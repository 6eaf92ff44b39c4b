"""The sizes of tests/test_gpu_scored_shares.py are divided into balanced shares that end inside units (csrc/attn_division.h on the host: no GPU)."""
import subprocess

import pytest

from paper_2506_14158_amd import binding as B
from tests.test_attn_division import player  # noqa: F401
from tests.test_gpu_division import plan_inputs
from tests.test_gpu_scored_shares import SHARES


@pytest.mark.parametrize("case", SHARES, ids=lambda c: c.name)
def test_shares_are_balanced(player, case):  # noqa: F811
    r = subprocess.run([player, "plan"] + [str(x) for x in plan_inputs(case)], capture_output=True, text=True, check=True)
    teams, split, parts = (int(x) for x in r.stdout.split())
    assert split == 0 and parts > 1 and teams > case.B * case.Hkv // 2, r.stdout
    code = {"f32": B.S4C_F32, "bf16": B.S4C_BF16, "f16": B.S4C_F16}[case.dtype]
    shape = B.AttnShape(case.B, case.Hkv * case.G, case.Hkv, case.D, case.N, case.max_len, code)
    assert B.s4c_tree_attn_num_splits(shape, case.max_len) == parts
