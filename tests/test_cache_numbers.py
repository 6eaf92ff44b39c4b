"""Numbers beyond 32 bits reach no entry point of a bounded cache as their low bits (no GPU)."""
from types import SimpleNamespace

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2506_14158_amd import binding as B
from paper_2506_14158_amd.verify import TreeVerifier
from tests.test_cache_errors import LY, Bn, D, Hkv, Hq, N, S, fakes

BIG = 1 << 32
CALLS = {
    "attention": lambda v, x: B.s4c_tree_attn_scored(x.q, x.tree, x.tree, x.cache, x.cache, x.n, x.parent, BIG + S, x.score, v.out, x.lse),
    "weights": lambda v, x: B.s4c_kv_weigh(x.q, x.cache, x.lse, x.n, x.path, x.n, BIG + S, x.score, x.w, x.w),
    "eviction": lambda v, x: B.s4c_kv_evict(x.caches, x.caches, x.ws, x.poss, x.n, x.n, BIG + 50, 5, x.ws, x.poss, x.n, v.evict_ws),
    "eviction, recent": lambda v, x: B.s4c_kv_evict(x.caches, x.caches, x.ws, x.poss, x.n, x.n, 50, BIG + 5, x.ws, x.poss, x.n, v.evict_ws),
    "workspace": lambda v, x: B.s4c_kv_evict_workspace_size(LY, Bn, Hkv, BIG + 50, S),
}


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up tensors of a device")
@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
@pytest.mark.parametrize("name", CALLS)
def test_refused(name):
    with FakeTensorMode():
        x = SimpleNamespace(**fakes(), score=B.PLAIN_SCORE)
        v = TreeVerifier(Bn, N, Hq, Hkv, D, S, 500, torch.bfloat16, 4, S, layers=LY, budget=50, recent=5)
        with pytest.raises(ValueError, match="beyond 32 bits"):
            CALLS[name](v, x)
