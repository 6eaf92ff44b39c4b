"""A step of several layers over a bounded cache, as README.md shows it, with a sequence whose cache is full."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as K
from paper_2506_14158_amd import binding as s4c
from paper_2506_14158_amd.verify import TreeVerifier
from tests.test_gpu_scored import f64

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def host(t):
    return t.cpu().numpy()


def test_a_sequence_whose_rows_do_not_fit_is_left_as_it_is():
    layers, B, N, Hq, Hkv, D, S_cap, V, budget, recent = 2, 3, 5, 4, 2, 64, 48, 40, 32, 8
    g = torch.Generator().manual_seed(1)
    f = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    q, k_tree, v_tree = f(layers, B, N, Hq, D), f(layers, B, N, Hkv, D), f(layers, B, N, Hkv, D)
    k_cache, v_cache = f(layers, B, Hkv, S_cap, D), f(layers, B, Hkv, S_cap, D)
    cache_len = torch.tensor([20, 46, 43], **I32)                 # five rows: 25, no room, full to the last row
    parent = torch.tensor([[-1, 0, 1, 2, 3]] * B, **I32)
    logits = f(B, N, V)
    tokens = torch.zeros(B, N, **I32)
    tokens[:, 1:] = logits[:, :-1].float().argmax(-1).to(torch.int32)          # the whole chain is accepted
    pos = torch.arange(S_cap, **I32).repeat(layers, B, Hkv, 1) + 7
    root_pos = cache_len + 7
    totals = torch.rand(layers, B, Hkv, S_cap, generator=g).cuda()
    lse, out = torch.empty(layers, B, N, Hq, device="cuda"), torch.empty(B, N, Hq, D, dtype=torch.bfloat16, device="cuda")
    cap, slopes = 10.0, torch.tensor([0.25, 0.125, 0.0625, 0.03125], device="cuda")
    before = [t.clone() for t in (k_cache, v_cache, totals, pos, root_pos)]

    tv = TreeVerifier(B, N, Hq, Hkv, D, S_cap, V, torch.bfloat16, N, S_cap, layers=layers, budget=budget, recent=recent)
    scores = [s4c.Score(cap, slopes, pos[l], root_pos) for l in range(layers)]
    for l in range(layers):
        tv.tree_attn_scored(q[l], k_tree[l], v_tree[l], k_cache[l], v_cache[l], cache_len, parent, scores[l], out=out, lse=lse[l])
    tv.accept_path(logits, parent, tokens, s4c.S4C_GREEDY)
    assert tv.accept_len.tolist() == [4, 4, 4]
    tv.commit_path(k_tree, v_tree, k_cache, v_cache, cache_len)
    tv.accept_len.masked_fill_(tv.compact_status != 0, -1)
    weighed = []
    for l in range(layers):
        weighed.append(K.kv_weigh(f64(q[l]), f64(k_cache[l]), f64(lse[l]), host(cache_len), host(tv.path), host(tv.accept_len), f64(totals[l]), 0.0, cap,
                                  f64(slopes), host(pos[l]), host(root_pos)))
        tv.kv_weigh(q[l], k_cache[l], cache_len, scores[l], totals[l], lse=lse[l])
    root_pos += tv.accept_len + 1

    assert tv.compact_status.tolist() == tv.weigh_status.tolist() == [0, s4c.S4C_SEQ_BAD_LEN, 0]
    assert cache_len.tolist() == [25, 46, 48] and root_pos.tolist() == [32, 53, 55]
    for now, then in zip((k_cache, v_cache, totals, pos), before):
        assert torch.equal(now[:, 1], then[:, 1])
    for l in range(layers):
        for b, n in ((0, 25), (2, 48)):
            assert np.allclose(f64(totals[l])[b, :, :n], weighed[l][0][b, :, :n], rtol=1e-4, atol=1e-5)
            assert np.array_equal(host(pos[l, b]), weighed[l][1][b])

    kept, new_len = K.kv_evict(f64(totals), host(pos), host(cache_len), host(root_pos), budget, recent)
    tv.kv_evict(k_cache, v_cache, totals, pos, cache_len, root_pos)
    assert not tv.evict_status.any()
    assert np.array_equal(host(tv.kept), kept) and np.array_equal(host(cache_len), new_len) and new_len.tolist() == [25, 32, 32]
