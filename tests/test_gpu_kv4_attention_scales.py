"""Attention under scales down to those of the smallest numbers, and 0."""
import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [2.0 ** -103, -(2.0 ** -106), 2.0 ** -120])
@pytest.mark.parametrize("q", [1, 9, 70])
@pytest.mark.parametrize("D", [64, 128])
def test_small_scales_of_large_scores(D, q, scale):
    g = torch.Generator().manual_seed(71)
    pool = base.cache(g, 3, 1, D)
    table, lens = torch.tensor([[2, 0, 1]], dtype=torch.int32), [150]
    x = (torch.randn((q, 2, D), generator=g) * 2.0 ** 100).to(torch.bfloat16)
    cu = torch.tensor([0, q], dtype=torch.int32)
    out, lse = brq.kv4_attention(x.cuda(), pool.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), scale, cu_q=cu.cuda(), max_q=q, want_lse=True)
    base.check(out, ref.attention(x, ref.cache_values(pool, 1, D), table, lens, scale, True, 0, cu, q, 192), lse)


@pytest.mark.parametrize("q", [1, 70])
def test_a_scale_of_zero_weighs_all_tokens_alike(q):
    base_run = base.run(1, [q], [150], 2, 1, 64, seed=72, sharp=0.0)
    x, pool, table, cu, want, lse = base_run
    g = torch.Generator().manual_seed(73)
    x = torch.randn(x.shape, generator=g).to(torch.bfloat16)
    out, l2 = brq.kv4_attention(x.cuda(), pool.cuda(), table.cuda(), torch.tensor([150], dtype=torch.int32).cuda(), 0.0, cu_q=None if cu is None else cu.cuda(),
                                max_q=q, want_lse=True)
    assert torch.equal(out, want) and torch.equal(l2, lse)
