"""Attention of up to 32 rows is a weighted mean: values that are the same for all tokens come out as they are, to the last bit, however
the weights are rounded."""
import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sharp", [0.5, 2.0, 6.0, 20.0])
@pytest.mark.parametrize("q,G,n", [(1, 4, 3), (1, 4, 700), (4, 4, 700), (1, 16, 1100), (2, 16, 700), (32, 1, 1100), (1, 32, 4000)])
@pytest.mark.parametrize("D", [64, 128])
def test_equal_values(D, q, G, n, sharp):
    """An output is off by roundings in 32 bits alone, 2^-24 for each of some thousand steps at most, and then rounded to bf16, where a
    4-bit value under a power of two is a number: the nearest one."""
    g = torch.Generator().manual_seed(121)
    S, Hk, cols = 3, 2, -(-n // 64)
    pool = base.cache(g, S * cols, Hk, D).view(S * cols, Hk, 68 * D)
    kc, ks, vc, vs = ref.page_index(D)
    one = torch.randint(0, 256, (D // 2,), generator=g).to(torch.uint8)
    pool[:, :, vc], pool[:, :, vs] = one, torch.tensor([120 + i for i in range(D // 32)], dtype=torch.uint8)
    pool = pool.view(S * cols, -1)
    want = ref.cache_values(pool, Hk, D)[1][0, 0, 0]
    route, parts = brq.diag_kv4_attention_route(S * q, S, G * Hk, Hk, D, q, cols * 64, cus=torch.cuda.get_device_properties(0).multi_processor_count)
    assert route == ("few_16" if q * G <= 16 else "few_32")
    x = (torch.randn((S * q, G * Hk, D), generator=g) * sharp).to(torch.bfloat16)
    cu = torch.arange(0, S * q + 1, q, dtype=torch.int32)
    out = brq.kv4_attention(x.cuda(), pool.cuda(), torch.arange(S * cols, dtype=torch.int32).view(S, cols).cuda(),
                            torch.tensor([n, n, max(1, n // 2)], dtype=torch.int32).cuda(), cu_q=cu.cuda(), max_q=q)
    got = out.cpu().double()
    seen = torch.ones(S * q, dtype=torch.bool)
    for s, m in enumerate([n, n, max(1, n // 2)]):
        seen[s * q: s * q + max(0, q - m)] = False
    assert torch.equal(got[seen], want.expand(got[seen].shape)) and not got[~seen].any()
