"""Parts of a long context are joined however many rows a call brings, rows that are no sequence's among them."""
import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_grid_has_workgroups():
    """2^24 rows, 2 of them a sequence's, over 72 pages: 9 parts, 40 GB of their sums."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    g = torch.Generator().manual_seed(95)
    T, D, n = 1 << 24, 64, 72 * 64
    pool, table = base.cache(g, 72, 1, D), torch.randperm(72, generator=g).to(torch.int32)[None]
    first = T - 5
    x = torch.randn((2, 1, D), generator=g).to(torch.bfloat16)
    try:
        q = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda")
        q[first: first + 2] = x.cuda()
        out, lse = torch.full((T, 1, D), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, 1), 9.0, device="cuda")
        brq.kv4_attention(q, pool.cuda(), table.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), cu_q=torch.tensor([first, first + 2], dtype=torch.int32).cuda(),
                          max_q=2, out=out, lse=lse)
        want = ref.attention(x, ref.cache_values(pool, 1, D), table, [n], D ** -0.5, True, 0, torch.tensor([0, 2]), 2, n)
        base.check(out[first: first + 2], want, lse[first: first + 2])
        assert bool((lse[:first] == 9.0).all()) and bool((lse[first + 2:] == 9.0).all()) and bool((out[:first] == 9.0).all())
    finally:
        del q, out, lse
        torch.cuda.empty_cache()
