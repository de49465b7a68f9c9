"""Infinities and NaN in values: what the cache makes of them, and rows that do not see their tokens."""
import math

import pytest
import torch

import paper_2511_04214_amd as brq

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def filled(D, n, v, Bv, dtype=BF16):
    """(pool, table, v as read back) of one sequence's n tokens with two heads."""
    g = torch.Generator().manual_seed(51)
    pages = -(-n // 64)
    pool = torch.zeros((pages, brq.kv4_page_bytes(2, D)), dtype=torch.uint8, device="cuda")
    k = torch.randn((n, 2, D), generator=g).to(dtype).cuda()
    slots = torch.arange(n, device="cuda")
    brq.kv4_append(pool, slots, k, v.to(dtype).cuda(), B=32, Bv=Bv)
    return pool, torch.arange(pages, dtype=torch.int32, device="cuda")[None], brq.kv4_read(pool, slots, D, out_dtype=torch.float32)[1]


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("Bv", [1, 32])
@pytest.mark.parametrize("D", [64, 128])
def test_values_in_the_cache_are_finite(D, Bv, bad):
    """A group that holds one saturates; the others are as they were."""
    g = torch.Generator().manual_seed(52)
    v = torch.randn((70, 2, D), generator=g)
    want = filled(D, 70, v, Bv)[2]
    v[66, 1, 37] = bad
    v[5, 0] = bad
    got = filled(D, 70, v, Bv)[2]
    assert torch.isfinite(got).all()
    keep = torch.ones((70, 2, D), dtype=torch.bool)
    keep[66, 1, 32:64] = False
    keep[5, 0] = False
    assert torch.equal(got[keep.cuda()], want[keep.cuda()])


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("q,n,at", [(4, 70, 67), (20, 130, 120), (100, 100, 70), (300, 300, 290), (40, 900, 880)])
@pytest.mark.parametrize("max_kv", [None, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_in_front_of_a_token_that_is_not_finite(D, max_kv, q, n, at, bad):
    """Rows at earlier positions do not see it, whatever page they share with it; nor do rows whose window it has left."""
    g = torch.Generator().manual_seed(53)
    v = torch.randn((n, 2, D), generator=g)
    x = torch.randn((q, 2, D), generator=g).to(BF16).cuda()
    a = dict(cu_q=torch.tensor([0, q], dtype=torch.int32, device="cuda"), max_q=q, max_kv=max_kv, want_lse=True)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    pool, table, _ = filled(D, n, v, 32)
    v[at, :, 3] = bad
    worse, _, _ = filled(D, n, v, 32)
    first = at - (n - q)                                    # the row at the token's own position
    for window in (0, 2):
        want, wl = brq.kv4_attention(x, pool, table, lens, window=window, **a)
        got, gl = brq.kv4_attention(x, worse, table, lens, window=window, **a)
        blind = torch.ones(q, dtype=torch.bool, device="cuda")
        blind[first: first + 2 if window else q] = False
        assert torch.isfinite(want).all() and torch.equal(got[blind], want[blind]) and torch.equal(gl, wl)
        assert not torch.equal(got[first], want[first])
