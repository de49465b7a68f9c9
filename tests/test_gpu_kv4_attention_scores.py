"""Scores are sums of exact products in 32 bits: where every partial sum, in whatever order, is a number of 24 bits, the sum is exact.

All tokens of a context have the same key, so that a row's lse is its score + log n.  One product is +-2^8 (or one +2^8 and one
-2^8), all others odd multiples of 2^-10 up to 15 * 2^-10; every partial sum is a multiple of 2^-10 below 2^10.  (A sum that keeps 14 bits below
its largest term would lose all but the largest: an error of 2^-18 of it and more.)

What is left between score and lse: scale log2(e) (two roundings), the product with the score, the sum with log2 l, ln 2 and the product with
it, 2^-24 each: 6 * 2^-24 of the score's magnitude; the exponentials and the sum of up to 400 of them in chains of 16 tokens a page and
group and joins, 2^-23 and 2^-24 each of a number near 1, and log2's last bit: below 2^-18.
"""
import math

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq

pytestmark = pytest.mark.gpu
# kernel, parts, D: sequences, heads of the cache, heads of a group, rows of each sequence, max_kv
CALLS = {("few_16", 1): (8, 1, 16, 1, 500), ("few_16", 3): (8, 1, 4, 4, 1100), ("few_32", 1): (4, 1, 32, 1, 500), ("few_32", 3): (4, 2, 1, 32, 1100),
         ("one", 1): (2, 1, 1, 64, 384), ("pair", 1): (2, 1, 1, 128, 500), ("pair", 4): (2, 1, 1, 128, 1000), ("tall", 1): (4, 32, 1, 300, 500)}


@pytest.mark.parametrize("cancel", [False, True])
@pytest.mark.parametrize("n", [1, 70, 400])
@pytest.mark.parametrize("call,D", [(c, D) for c in CALLS for D in (64, 128) if c[0] != "tall" or D == 128])
def test_sums_of_exact_products(call, D, n, cancel):
    S, Hk, G, q, max_kv = CALLS[call]
    n = min(n, max_kv)
    got = brq.diag_kv4_attention_route(S * q, S, Hk * G, Hk, D, q, max_kv, False, 0, torch.cuda.get_device_properties(0).multi_processor_count)
    assert (got[0], got[1] > 1) == (call[0], call[1] > 1)
    g = torch.Generator().manual_seed(111)
    # keys of magnitude 1/2 ... 4 under a scale of 1, the same for all tokens; values of any kind
    codes = torch.randint(1, 7, (Hk, D), generator=g) + 8 * torch.randint(0, 2, (Hk, D), generator=g)
    codes[(codes & 7).remainder(2) == 1] = 1                                         # magnitudes 1.5 and 3: 1/2
    key = ref.GRID[codes & 7] * (1 - 2 * (codes >> 3))
    kc, ks, vc, vs = ref.page_index(D)
    pool = torch.randint(0, 256, (1, Hk, 68 * D), generator=g, dtype=torch.uint8)
    for h in range(Hk):
        pool[0, h][kc] = (codes[h, 0::2] | codes[h, 1::2] << 4).to(torch.uint8).expand(64, -1)
    pool[:, :, ks.flatten()], pool[:, :, vs.flatten()] = 127, 126
    assert torch.equal(ref.cache_values(pool.view(1, -1), Hk, D)[0][0], key.expand(64, Hk, D))
    # products: odd multiples of 2^-10, the large ones at every channel in turn
    T = S * q
    kq = key.repeat_interleave(G, 0).expand(T, Hk * G, D)
    small = (2 * torch.randint(0, 8, (T, Hk * G, D), generator=g) + 1).double() * (1 - 2 * torch.randint(0, 2, (T, Hk * G, D), generator=g)) * 2.0 ** -10
    at = (torch.arange(T)[:, None] * G + torch.arange(Hk * G)[None]).remainder(D)[..., None]
    products = small.scatter(2, at, 256.0)
    if cancel:
        products = products.scatter(2, (at + 1 + at.remainder(D - 1)).remainder(D), -256.0)
    x = (products / kq).to(torch.bfloat16)
    assert torch.equal(x.double() * kq, products)                                     # (powers of two apart: exact in 8 bits)
    table = torch.zeros((S, -(-n // 64)), dtype=torch.int32, device="cuda")
    lens = torch.full((S,), n, dtype=torch.int32, device="cuda")
    _, lse = brq.kv4_attention(x.cuda(), pool.view(1, -1).cuda(), table, lens, 1.0, False, cu_q=torch.arange(0, T + 1, q, dtype=torch.int32).cuda(),
                               max_q=q, max_kv=max_kv, want_lse=True)
    score = products.sum(-1)
    err = (lse.cpu().double() - score - math.log(n)).abs()
    bound = 6 * 2.0 ** -24 * (score.abs() + math.log(n)) + 2.0 ** -18
    assert (err <= bound).all(), float((err / bound).max())
