"""Attention of many rows in each of the forms a call can take: one group of wavefronts a tile (contexts of up to 6 pages), two that
share a tile's pages, tall tiles (where there are many).  The bound max_kv, not the lengths, says which, so the same small cases go
through all."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base

pytestmark = pytest.mark.gpu
# sequences, heads of the cache, max_kv
FORMS = {"one": (12, 2, 384), "pair": (12, 2, 500), "pair in parts": (12, 2, 1000), "tall": (130, 4, 1000)}


def lengths(S, seed):
    g = torch.Generator().manual_seed(seed)
    qs = torch.randint(1, 6, (S,), generator=g).tolist()
    lens = [n + int(torch.randint(0, 200, (1,), generator=g)) for n in qs]
    qs[3], lens[3] = 290, 290                            # a whole prompt, over more than one tile, an odd number of pages
    qs[4], lens[4] = 130, 384                            # an even number
    qs[5], lens[5] = 64, 64                              # one page
    qs[6], lens[6] = 0, 70                               # no rows
    qs[7], lens[7] = 5, 2                                # rows in front of the first token
    qs[8], lens[8] = 3, 0                                # no tokens
    qs[9], lens[9] = 20, 129                             # a token of the last page
    return qs, lens


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 70), (False, 0)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_ragged(form, D, causal, window):
    S, Hk, max_kv = FORMS[form]
    base.run(S, *lengths(S, D), Hk, Hk, D, causal, window, seed=31, max_kv=max_kv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_heads_in_groups(form, D):
    S, Hk, max_kv = FORMS[form]
    base.run(S, *lengths(S, 32), 3 * Hk, Hk, D, seed=32, sharp=4.0, max_kv=max_kv)
    base.run(S, *lengths(S, 33), 2 * Hk, Hk, D, seed=33, spread=6, max_kv=max_kv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_pages_that_are_none_and_bytes_behind_the_end(form, D):
    """First, middle, last and all pages missing; what stands behind a context's end changes nothing."""
    g = torch.Generator().manual_seed(34)
    S, Hk, max_kv = FORMS[form]
    pool = base.cache(g, 40, Hk, D)
    table = torch.randint(0, 39, (S, 5), generator=g).to(torch.int32)
    table[0, 0], table[1, 1], table[2, 3], table[3], table[4, :3], table[6, 1:4] = -1, 40, 1 << 30, -1, -7, -1
    table[5] = torch.tensor([1, 2, 39, 0, 3])            # page 39: its one token, and what is behind it
    lens, qs = [256, 250, 320, 200, 256, 129, 320] + [100] * (S - 7), [70, 3, 90, 20, 5, 129, 140] + [2] * (S - 7)
    cu = torch.tensor([0] + qs).cumsum(0).to(torch.int32)
    q = torch.randn((sum(qs), Hk, D), generator=g).to(torch.bfloat16)
    a = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    kw = dict(cu_q=cu.cuda(), max_q=140, max_kv=max_kv, want_lse=True)
    out, lse = brq.kv4_attention(q.cuda(), pool.cuda(), *a, **kw)
    base.check(out, ref.attention(q, ref.cache_values(pool, Hk, D), table, lens, D ** -0.5, True, 0, cu, 140, max_kv), lse)
    bad = pool.clone().view(40, Hk, 68 * D)
    kc, ks, vc, vs = ref.page_index(D)
    for at, fill in ((kc, 0x77), (vc, 0xff), (ks, 0xff), (vs, 0xff)):
        bad[39][:, at[1:].flatten()] = fill
    again, l2 = brq.kv4_attention(q.cuda(), bad.view(40, -1).cuda(), *a, **kw)
    assert torch.equal(out, again) and torch.equal(lse, l2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_repeats_strides_streams_and_graphs(form, D):
    S, Hk, max_kv = FORMS[form]
    qs, lens = lengths(S, 7)
    q, pool, table, cu, out, lse = base.run(S, qs, lens, 2 * Hk, Hk, D, seed=35, max_kv=max_kv)
    dev = [t.cuda() for t in (q, pool, table)] + [torch.tensor(lens, dtype=torch.int32).cuda()]
    a = dict(cu_q=cu.cuda(), max_q=max(qs), max_kv=max_kv, want_lse=True)
    wide = torch.zeros((q.shape[0], 2 * Hk + 3, D + 8), dtype=torch.bfloat16, device="cuda")
    wide[:, 1: 2 * Hk + 1, :D] = dev[0]
    got, l2 = brq.kv4_attention(wide[:, 1: 2 * Hk + 1, :D], *dev[1:], out=torch.empty((2 * Hk, q.shape[0], D), dtype=torch.bfloat16, device="cuda").transpose(0, 1), **a)
    assert torch.equal(got, out) and torch.equal(l2, lse)
    y, z = torch.zeros_like(out), torch.zeros_like(lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        brq.kv4_attention(*dev, out=y, lse=z, **a)
    for _ in range(3):
        y.zero_(), z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, out) and torch.equal(z, lse)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 128, 500])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_a_nan_in_a_query_is_its_rows_alone(form, D, n):
    g = torch.Generator().manual_seed(36)
    S, Hk, max_kv = FORMS[form]
    q, cols = 20, -(-n // 64)
    pool = base.cache(g, 10, Hk, D)
    table = torch.randint(0, 10, (S, cols), generator=g).to(torch.int32)
    x = torch.randn((S * q, Hk, D), generator=g).to(torch.bfloat16)
    a = (pool.cuda(), table.cuda(), torch.full((S,), n, dtype=torch.int32).cuda())
    kw = dict(cu_q=torch.arange(0, S * q + 1, q, dtype=torch.int32).cuda(), max_q=q, max_kv=max_kv, causal=False, want_lse=True)
    out, lse = brq.kv4_attention(x.cuda(), *a, **kw)
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    t = S * q // 2
    x[t, 1, 7] = math.nan
    got, l2 = brq.kv4_attention(x.cuda(), *a, **kw)
    assert torch.isnan(got[t, 1]).all() and torch.isnan(l2[t, 1])
    keep = torch.ones((S * q, Hk), dtype=torch.bool, device="cuda")
    keep[t, 1] = False
    assert torch.equal(got[keep], out[keep]) and torch.equal(l2[keep], lse[keep])


def test_few_long_sequences_among_many_short():
    """A grid sized by the rows, not by sequences times the longest: every tile of every sequence is reached, in more than 64 sequences."""
    S = 150
    qs, lens = [0] * S, [10] * S
    for s, n in ((0, 3), (63, 200), (64, 1), (65, 129), (149, 300)):
        qs[s], lens[s] = n, n + 30
    for max_kv in (384, 1000):
        base.run(S, qs, lens, 4, 2, 64, seed=37, max_kv=max_kv)
        base.run(S, qs, lens, 4, 2, 128, seed=37, max_kv=max_kv, window=100)


@pytest.mark.parametrize("window", [1, 300, 1000, 3000])
@pytest.mark.parametrize("D", [64, 128])
def test_windows_in_long_contexts(D, window):
    """Parts are counted by what a window shows; it stands anywhere in a context."""
    base.run(1, [1], [5000], 8, 2, D, window=window, seed=38)
    base.run(3, [1, 1, 1], [5000, 700, 64], 8, 2, D, window=window, seed=39)
    base.run(3, [4, 1, 0], [3000, 1100, 0], 8, 2, D, window=window, seed=40)
    base.run(2, [40, 3], [3000, 1100], 4, 1, D, window=window, seed=41)


@pytest.mark.parametrize("q,G", [(1, 17), (1, 32), (4, 8), (31, 1), (32, 1), (2, 16), (5, 6), (3, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_two_tiles_of_16_rows(D, q, G):
    """17 to 32 rows of a sequence; sequences with fewer, none, more than tokens; whole and in parts; in windows."""
    qs = [q, max(q - 1, 0), 1, 0, q, q, q, q]
    lens = [700, 65, 1, 30, max(q - 3, 0), 64, 0, 1800]
    base.run(8, qs, lens, 2 * G, 2, D, seed=42, sharp=2.0)
    base.run(8, qs, lens, 2 * G, 2, D, seed=43, window=100)
    base.run(8, qs, lens, 2 * G, 2, D, seed=44, causal=False, max_kv=1000)


@pytest.mark.parametrize("q,n", [(4, 200), (3, 3000)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_in_one_of_32_rows(D, q, n):
    g = torch.Generator().manual_seed(45)
    pool = base.cache(g, 50, 1, D)
    table = torch.randint(0, 50, (2, -(-n // 64)), generator=g).to(torch.int32)
    x = torch.randn((2 * q, 8, D), generator=g).to(torch.bfloat16)
    a = (pool.cuda(), table.cuda(), torch.full((2,), n, dtype=torch.int32).cuda())
    kw = dict(cu_q=torch.tensor([0, q, 2 * q], dtype=torch.int32).cuda(), max_q=q, want_lse=True)
    out, lse = brq.kv4_attention(x.cuda(), *a, **kw)
    x[q - 1, 3, 7] = math.nan
    got, l2 = brq.kv4_attention(x.cuda(), *a, **kw)
    assert torch.isnan(got[q - 1, 3]).all() and torch.isnan(l2[q - 1, 3])
    keep = torch.ones((2 * q, 8), dtype=torch.bool, device="cuda")
    keep[q - 1, 3] = False
    assert torch.equal(got[keep], out[keep]) and torch.equal(l2[keep], lse[keep])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S,q,Hk", [(70, 1, 8), (256, 1, 3), (100, 3, 8), (257, 1, 3), (65, 1, 16)])
def test_the_longest_sequences_first(S, q, Hk, D):
    """More sequences than fit at once, in the order of their lengths: equal lengths, none, less than none, more than the table has."""
    g = torch.Generator().manual_seed(46)
    lens = torch.randint(1, 200, (S,), generator=g).tolist()
    lens[:8] = [0, 3100, 64, 64, 64, 65, 63, 1]
    lens[10:14] = [-5, 3100, 3099, 128]
    base.run(S, [q] * S, lens, 2 * Hk if q == 1 else Hk, Hk, D, seed=47, max_kv=3500)
