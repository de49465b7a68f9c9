"""Attention over the cache where a call has a tile of 256 rows for every CU (many heads of the cache, many sequences), and rows
that hold NaN."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base

pytestmark = pytest.mark.gpu


def lengths(S, seed):
    g = torch.Generator().manual_seed(seed)
    qs = torch.randint(1, 6, (S,), generator=g).tolist()
    lens = [n + int(torch.randint(0, 200, (1,), generator=g)) for n in qs]
    qs[3], lens[3] = 300, 300                            # a whole prompt, over more than one tile
    qs[5], lens[5] = 64, 64
    qs[6], lens[6] = 0, 70                               # no rows
    qs[7], lens[7] = 5, 2                                # rows in front of the first token
    qs[8], lens[8] = 3, 0                                # no tokens
    qs[9], lens[9] = 20, 129
    return qs, lens


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 70), (False, 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_ragged(D, causal, window):
    qs, lens = lengths(130, D)
    run = base.run(130, qs, lens, 2, 2, D, causal, window, seed=21)
    assert run[0].shape[0] == sum(qs)


@pytest.mark.parametrize("D", [64, 128])
def test_heads_in_groups(D):
    qs, lens = [300] + [7] * 63, [513] + list(range(7, 70))
    base.run(64, qs, lens, 12, 4, D, seed=22, sharp=4.0)
    base.run(64, qs, lens, 12, 4, D, seed=23, spread=6, max_kv=300)


@pytest.mark.parametrize("D", [64, 128])
def test_pages_that_are_none_and_bytes_behind_the_end(D):
    """First, middle and last pages missing, all of a sequence's; what stands behind a context's end changes nothing."""
    g = torch.Generator().manual_seed(24)
    S, Hk = 130, 2
    pool = base.cache(g, 40, Hk, D)
    table = torch.randint(0, 39, (S, 4), generator=g).to(torch.int32)
    table[0, 0], table[1, 1], table[2, 3], table[3], table[4, :3] = -1, 40, 1 << 30, -1, -7
    lens = [256, 250, 256, 200, 256, 129] + [100] * (S - 6)
    qs = [70, 3, 90, 20, 5, 129] + [2] * (S - 6)
    table[5] = torch.tensor([1, 2, 39, 0])               # page 39: its one token, and what is behind it
    cu = torch.tensor([0] + qs).cumsum(0).to(torch.int32)
    q = torch.randn((sum(qs), Hk, D), generator=g).to(torch.bfloat16)
    a = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    kw = dict(cu_q=cu.cuda(), max_q=129, want_lse=True)
    out, lse = brq.kv4_attention(q.cuda(), pool.cuda(), *a, **kw)
    base.check(out, ref.attention(q, ref.cache_values(pool, Hk, D), table, lens, D ** -0.5, True, 0, cu, 129, 256), lse)
    bad = pool.clone().view(40, Hk, 68 * D)
    kc, ks, vc, vs = ref.page_index(D)
    for at, fill in ((kc, 0x77), (vc, 0xff), (ks, 0xff), (vs, 0xff)):
        bad[39][:, at[1:].flatten()] = fill
    again, l2 = brq.kv4_attention(q.cuda(), bad.view(40, -1).cuda(), *a, **kw)
    assert torch.equal(out, again) and torch.equal(lse, l2)


@pytest.mark.parametrize("D", [64, 128])
def test_repeats_strides_and_graphs(D):
    qs, lens = lengths(130, 7)
    q, pool, table, cu, out, lse = base.run(130, qs, lens, 2, 2, D, seed=25)
    dev = [t.cuda() for t in (q, pool, table)] + [torch.tensor(lens, dtype=torch.int32).cuda()]
    a = dict(cu_q=cu.cuda(), max_q=max(qs), want_lse=True)
    wide = torch.zeros((q.shape[0], 5, D + 8), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:3, :D] = dev[0]
    got, l2 = brq.kv4_attention(wide[:, 1:3, :D], *dev[1:], out=torch.empty((2, q.shape[0], D), dtype=torch.bfloat16, device="cuda").transpose(0, 1), **a)
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


@pytest.mark.parametrize("S,q,n", [(2, 1, 100), (1, 1, 5000), (2, 40, 100), (1, 30, 3000), (130, 20, 70)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_in_a_query_is_its_rows_alone(S, q, n, D):
    g = torch.Generator().manual_seed(26)
    Hk = 2
    cols = -(-n // 64)
    pool = base.cache(g, S * cols, Hk, D)
    table = torch.arange(S * cols, dtype=torch.int32).view(S, cols)
    x = torch.randn((S * q, 4, D), generator=g).to(torch.bfloat16)
    a = (pool.cuda(), table.cuda(), torch.full((S,), n, dtype=torch.int32).cuda())
    kw = dict(cu_q=None if q == 1 else torch.arange(0, S * q + 1, q, dtype=torch.int32).cuda(), max_q=q, want_lse=True)
    out, lse = brq.kv4_attention(x.cuda(), *a, **kw)
    t = S * q // 2
    x[t, 1, 7] = math.nan
    got, l2 = brq.kv4_attention(x.cuda(), *a, **kw)
    assert torch.isnan(got[t, 1]).all() and torch.isnan(l2[t, 1])
    keep = torch.ones((S * q, 4), dtype=torch.bool, device="cuda")
    keep[t, 1] = False
    assert torch.equal(got[keep], out[keep]) and torch.equal(l2[keep], lse[keep])
