"""Attention of many rows on each of its kernels, by name: every test first makes sure that its call takes the kernel it is about."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base
from kv4_forms import FORMS, GROUPED, NAN, plan
from test_gpu_kv4_attention_forms import lengths

pytestmark = pytest.mark.gpu
# heads of 64 have no tall tiles
KERNELS = [(form, D) for form in FORMS for D in (64, 128) if form != "tall" or D == 128]


def cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def runs(form, D, T, max_q, causal=True, window=0, forms=FORMS, G=1):
    route, parts = plan(form, D, forms, T, max_q, causal, window, G, cus())
    assert route == form.split()[0] and (parts > 1) == ("parts" in form and (window == 0 or window >= 500))


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 70), (True, 500), (True, (1 << 31) - 1), (False, 0)])
@pytest.mark.parametrize("form,D", KERNELS)
def test_ragged(form, D, causal, window):
    """Whole prompts, chunks, one page, no rows, no tokens, rows in front of the first token."""
    S, Hk, max_kv = FORMS[form]
    qs, lens = lengths(S, D)
    runs(form, D, sum(qs), max(qs), causal, window)
    base.run(S, qs, lens, Hk, Hk, D, causal, window, seed=101, max_kv=max_kv)


@pytest.mark.parametrize("form,D", KERNELS)
def test_heads_in_groups(form, D):
    S, Hk, max_kv = GROUPED[form]
    qs, lens = lengths(S, 102)
    runs(form, D, sum(qs), max(qs), forms=GROUPED, G=3)
    base.run(S, qs, lens, 3 * Hk, Hk, D, seed=102, sharp=4.0, spread=6, max_kv=max_kv)


@pytest.mark.parametrize("form,D", KERNELS)
def test_contexts_up_to_the_bound_and_past_it(form, D):
    """Odd and even numbers of pages, one token into a page, one short of it; more tokens than max_kv, more rows than max_q."""
    S, Hk, max_kv = FORMS[form]
    qs, lens = lengths(S, 103)
    lens[:4] = [max_kv, max_kv - 1, max_kv - 63, max_kv + 200]
    lens[10], lens[11] = max_kv - 64, max_kv // 2 + 1
    runs(form, D, sum(qs), 289)
    base.run(S, qs, lens, Hk, Hk, D, seed=103, max_kv=max_kv, max_q=289)


@pytest.mark.parametrize("form,D", KERNELS)
def test_pages_that_are_none_and_bytes_behind_the_end(form, D):
    """First, middle, last and all pages missing; what stands behind a context's end changes nothing."""
    g = torch.Generator().manual_seed(104)
    S, Hk, max_kv = FORMS[form]
    pool = base.cache(g, 40, Hk, D)
    table = torch.randint(0, 39, (S, 5), generator=g).to(torch.int32)
    table[0, 0], table[1, 1], table[2, 3], table[3], table[4, :3], table[6, 1:4] = -1, 40, 1 << 30, -1, -7, -1
    table[5] = torch.tensor([1, 2, 39, 0, 3])            # page 39: its one token, and what is behind it
    lens, qs = [256, 250, 320, 200, 256, 129, 320] + [100] * (S - 7), [70, 3, 90, 20, 5, 129, 140] + [2] * (S - 7)
    if form == "tall":
        qs[2], lens[2] = 280, 320
    runs(form, D, sum(qs), max(qs))
    cu = torch.tensor([0] + qs).cumsum(0).to(torch.int32)
    q = torch.randn((sum(qs), Hk, D), generator=g).to(torch.bfloat16)
    a = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    kw = dict(cu_q=cu.cuda(), max_q=max(qs), max_kv=max_kv, want_lse=True)
    out, lse = brq.kv4_attention(q.cuda(), pool.cuda(), *a, **kw)
    base.check(out, ref.attention(q, ref.cache_values(pool, Hk, D), table, lens, D ** -0.5, True, 0, cu, max(qs), max_kv), lse)
    bad = pool.clone().view(40, Hk, 68 * D)
    kc, ks, vc, vs = ref.page_index(D)
    for at, fill in ((kc, 0x77), (vc, 0xff), (ks, 0xff), (vs, 0xff)):
        bad[39][:, at[1:].flatten()] = fill
    again, l2 = brq.kv4_attention(q.cuda(), bad.view(40, -1).cuda(), *a, **kw)
    assert torch.equal(out, again) and torch.equal(lse, l2)


@pytest.mark.parametrize("form,D", KERNELS)
def test_repeats_strides_streams_and_graphs(form, D):
    S, Hk, max_kv = FORMS[form]
    qs, lens = lengths(S, 105)
    runs(form, D, sum(qs), max(qs))
    q, pool, table, cu, out, lse = base.run(S, qs, lens, Hk, Hk, D, seed=105, max_kv=max_kv)
    dev = [t.cuda() for t in (q, pool, table)] + [torch.tensor(lens, dtype=torch.int32).cuda()]
    a = dict(cu_q=cu.cuda(), max_q=max(qs), max_kv=max_kv, want_lse=True)
    wide = torch.zeros((q.shape[0], Hk + 3, D + 8), dtype=torch.bfloat16, device="cuda")
    wide[:, 1: Hk + 1, :D] = dev[0]
    got, l2 = brq.kv4_attention(wide[:, 1: Hk + 1, :D], *dev[1:], out=torch.empty((Hk, q.shape[0], D), dtype=torch.bfloat16, device="cuda").transpose(0, 1), **a)
    assert torch.equal(got, out) and torch.equal(l2, lse)
    for _ in range(5):
        got, l2 = brq.kv4_attention(*dev, **a)
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


@pytest.mark.parametrize("n", [1, 63, 64, 65, 128, 300, 380])
@pytest.mark.parametrize("form,D", KERNELS)
def test_a_nan_in_a_query_is_its_rows_alone(form, D, n):
    """In the first and the last row of a tile and of a sequence, and in between; every other row keeps its bits."""
    g = torch.Generator().manual_seed(106)
    S, Hk, max_kv, q = NAN[form]
    route, parts = brq.diag_kv4_attention_route(S * q, S, Hk, Hk, D, q, max_kv, False, 0, cus())
    assert route == form.split()[0] and (parts > 1) == ("parts" in form)
    cols = -(-n // 64)
    pool = base.cache(g, 10, Hk, D)
    table = torch.randint(0, 10, (S, cols), generator=g).to(torch.int32)
    x = torch.randn((S * q, Hk, D), generator=g).to(torch.bfloat16)
    a = (pool.cuda(), table.cuda(), torch.full((S,), n, dtype=torch.int32).cuda())
    kw = dict(cu_q=torch.arange(0, S * q + 1, q, dtype=torch.int32).cuda(), max_q=q, max_kv=max_kv, causal=False, want_lse=True)
    out, lse = brq.kv4_attention(x.cuda(), *a, **kw)
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    for t, h, d in ((0, 0, 0), (q - 1, Hk - 1, D - 1), (q + q // 2, 1, 7), (2 * q + min(q - 1, 255), 0, D // 2)):
        y = x.clone()
        y[t, h, d] = math.nan
        got, l2 = brq.kv4_attention(y.cuda(), *a, **kw)
        assert torch.isnan(got[t, h]).all() and torch.isnan(l2[t, h])
        keep = torch.ones((S * q, Hk), dtype=torch.bool, device="cuda")
        keep[t, h] = False
        assert torch.equal(got[keep], out[keep]) and torch.equal(l2[keep], lse[keep])
