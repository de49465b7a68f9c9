"""Head norms with position and block rotation, forward and backward, and the cache's write and read-back, against 64 bits."""
import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5
# roundings of 2^-24 on the way of a value, counted: at most 12 in the sum of 256 squares, 2 of the root, 3 of the norm, 3 of the
# rotation by position, 8 + 1 of the block rotation
STEPS = 32


def tables(rows, rot, g):
    a = torch.rand((rows, rot // 2), generator=g) * 6.3
    return a.cos(), a.sin()


def data(T, Hq, Hk, D, dtype, rot, norm, seed=0, rows=50):
    g = torch.Generator().manual_seed(seed + T * 7 + Hq + D)
    x = torch.randn((T, Hq + 2 * Hk, D), generator=g) * torch.exp(torch.randn((T, Hq + 2 * Hk, 1), generator=g))
    x = x.to(dtype)
    w = [1 + 0.5 * torch.randn(D, generator=g) if norm else None for _ in range(2)]
    cos, sin = tables(rows, rot, g) if rot else (None, None)
    pos = torch.randint(0, rows, (T,), generator=g) if rot else None
    return x, w, cos, sin, pos, g


def cu(*t):
    return [None if x is None else x.cuda() for x in t]


CASES = [(1, 1, 1, 64, 64, False, 1, True), (3, 7, 1, 64, 32, True, 8, True), (5, 4, 2, 128, 128, False, 32, True), (2, 32, 8, 128, 128, False, 128, True),
         (33, 5, 5, 128, 96, False, 16, True), (9, 3, 1, 128, 16, True, 64, True), (4, 2, 2, 256, 256, False, 256, True), (4, 2, 1, 256, 128, True, 128, False),
         (7, 9, 3, 64, 64, False, 64, False), (6, 8, 2, 128, 0, False, 32, True), (300, 4, 1, 64, 48, False, 1, True), (11, 1, 1, 256, 0, False, 1, False)]


@pytest.mark.parametrize("T,Hq,Hk,D,rot,inter,B,norm", CASES)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
def test_forward(T, Hq, Hk, D, rot, inter, B, norm, dtype, out):
    x, w, cos, sin, pos, _ = data(T, Hq, Hk, D, dtype, rot, norm)
    xd = x.cuda()
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    got = brq.qk_norm_rope(xd[:, :Hq], xd[:, Hq: Hq + Hk], wq, wk, EPS, c, s, p, inter, B, out_dtype=out)
    for y, a, b, weight in ((got[0], 0, Hq, w[0]), (got[1], Hq, Hq + Hk, w[1])):
        want, mag = ref.forward(x[:, a:b], weight, EPS, cos, sin, pos, inter, B)
        assert y.dtype == out
        err = (y.cpu().double() - want).abs()
        bound = STEPS * 2.0 ** -24 * mag + (2.0 ** -8 * want.abs() if out == BF16 else 0.0) + 1e-30
        assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("T,Hq,Hk,D,rot,inter,B,norm", CASES)
@pytest.mark.parametrize("dtype,gdt", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
def test_backward(T, Hq, Hk, D, rot, inter, B, norm, dtype, gdt):
    x, w, cos, sin, pos, g = data(T, Hq, Hk, D, dtype, rot, norm)
    gq, gk = (torch.randn((T, n, D), generator=g).to(gdt) for n in (Hq, Hk))
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    xd = x.cuda()
    dq, dk, dwq, dwk = brq.qk_norm_rope_backward(xd[:, :Hq], xd[:, Hq: Hq + Hk], gq.cuda(), gk.cuda(), wq, wk, EPS, c, s, p, inter, B)
    for dx, dw, gr, a, b, weight in ((dq, dwq, gq, 0, Hq, w[0]), (dk, dwk, gk, Hq, Hq + Hk, w[1])):
        want, mag, want_w, mag_w = ref.backward(x[:, a:b], gr, weight, EPS, cos, sin, pos, inter, B)
        err = (dx.cpu().double() - want).abs()
        bound = 2 * STEPS * 2.0 ** -24 * mag + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0) + 1e-30
        assert dx.dtype == dtype and (err <= bound).all(), float((err / bound).max())
        assert (dw is None) == (weight is None)
        if dw is not None:      # besides: no chain of additions is longer than the number of terms
            assert ((dw.cpu().double() - want_w).abs() <= (2 * STEPS + min(256, T * (b - a))) * 2.0 ** -24 * mag_w + 1e-30).all()


@pytest.mark.parametrize("inter,rot,B", [(False, 64, 32), (True, 32, 64)])
def test_backward_against_differences(inter, rot, B):
    T, Hq, Hk, D = 4, 3, 1, 64
    x, w, cos, sin, pos, g = data(T, Hq, Hk, D, F32, rot, True)
    gq = torch.randn((T, Hq, D), generator=g)
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    dq, _, dwq, _ = brq.qk_norm_rope_backward(x[:, :Hq].cuda(), None, gq.cuda(), None, wq, None, EPS, c, s, p, inter, B)
    assert brq.qk_norm_rope_backward(x[:, :Hq].cuda(), None, gq.cuda(), None, wq, None, EPS, c, s, p, inter, B)[1] is None

    def loss(xx, ww):
        return float((ref.forward(xx, ww, EPS, cos, sin, pos, inter, B)[0] * gq.double()).sum())
    h, x64, w64 = 1e-5, x[:, :Hq].double(), w[0].double()
    for _ in range(4):
        d, e = torch.randn(x64.shape, generator=g, dtype=torch.float64) * x64.abs(), torch.randn(D, generator=g, dtype=torch.float64)
        for got, num in ((dq.cpu().double() * d, (loss(x64 + h * d, w64) - loss(x64 - h * d, w64)) / (2 * h)),
                         (dwq.cpu().double() * e, (loss(x64, w64 + h * e) - loss(x64, w64 - h * e)) / (2 * h))):
            # differences: h^2 of truncation, 1e-16 / h of cancellation; gradients: 32 bits
            assert abs(float(got.sum()) - num) <= 1e-5 * float(got.abs().sum()) + 1e-8


def test_shared_and_strided_inputs():
    """One head given to all (stride 0), rows with gaps, outputs into views: as with contiguous copies."""
    T, H, D = 6, 4, 128
    x, w, cos, sin, pos, g = data(T, H, H, D, BF16, D, True)
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    xd = x.cuda()
    one = xd[:, :1].expand(T, H, D)
    wide = torch.zeros((T, 3 * H, D + 8), dtype=BF16, device="cuda")
    a = brq.qk_norm_rope(one, xd[:, 0::3], wq, wk, EPS, c, s, p, B=32, q_out=wide[:, H: 2 * H, :D], k_out=None)
    b = brq.qk_norm_rope(one.contiguous(), xd[:, 0::3].contiguous(), wq, wk, EPS, c, s, p, B=32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert int((wide[..., D:] != 0).sum()) == 0 and int((wide[:, :H] != 0).sum()) == 0
    heads_first = torch.empty((H, T, D), dtype=BF16, device="cuda").transpose(0, 1)
    assert torch.equal(brq.qk_norm_rope(one, None, wq, None, EPS, c, s, p, B=32, q_out=heads_first)[0], b[0])
    gq = torch.randn((T, 1, D), generator=g).to(BF16).cuda()
    d1 = brq.qk_norm_rope_backward(one, None, gq.expand(T, H, D), None, wq, None, EPS, c, s, p, B=32)
    d2 = brq.qk_norm_rope_backward(one.contiguous(), None, gq.expand(T, H, D).contiguous(), None, wq, None, EPS, c, s, p, B=32)
    assert torch.equal(d1[0], d2[0]) and torch.equal(d1[2], d2[2])


def test_positions_outside_the_tables_and_no_tokens():
    T, D = 5, 64
    x, w, cos, sin, pos, _ = data(T, 2, 1, D, BF16, D, True)
    pos = torch.tensor([0, -1, 49, 50, 1 << 40])
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    xd = x.cuda()
    q, k = brq.qk_norm_rope(xd[:, :2], xd[:, 2:3], wq, wk, EPS, c, s, p)
    for y in (q, k):
        assert torch.equal(torch.isnan(y).all(-1).all(-1).cpu(), torch.tensor([False, True, False, True, True]))
        assert not torch.isnan(y[[0, 2]]).any()
    pool = torch.zeros((2, brq.kv4_page_bytes(1, D)), dtype=torch.uint8, device="cuda")
    slots = torch.tensor([3, 4, 1000, 5, 6], device="cuda")                       # token 2: outside the cache
    assert torch.isnan(brq.kv4_append(pool, slots, xd[:, 2:3], xd[:, 3:4], q=xd[:, :2], wq=wq, wk=wk, eps=EPS, cos=c, sin=s, positions=p)[1]).all()
    kk, vv = brq.kv4_read(pool, torch.arange(-1, 130, device="cuda"), D)
    filled = (kk != 0).any(-1).any(-1).cpu()
    assert filled.nonzero().flatten().tolist() == [0, 4, 129, 130]                # slot 3, and the three that are NaN
    assert torch.isnan(kk[[0, 129, 130]]).all() and torch.isnan(vv[[0, 129, 130]]).all()
    e = xd[:0]
    q, k = brq.qk_norm_rope(e[:, :2], e[:, 2:3], wq, wk, EPS, c, s, p[:0])
    assert q.shape == (0, 2, D) and k.shape == (0, 1, D)
    dq, dk, dwq, dwk = brq.qk_norm_rope_backward(e[:, :2], e[:, 2:3], q, k, wq, wk, EPS, c, s, p[:0])
    assert dq.shape == (0, 2, D) and int((dwq != 0).sum()) == 0 and int((dwk != 0).sum()) == 0
    assert brq.kv4_append(pool, slots[:0], e[:, 2:3], e[:, 3:4]) is None
    assert brq.kv4_read(pool, slots[:0], D)[0].shape == (0, 1, D)


@pytest.mark.parametrize("T,Hq,Hk,D,rot,inter,B,Bv,norm", [
    (1, 4, 1, 128, 128, False, 32, 32, True), (130, 4, 2, 128, 64, True, 128, 1, True), (67, 7, 1, 64, 64, False, 64, 64, True),
    (200, 8, 8, 64, 0, False, 1, 8, False), (19, 5, 5, 128, 32, False, 8, 128, True)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_is_the_quantizer_behind_the_norm(T, Hq, Hk, D, rot, inter, B, Bv, norm, dtype):
    """Bit for bit: qk_norm_rope kept in 32 bits (block_rotate for values), then mxfp4_quantize; and where the bytes go."""
    x, w, cos, sin, pos, g = data(T, Hq, Hk, D, dtype, rot, norm, seed=3)
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    xd = x.cuda()
    q, k, v = xd[:, :Hq], xd[:, Hq: Hq + Hk], xd[:, Hq + Hk:]
    pages = (T + 63) // 64 + 2
    slots = torch.randperm(pages * 64, generator=g)[:T]
    before = torch.randint(0, 256, (pages, brq.kv4_page_bytes(Hk, D)), generator=g, dtype=torch.uint8)
    pool = before.cuda()
    qo = brq.kv4_append(pool, slots.cuda(), k, v, q=q, wq=wq, wk=wk, eps=EPS, cos=c, sin=s, positions=p, interleaved=inter, B=B, Bv=Bv)
    want_q, k32 = brq.qk_norm_rope(q, k, wq, wk, EPS, c, s, p, inter, B, out_dtype=F32)
    assert torch.equal(qo, want_q.to(dtype))
    v32 = v.reshape(T * Hk, D).float().contiguous()
    v32 = v32 if Bv == 1 else brq.block_rotate(v32, Bv)
    want = before.clone().view(pages, Hk, 68 * D)
    for y, (ci, si) in ((k32.reshape(T * Hk, D), ref.page_index(D)[:2]), (v32, ref.page_index(D)[2:])):
        codes, scales = (z.cpu().view(T, Hk, -1) for z in brq.mxfp4_quantize(y.contiguous()))
        for t in range(T):
            page, place = divmod(int(slots[t]), 64)
            want[page][:, ci[place]], want[page][:, si[place]] = codes[t], scales[t]
    assert torch.equal(pool.cpu().view(want.shape), want)
    all_k, all_v = ref.cache_values(want.view(pages, -1), Hk, D)
    for out in (BF16, F32):
        for got, all_ in zip(brq.kv4_read(pool, slots.cuda(), D, out_dtype=out), (all_k, all_v)):
            assert got.dtype == out and torch.equal(got.cpu().double(), all_.reshape(-1, Hk, D)[slots])


def test_largest_and_smallest_values_are_read_back_exactly():
    D = 64
    pool = torch.zeros((1, brq.kv4_page_bytes(1, D)), dtype=torch.uint8)
    kc, ks, vc, vs = ref.page_index(D)
    pool[0][kc] = torch.arange(64 * 32).reshape(64, 32).remainder(256).to(torch.uint8)
    pool[0][vc] = torch.arange(64 * 32).reshape(64, 32).mul(7).remainder(256).to(torch.uint8)
    pool[0][ks], pool[0][vs] = torch.arange(128).reshape(64, 2).mul(2).clamp(max=252).to(torch.uint8), torch.arange(128).reshape(64, 2).to(torch.uint8)
    want = ref.cache_values(pool, 1, D)
    for out in (F32, BF16):
        for got, w in zip(brq.kv4_read(pool.cuda(), torch.arange(64, device="cuda"), D, out_dtype=out), want):
            assert torch.equal(got.cpu().double(), w.reshape(64, 1, D))


def test_on_another_stream_and_in_a_graph():
    T, Hq, Hk, D = 37, 8, 2, 128
    x, w, cos, sin, pos, g = data(T, Hq, Hk, D, BF16, D, True)
    c, s, p, wq, wk = cu(cos, sin, pos, *w)
    xd = x.cuda()
    q, k, v = xd[:, :Hq], xd[:, Hq: Hq + Hk], xd[:, Hq + Hk:]
    gq, gk = torch.randn((T, Hq, D), generator=g).to(BF16).cuda(), torch.randn((T, Hk, D), generator=g).to(BF16).cuda()
    a = dict(wq=wq, wk=wk, eps=EPS, cos=c, sin=s, positions=p, B=32)
    slots = torch.randperm(64, generator=g)[:T].cuda()

    def step(pool, **kw):
        return [*brq.qk_norm_rope(q, k, **a, **kw), *brq.qk_norm_rope_backward(q, k, gq, gk, **a, **kw),
                brq.kv4_append(pool, slots, k, v, q=q, Bv=32, **a, **kw), *brq.kv4_read(pool, slots, D, **kw)]
    pool = torch.zeros((1, brq.kv4_page_bytes(Hk, D)), dtype=torch.uint8, device="cuda")
    want = step(pool)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(torch.zeros_like(pool).record_stream(side) or pool, stream=side)
    side.synchronize()
    assert all(torch.equal(y, z) for y, z in zip(got, want))
    graph, pool2 = torch.cuda.CUDAGraph(), torch.zeros_like(pool)
    with torch.cuda.graph(graph):
        out = step(pool2)
    for _ in range(3):
        for y in out:
            y.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, z) for y, z in zip(out, want))
