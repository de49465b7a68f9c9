"""add_rms_norm, its gradients and its fused form against the formulas in 64 bits.

Tolerances, with u = 2^-24 (one fp32 rounding) and half a step of the output's type on top (bf16: 2^-8):
  y    The sum of K squares: at most 8 C products in a lane's chain of C chunks of 8 (C <= 8: 64, then C - 1 sums), 6 sums over lanes, 15 over wavefronts, all of
       positive terms: (8 + 8 + 6 + 15 + 1) u < 40 u with the chain of 8 products per chunk.  The mean's division and eps 2 u, so the
       root's argument 42 u, its inverse root 21 u + 2 u (sqrt, within one step) + 1 u (division): 24 u.  Two products: 26 u.  Taken: 28 u |y|.
  dh   r (g - u mean): r 24 u, g = gy w 1 u, the difference and the product 2 u: 27 u r |g|.  u = h r 25 u, the mean of g u: its sum has as
       many roundings as that of squares and the products' two, of Sum |g h|: 42 u, times r 24 u, times 1 / K and roundings 3 u; then 25 + 42 + 27
       + the outer r, product and difference 27: 121 u.  Taken: 30 u r |g| + 130 u r |h r| mean |g h r| + 2 u |gh| + 1 u |dh|.
  dw   (n + 27) u Sum |gy h r| where n sums stand one behind the other: rows of a workgroup, its row groups (<= 4), every 64th row of partial
       sums, 64 of those.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def brq():
    import paper_2511_04214_amd as b
    b.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return b


def rand(g, *shape, dtype=F32, pitch=0):
    """Random values; `pitch`: rows of a buffer that is wider by so many."""
    t = torch.randn((*shape[:-1], shape[-1] + pitch), generator=g).to(dtype).cuda()
    return t[..., : shape[-1]]


def within(got, want, tol):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), "worst at %.3f of the tolerance" % float((err / tol.clamp(min=1e-300)).max())


def check_norm(y, h, w, eps, dtype):
    """y against the definition of the stored h."""
    h = h.double()
    want = h / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    want = want if w is None else want * w.double()
    within(y, want, (28 * U + (HALF[BF16] if dtype == BF16 else 0)) * want.abs() + 2.0 ** -126)


# one wavefront, parts of one, one element group; two to sixteen wavefronts, one to eight chunks a lane, ragged ends of each
KS = [32, 64, 480, 512, 544, 1024, 1056, 2016, 2048, 2080, 4096, 4128, 8192, 8224, 16384, 16416, 32736, 32768]
MS = [1, 2, 3, 5, 257]


@pytest.mark.parametrize("K", KS)
def test_norm_over_sizes(brq, K):
    g = torch.Generator().manual_seed(K)
    for M in MS:
        if M * K > 1 << 22 and M > 3:
            M = 4
        for xdt, rdt, ydt, weight, pitch in ((BF16, BF16, BF16, True, 0), (BF16, F32, BF16, True, 8), (F32, F32, F32, False, 16), (F32, BF16, F32, True, 0), (BF16, None, F32, True, 24)):
            print("case", M, K, xdt, rdt, ydt, weight, pitch, flush=True)
            x = rand(g, M, K, dtype=xdt, pitch=pitch)
            res = None if rdt is None else rand(g, M, K, dtype=rdt, pitch=pitch)
            w = 1 + 0.3 * rand(g, K) if weight else None
            y, h = brq.add_rms_norm(x, residual=res, weight=w, eps=1e-5, out_dtype=ydt)
            assert y.dtype == ydt and y.shape == x.shape
            if res is None:
                assert h is None
                h = x
            else:
                assert h.dtype == rdt and torch.equal(h, (x.float() + res.float()).to(rdt))
            check_norm(y, h, w, 1e-5, ydt)


def test_rows_that_are_special(brq):
    g = torch.Generator().manual_seed(0)
    K = 544
    x = rand(g, 9, K)
    x[1] = 0                                    # nothing but eps
    x[2] *= 1e-18                               # squares of 1e-36, eps far above
    x[3] *= 1e17                                # squares of 1e34: their sum is still finite
    x[4, 7] = float("nan")
    x[5, K - 1] = float("inf")
    x[6] = 0
    x[6, 3] = -2.0
    y, _ = brq.add_rms_norm(x, eps=1e-6)
    ok = [0, 1, 2, 3, 6, 7, 8]
    check_norm(y[ok], x[ok], None, 1e-6, F32)
    assert bool((y[1] == 0).all()) and bool(y[4].isnan().all())
    assert bool(y[5, K - 1].isnan()) and bool((y[5, : K - 1] == 0).all())                # inf / inf, and anything finite over it
    z, _ = brq.add_rms_norm(x, eps=0.0)
    assert bool(z[1].isnan().all())
    check_norm(z[[0, 2, 3, 6, 7, 8]], x[[0, 2, 3, 6, 7, 8]], None, 0.0, F32)


def test_in_place_and_guards(brq):
    """The sum in the residual's or x's place, the result over x; nothing beside the rows is written."""
    g = torch.Generator().manual_seed(1)
    for K in (96, 1120, 4096):
        w = rand(g, K)
        x0, r0 = rand(g, 7, K, dtype=BF16), rand(g, 7, K, dtype=BF16)
        y0, h0 = brq.add_rms_norm(x0, residual=r0, weight=w)
        for place in ("residual", "x", "out over x"):
            buf = [torch.full((9, K + 16), 3.0, dtype=BF16, device="cuda") for _ in range(3)]
            x, r, o = (b[1:8, 8: K + 8] for b in buf)
            x.copy_(x0)
            r.copy_(r0)
            y, h = brq.add_rms_norm(x, residual=r, weight=w, out=x if place == "out over x" else o, h_out=r if place == "residual" else x if place == "x" else None)
            assert torch.equal(y, y0) and torch.equal(h, h0)
            for b in buf:
                assert bool((b[0] == 3).all()) and bool((b[8] == 3).all()) and bool((b[:, :8] == 3).all()) and bool((b[:, K + 8:] == 3).all())
        y, h = brq.add_rms_norm(x0, residual=r0, weight=w, want_h=False)
        assert h is None and torch.equal(y, y0)
        y, h = brq.add_rms_norm(x0[:0], residual=r0[:0], weight=w)
        assert y.shape == h.shape == (0, K)


BLOCKS = [1, 8, 16, 32, 64, 128, 256, 512]


@pytest.mark.parametrize("B", BLOCKS)
def test_fused_is_the_two_calls(brq, B):
    """Codes and scales bit for bit, padding of K included; bytes of rows that do not exist are left alone."""
    g = torch.Generator().manual_seed(B)
    for M, K in ((1, max(B, 32)), (3, 1536), (65, 512 * 5), (300, 4096), (2, 8192), (5, B * 7 if B >= 32 else 224), (130, 16384)):
        for xdt, rdt, ydt, layout in ((BF16, BF16, F32, "tiled"), (F32, F32, BF16, "rowmajor"), (BF16, F32, BF16, "tiled"), (F32, None, F32, "rowmajor")):
            print("case", B, M, K, xdt, rdt, ydt, layout, flush=True)
            x, w = rand(g, M, K, dtype=xdt, pitch=8), 1 + 0.3 * rand(g, K)
            res = None if rdt is None else rand(g, M, K, dtype=rdt)
            signs = (torch.randint(0, 2, (K,), generator=g) * 2 - 1).to(torch.int8).cuda() if B > 1 and M != 3 else None
            y, h0 = brq.add_rms_norm(x, residual=res, weight=w, out_dtype=ydt)
            nc, ns = brq.operand_bytes(M, K, layout)
            shape = ((M, K // 2), (M, K // 32)) if layout == "rowmajor" else ((nc,), (ns,))
            want, got = ([torch.full(s, 0xA5, dtype=torch.uint8, device="cuda") for s in shape] for _ in range(2))
            if B == 1:
                brq.mxfp4_quantize(y, codes=want[0], scales=want[1], layout=layout)
            else:
                brq.rotate_quantize_fused(y, B, codes=want[0], scales=want[1], layout=layout, signs=signs)
            c, s, h = brq.add_rms_norm_rotate_quantize_fused(x, B, residual=res, weight=w, y_dtype=ydt, codes=got[0], scales=got[1], layout=layout, signs=signs)
            assert c is got[0] and s is got[1] and torch.equal(c, want[0]) and torch.equal(s, want[1])
            assert (h is None) == (rdt is None) and (h is None or torch.equal(h, h0))


def test_fused_makes_its_buffers(brq):
    g = torch.Generator().manual_seed(5)
    x, r = rand(g, 3, 96), rand(g, 3, 96)
    for layout in ("rowmajor", "tiled"):
        c, s, h = brq.add_rms_norm_rotate_quantize_fused(x, 32, residual=r, layout=layout, want_h=False)
        assert h is None
        y, _ = brq.add_rms_norm(x, residual=r)
        want = brq.rotate_quantize_fused(y, 32, layout=layout)
        if layout == "tiled":
            c, s = brq.to_rowmajor(c, s, 3, 96)
            want = brq.to_rowmajor(*want, 3, 96)
        assert torch.equal(c, want[0]) and torch.equal(s, want[1])


def backward_reference(h, gy, gh, w, eps):
    h, gy = h.double(), gy.double()
    K = h.shape[-1]
    r = 1 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    gw = gy if w is None else gy * w.double()
    u = h * r
    dh = r * (gw - u * (gw * u).mean(-1, keepdim=True))
    tol = 30 * U * r * gw.abs() + 130 * U * r * u.abs() * (gw * u).abs().mean(-1, keepdim=True)
    if gh is not None:
        dh, tol = dh + gh.double(), tol + 2 * U * gh.double().abs()
    return dh, tol + U * dh.abs(), (gy * u).sum(0), (gy * u).abs().sum(0)


def chain(brq, M, K):
    """Sums that stand one behind the other in dw."""
    parts = max(1, brq.add_rms_norm_backward_workspace(M, K) // (4 * K))
    return -(-M // parts) + 4 + -(-parts // 64) + 64


@pytest.mark.parametrize("K", KS)
def test_backward_over_sizes(brq, K):
    g = torch.Generator().manual_seed(K + 1)
    for M in (1, 2, 5, 333, 1500):
        if M * K > 1 << 22:
            M = min(M, 300 if K <= 16416 else 70)
        for hdt, gdt, other, weight, pitch in ((BF16, BF16, True, True, 0), (F32, BF16, True, True, 8), (F32, F32, False, True, 16), (BF16, F32, True, False, 0)):
            print("case", M, K, hdt, gdt, other, weight, pitch, flush=True)
            h, gy = rand(g, M, K, dtype=hdt, pitch=pitch), rand(g, M, K, dtype=gdt, pitch=pitch)
            gh, w = rand(g, M, K, dtype=hdt) if other else None, 1 + 0.3 * rand(g, K) if weight else None
            dh, dw = brq.add_rms_norm_backward(h, gy, gh=gh, weight=w, eps=1e-5)
            want, tol, wdw, scale = backward_reference(h, gy, gh, w, 1e-5)
            assert dh.dtype == hdt
            within(dh, want, tol + (HALF[BF16] * want.abs() if hdt == BF16 else 0) + 2.0 ** -126)
            if w is None:
                assert dw is None
            else:
                within(dw, wdw, (chain(brq, M, K) + 27) * U * scale + 2.0 ** -126)
            again = brq.add_rms_norm_backward(h, gy, gh=gh, weight=w, eps=1e-5)
            assert torch.equal(again[0], dh) and (dw is None or torch.equal(again[1], dw))


def test_backward_against_differences(brq):
    """Along random directions the loss moves as the gradients say: central differences of the definition in 64 bits."""
    g = torch.Generator().manual_seed(9)
    M, K, eps = 6, 160, 1e-3
    x, w, gy, gh = rand(g, M, K), 1 + 0.3 * rand(g, K), rand(g, M, K), rand(g, M, K)
    dh, dw = brq.add_rms_norm_backward(x, gy, gh=gh, weight=w, eps=eps)

    def loss(x, w):
        x, w = x.double(), w.double()
        return ((x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w) * gy.double()).sum() + (x * gh.double()).sum()
    for seed in range(4):
        d = torch.Generator().manual_seed(100 + seed)
        vx, vw = rand(d, M, K).double(), rand(d, K).double()
        t = 1e-4
        for slope, by in (((loss(x + t * vx, w) - loss(x - t * vx, w)) / (2 * t), (dh.double() * vx)), ((loss(x, w + t * vw) - loss(x, w - t * vw)) / (2 * t), (dw.double() * vw))):
            # t^2 / 6 of the third derivative (of order 1 an element) and 64-bit roundings over t: below 1e-6 of the terms; gradients 130 u
            assert abs(float(slope - by.sum())) <= 1e-5 * float(by.abs().sum())


def test_backward_special(brq):
    g = torch.Generator().manual_seed(2)
    K = 1056
    w = rand(g, K)
    h, gy, gh = (rand(g, 5, K, dtype=BF16) for _ in range(3))
    dh0, dw0 = brq.add_rms_norm_backward(h, gy, gh=gh, weight=w)
    buf = gh.clone()
    dh, dw = brq.add_rms_norm_backward(h, gy, gh=buf, weight=w, dh=buf)              # in the other gradient's place
    assert dh is buf and torch.equal(dh, dh0) and torch.equal(dw, dw0)
    out = torch.full((7, K + 8), 3.0, dtype=BF16, device="cuda")
    brq.add_rms_norm_backward(h, gy, gh=gh, weight=w, dh=out[1:6, :K])
    assert torch.equal(out[1:6, :K], dh0) and bool((out[0] == 3).all()) and bool((out[6] == 3).all()) and bool((out[:, K:] == 3).all())
    dh, dw = brq.add_rms_norm_backward(h[:0], gy[:0], gh=gh[:0], weight=w)
    assert dh.shape == (0, K) and bool((dw == 0).all())
    h[3] = 0                                                                          # a row of zeros: r = 1 / sqrt(eps)
    dh, dw = brq.add_rms_norm_backward(h, gy, gh=gh, weight=w, eps=1e-5)
    want, tol, wdw, scale = backward_reference(h, gy, gh, w, 1e-5)
    within(dh, want, tol + HALF[BF16] * want.abs())
    within(dw, wdw, (chain(brq, 5, K) + 27) * U * scale)
    ws = torch.empty(brq.add_rms_norm_backward_workspace(5, K), dtype=torch.uint8, device="cuda")
    again = brq.add_rms_norm_backward(h, gy, gh=gh, weight=w, eps=1e-5, workspace=ws)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dw)
    with pytest.raises(brq.BrqError):
        brq.add_rms_norm_backward(h, gy, gh=gh, weight=w, workspace=ws[:16])


def test_refused_tensors(brq):
    x, w = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        with pytest.raises(ValueError):
            brq.add_rms_norm(x, residual=x[:3], stream=stream)
        with pytest.raises((ValueError, brq.BrqError)):
            brq.add_rms_norm(x, residual=x[:1].expand(4, 64), stream=stream)              # rows on top of one another
        with pytest.raises(ValueError):
            brq.add_rms_norm(x, h_out=torch.empty_like(x), stream=stream)
        with pytest.raises(TypeError):
            brq.add_rms_norm(x, residual=x.clone(), h_out=torch.empty((4, 64), device="cuda"), stream=stream)
        with pytest.raises(ValueError):
            brq.add_rms_norm(x, weight=w[:32], stream=stream)
        with pytest.raises(TypeError):
            brq.add_rms_norm(x, weight=w.double(), stream=stream)
        with pytest.raises(TypeError):
            brq.add_rms_norm(x.half(), stream=stream)
        with pytest.raises(brq.BrqError):
            brq.add_rms_norm(x[:, :40], stream=stream)
        with pytest.raises(TypeError):
            brq.add_rms_norm_backward(x, x.clone(), gh=x.float(), stream=stream)
        with pytest.raises(TypeError):
            brq.add_rms_norm_rotate_quantize_fused(x, 32, y_dtype=torch.float16, stream=stream)
        with pytest.raises(brq.BrqError):
            brq.add_rms_norm_rotate_quantize_fused(x, 128, stream=stream)


def test_more_rows_than_a_launch_takes(brq):
    """More than 2^21 groups of rows: the rows on both sides of the border and the last ones are as they are alone, and no other row is missing."""
    g = torch.Generator().manual_seed(11)
    border, K = 1 << 23, 32                             # (four rows a workgroup)
    M = border + 6
    x = torch.full((M, K), 0.5, dtype=BF16, device="cuda")
    x[border - 5:] = rand(g, 11, K, dtype=BF16)
    w = rand(g, K)
    y, h = brq.add_rms_norm(x, residual=x, weight=w)
    q, s, _ = brq.add_rms_norm_rotate_quantize_fused(x, 32, residual=x, weight=w, want_h=False)
    for i, t in enumerate((y, h, q, s)):
        few = x[border - 6:].clone()
        assert torch.equal(t[border - 6:], (*brq.add_rms_norm(few, residual=few, weight=w), *brq.add_rms_norm_rotate_quantize_fused(few, 32, residual=few, weight=w)[:2])[i])
        assert torch.equal(t[: border - 5].amax(0), t[0]) and torch.equal(t[: border - 5].amin(0), t[0])
    T = border + 64                                     # tiled: whole slabs of 64 rows, K padded to 512 with zeros
    x = torch.full((T, K), 0.5, dtype=BF16, device="cuda")
    x[-70:] = rand(g, 70, K, dtype=BF16)
    codes, scales = (torch.full((T * n,), 255, dtype=torch.uint8, device="cuda") for n in (256, 16))
    brq.add_rms_norm_rotate_quantize_fused(x, 32, weight=w, codes=codes, scales=scales, layout="tiled")
    few = x[-128:].clone()
    c, s, _ = brq.add_rms_norm_rotate_quantize_fused(few, 32, weight=w, layout="tiled")
    assert torch.equal(codes[-c.numel():], c) and torch.equal(scales[-s.numel():], s)
    slabs = codes.view(-1, 64 * 256)[:-2]
    assert torch.equal(slabs.amax(0), slabs[0]) and torch.equal(slabs.amin(0), slabs[0])
