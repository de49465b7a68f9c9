"""The residual side's calls one after another, as a layer makes them: against 64 bits, in captured graphs, on other streams, at offsets past 32 bits.

A layer of [T, D] activations with weights [F, D] and [D, F]:
    a, h = add_rms_norm_rotate_quantize_fused(x, residual)       z = gelu(a . W1^T + b1)
    c = rotate_quantize_fused(z)                                 h <- c . W2^T + b2 + h
Tolerances, u = 2^-24: a product of K terms made and added in fp32 in any order is within (K + 1) u Sum |a w|; no activation's slope exceeds 1.13;
the activations' own bounds are the header's; each addition u of its result; the output's rounding half a step (bf16: 2^-8).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: U, BF16: 2.0 ** -8}
LUT = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


@pytest.fixture(scope="module")
def brq():
    import paper_2511_04214_amd as b
    b.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return b


def values(codes, scales):
    """What row-major operands stand for, in 64 bits."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    return LUT.to(codes.device)[c] * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def product(a, w, K):
    """a . w^T in 64 bits and what fp32 may be off by."""
    return a @ w.T, (K + 1) * U * (a.abs() @ w.abs().T)


class Layer:
    def __init__(self, brq, T, D, F, B=32, dtype=BF16, layout="tiled", seed=0):
        g = torch.Generator().manual_seed(seed + T + D + F)
        r = lambda *s: torch.randn(s, generator=g)                                       # noqa: E731
        self.brq, self.T, self.D, self.F, self.B, self.layout = brq, T, D, F, B, layout
        self.w = [brq.rotate_quantize_fused((r(n, k) / k ** 0.5).bfloat16().cuda(), B, layout=layout) for n, k in ((F, D), (D, F))]
        self.b = [r(n).cuda() for n in (F, D)]
        self.norm = (1 + 0.2 * r(D)).cuda()
        self.x, self.res = r(T, D).to(dtype).cuda(), r(T, D).to(dtype).cuda()

    def operands(self, a, w, rows, N, K):
        return dict(zip(("aq", "as_", "wq", "ws"), (*a, *w)), a_layout=self.layout, w_layout=self.layout, M=rows, N=N, K=K)

    def __call__(self, stream=None, seen=None):
        brq, T, D, F = self.brq, self.T, self.D, self.F
        c, s, h = brq.add_rms_norm_rotate_quantize_fused(self.x, self.B, residual=self.res, weight=self.norm, layout=self.layout, stream=stream)
        z = brq.mxfp4_gemm_epilogue(**self.operands((c, s), self.w[0], T, F, D), bias=self.b[0], activation="gelu", out_dtype=BF16, stream=stream)
        q = brq.rotate_quantize_fused(z, self.B, layout=self.layout, stream=stream)
        if seen is not None:
            seen.update(a=(c, s), h=h.clone(), z=z, q=q)
        return brq.mxfp4_gemm_epilogue(**self.operands(q, self.w[1], T, D, F), bias=self.b[1], residual=h, out=h, stream=stream)

    def rows(self, q, M, K):
        return values(*(q if self.layout == "rowmajor" else self.brq.to_rowmajor(*q, M, K)))


# one token, few, a batch in decoding, one whose second product is split along K, a ragged prompt; blocks as wide as a wavefront holds
@pytest.mark.parametrize("T,D,F,B,dtype,layout", [(1, 256, 1024, 32, BF16, "tiled"), (13, 512, 2048, 64, F32, "tiled"), (48, 256, 7168, 32, BF16, "tiled"), (130, 256, 7168, 32, BF16, "tiled"),
                                                  (300, 512, 1536, 512, BF16, "rowmajor"), (700, 544, 1056, 32, F32, "rowmajor")])
def test_layer(brq, T, D, F, B, dtype, layout):
    m = Layer(brq, T, D, F, B, dtype, layout)
    seen = {}
    y = m(seen=seen)
    h = (m.x.float() + m.res.float()).to(dtype)
    assert torch.equal(seen["h"], h) and y.dtype == dtype
    # the operand: codes of the norm's result, which the norm's own tests hold to its formula
    n, _ = brq.add_rms_norm(h, weight=m.norm, out_dtype=F32)
    want = brq.rotate_quantize_fused(n, B)
    assert torch.equal(m.rows(seen["a"], T, D), values(*want))
    w1, w2 = m.rows(m.w[0], F, D), m.rows(m.w[1], D, F)
    p, e = product(m.rows(seen["a"], T, D), w1, D)
    t = p + m.b[0].double()
    e = e + U * t.abs()
    z = 0.5 * t * torch.special.erfc(-t / math.sqrt(2.0))
    tol = 1.13 * e + (16 + 2 * t.square()) * U * z.abs()
    assert bool(((seen["z"].double() - z).abs() <= tol + 2.0 ** -8 * (z.abs() + tol)).all())
    p, e = product(m.rows(seen["q"], T, F), w2, F)
    t = p + m.b[1].double()
    want = t + h.double()
    tol = e + U * (t.abs() + want.abs())
    assert bool(((y.double() - want).abs() <= tol + HALF[dtype] * (want.abs() + tol)).all())


def test_graph(brq):
    """Captured and replayed with other inputs, eager work in between: every replay is the eager result.  Two graphs that were captured with
    one workspace take their turns."""
    layers = [Layer(brq, T, 256, 7168, seed=T) for T in (1, 48, 130)]
    for m in layers:
        m()
    shared = torch.empty(max(brq.mxfp4_gemm_epilogue_workspace(m.T, 256, 7168, "tiled", "tiled") for m in layers), dtype=torch.uint8, device="cuda")
    assert shared.numel() > 0
    torch.cuda.synchronize()
    graphs = []
    for m in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            seen = {}
            y = m(seen=seen)
            again = brq.mxfp4_gemm_epilogue(**m.operands(seen["q"], m.w[1], m.T, 256, 7168), bias=m.b[1], activation="silu", workspace=shared)
        graphs.append((g, m, y, again, seen["q"]))
    gen = torch.Generator().manual_seed(1)
    for turn in range(4):
        for g, m, y, again, q in graphs:
            m.x.copy_(torch.randn(m.x.shape, generator=gen).to(m.x.dtype))
            g.replay()
            torch.cuda.synchronize()
            got, got2 = y.clone(), again.clone()
            want = m()
            assert torch.equal(got, want), (turn, m.T)
            want2 = brq.mxfp4_gemm_epilogue(**m.operands(q, m.w[1], m.T, 256, 7168), bias=m.b[1], activation="silu")
            assert torch.equal(got2, want2), (turn, m.T)


def test_gradients_in_a_graph(brq):
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g).cuda()                                    # noqa: E731
    for M, K in ((1, 96), (333, 4096), (70, 16384)):
        x, res, gy, gh, w = r(M, K).bfloat16(), r(M, K).bfloat16(), r(M, K).bfloat16(), r(M, K).bfloat16(), 1 + 0.1 * r(K)

        def step():
            y, h = brq.add_rms_norm(x, residual=res, weight=w)
            return (y, h, *brq.add_rms_norm_backward(h, gy, gh=gh, weight=w))
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()
        for turn in range(3):
            x.copy_(r(M, K))
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip([o.clone() for o in outs], step()):
                assert torch.equal(a, b), (M, K, turn)


def test_other_streams(brq):
    """By argument and as the current stream, behind work of that stream that makes the inputs late."""
    side = torch.cuda.Stream()
    g = torch.Generator().manual_seed(3)
    for T in (1, 48, 300):
        m = Layer(brq, T, 256, 7168, seed=T)
        want = m().clone()
        gy, gh = (torch.randn(m.x.shape, generator=g).bfloat16().cuda() for _ in range(2))
        want_g = brq.add_rms_norm_backward(m.x, gy, gh=gh, weight=m.norm)
        x = m.x.clone()
        big = torch.ones(1 << 27, device="cuda")
        torch.cuda.synchronize()
        for by_argument in (True, False):
            m.x.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                for _ in range(4):
                    big.mul_(1.0)                    # some milliseconds before the inputs are there
                m.x.copy_(x)
                if not by_argument:
                    got = m()
                    got_g = brq.add_rms_norm_backward(m.x, gy, gh=gh, weight=m.norm)
            if by_argument:
                got = m(stream=side)
                got_g = brq.add_rms_norm_backward(m.x, gy, gh=gh, weight=m.norm, stream=side)
            side.synchronize()
            assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(got_g, want_g)), (T, by_argument)


def test_rows_far_apart(brq):
    """Pitches that put the last rows past 4 GiB: norms, gradients, the product's result and residual."""
    g = torch.Generator().manual_seed(4)
    M, K, pitch = 70, 96, 1 << 25                    # 70 rows of 64 MiB (bfloat16) and 128 MiB
    r = lambda *s, dt=BF16: torch.randn(s, generator=g).to(dt).cuda()                    # noqa: E731
    wide = {dt: torch.empty((M, pitch), dtype=dt, device="cuda") for dt in (BF16, F32)}
    x, res, w = r(M, K), r(M, K, dt=F32), r(K, dt=F32)
    fx, fr, fy = wide[BF16][:, :K], wide[F32][:, :K], wide[F32][:, 1024: 1024 + K]
    fx.copy_(x)
    fr.copy_(res)
    y0, h0 = brq.add_rms_norm(x, residual=res, weight=w, out_dtype=F32)
    y, h = brq.add_rms_norm(fx, residual=fr, weight=w, out=fy, h_out=fr)
    assert torch.equal(y, y0) and torch.equal(h, h0)
    q0, q = brq.add_rms_norm_rotate_quantize_fused(x, 32, residual=h0, weight=w), brq.add_rms_norm_rotate_quantize_fused(fx, 32, residual=fr, weight=w)
    assert all(torch.equal(a, b) for a, b in zip(q0, q))
    gy = r(M, K, dt=F32)
    want = brq.add_rms_norm_backward(h0, y0, gh=gy, weight=w)
    fr.copy_(h0)
    fg = wide[F32][:, 2048: 2048 + K]
    fg.copy_(gy)
    got = brq.add_rms_norm_backward(fr, fy, gh=fg, weight=w, dh=fg)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for rows, n, k in ((M, 96, 512), (M, 96, 7168), (40, 96, 96), (16, 96, 2048)):       # a tile, split along K, any K, few rows
        layer = Layer(brq, rows, k, n, seed=k)
        a = brq.rotate_quantize_fused(layer.x, 32, layout="tiled")
        kw = layer.operands(a, layer.w[0], rows, n, k)
        small = r(rows, n, dt=F32)
        far = wide[F32][M - rows:, :n]
        far.copy_(small)
        want = brq.mxfp4_gemm_epilogue(**kw, bias=layer.b[0], residual=small)
        assert torch.equal(brq.mxfp4_gemm_epilogue(**kw, bias=layer.b[0], residual=far, out=far), want)


def test_many_rows(brq):
    """More elements than 32 bits count: the last rows are as they are alone."""
    g = torch.Generator().manual_seed(5)
    M, K = (1 << 20) + 5, 4128
    x = torch.empty((M, K), dtype=BF16, device="cuda")
    x[:-9].fill_(0.5)
    x[-9:] = torch.randn((9, K), generator=g).bfloat16().cuda()
    w = (1 + 0.1 * torch.randn(K, generator=g)).cuda()
    y, h = brq.add_rms_norm(x, residual=x, weight=w)
    y0, h0 = brq.add_rms_norm(x[-9:], residual=x[-9:], weight=w)
    assert torch.equal(y[-9:], y0) and torch.equal(h[-9:], h0)
    assert torch.equal(y[:-9].amax(0), y[0]) and torch.equal(y[:-9].amin(0), y[0])
    dh, dw = brq.add_rms_norm_backward(h, y, gh=x, weight=w, dh=x)
    gh = torch.full((1, K), 0.5, dtype=BF16, device="cuda")
    want, _ = brq.add_rms_norm_backward(h[:1], y[:1], gh=gh, weight=w)
    assert torch.equal(dh[: M - 9].amax(0), want[0]) and torch.equal(dh[: M - 9].amin(0), want[0])
    # every row but nine adds the same; rounded sums of n terms of one sign are within n u: chains of rows and the parts' 65 + 64
    one = brq.add_rms_norm_backward(h[:1], y[:1], weight=w)[1].double()
    nine = brq.add_rms_norm_backward(h0, y0, weight=w)[1].double()
    parts = max(1, brq.add_rms_norm_backward_workspace(M, K) // (4 * K))
    chain = -(-M // parts) + 4 + -(-parts // 64) + 64
    total = (M - 9) * one
    assert bool(((dw.double() - total - nine).abs() <= (chain + 27 + 27 + 1) * U * (total.abs() + 9 * 40 * 8)).all())


def test_weights_past_two_gib(brq):
    """Weight codes past 2^31 bytes: the last columns, on the kernels for few rows, one tile and prompts."""
    N, K, last = 75020, 57344, 130
    g = torch.Generator(device="cuda").manual_seed(6)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8, device="cuda")
    scales = torch.randint(126, 129, (N, K // 32), generator=g, dtype=torch.uint8, device="cuda")
    assert codes.numel() > 1 << 31
    w = values(codes[-last:], scales[-last:])
    bias = torch.randn(N, generator=g, device="cuda")
    for M in (1, 16, 40, 300):
        aq = torch.randint(0, 256, (M, K // 2), generator=g, dtype=torch.uint8, device="cuda")
        sa = torch.randint(126, 129, (M, K // 32), generator=g, dtype=torch.uint8, device="cuda")
        a = values(aq, sa)
        y = brq.mxfp4_gemm_epilogue(aq, sa, codes, scales, bias=bias, activation="relu")
        p, e = product(a, w, K)
        t = p + bias[-last:].double()
        tol = e + U * t.abs()
        assert bool(((y[:, -last:].double() - t.clamp(min=0)).abs() <= tol).all()), M


def test_other_device_is_refused(brq):
    """Tensors that are not all on one GPU."""
    x, w = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.ones(64)
    for stream in (None, torch.cuda.current_stream()):
        for call in (lambda: brq.add_rms_norm(x, weight=w, stream=stream), lambda: brq.add_rms_norm(x, residual=x.cpu(), stream=stream),
                     lambda: brq.add_rms_norm_backward(x, x.cpu(), stream=stream), lambda: brq.add_rms_norm_rotate_quantize_fused(x, 32, weight=w, stream=stream)):
            with pytest.raises((ValueError, TypeError, RuntimeError)):
                call()
        a = brq.rotate_quantize_fused(x, 32)
        for kw in (dict(bias=torch.zeros(4)), dict(residual=torch.zeros((4, 4))), dict(out=torch.zeros((4, 4)))):
            with pytest.raises((ValueError, TypeError, RuntimeError)):
                brq.mxfp4_gemm_epilogue(*a, *a, stream=stream, **kw)
