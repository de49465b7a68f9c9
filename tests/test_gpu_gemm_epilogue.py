"""mxfp4_gemm_epilogue on every kernel that takes it, by name, and through the dispatcher, against the formula in 64 bits.

The operands' scales are powers of two from 1/2 to 2 and K stays below 7200, so every partial sum of the product is a multiple of 2^-4 below 2^20: exact in fp32
in any order.  Biases and residuals are multiples of 2^-4 too where a bit-for-bit result is asked.  So
  none, relu   p + bias is exact; the residual's addition is one fp32 operation, then the output's rounding: compared with the same two roundings, bit for bit
  silu, gelu   u = 2^-24: (8 + 2 |t|) u |silu(t)| + 2^-119 |t| and (16 + 2 t^2) u |gelu(t)| + 2^-118 as the header states, u of the sum with the residual,
               half a step of the output (bf16: 2^-8)
"""
import math

import numpy as np
import pytest
import torch

from gpu_util import to_dev
from test_gpu_layout import to_tiled

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
LUT = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])
LAYOUTS = [("rowmajor", "rowmajor"), ("tiled", "tiled"), ("tiled", "rowmajor"), ("rowmajor", "tiled")]
GUARD = -7.0


@pytest.fixture(scope="module")
def brq():
    import paper_2511_04214_amd as b
    b.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return b


def operand(seed, rows, K):
    """(codes, scales) row-major and their values."""
    r = np.random.default_rng(seed)
    c = r.integers(0, 16, (rows, K), dtype=np.uint8)
    c[c == 8] = 0
    s = r.integers(126, 129, (rows, K // 32), dtype=np.uint8)
    v = LUT[c] * np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, 1)
    return (c[:, 0::2] | (c[:, 1::2] << 4), s), v


class Case:
    def __init__(self, M, N, K, seed=0):
        (a, va), (w, vw) = operand(seed + 1, M, K), operand(seed + 2, N, K)
        self.M, self.N, self.K = M, N, K
        self.a = {"rowmajor": [to_dev(t) for t in a], "tiled": [to_dev(t) for t in to_tiled(*a)]}
        self.w = {"rowmajor": [to_dev(t) for t in w], "tiled": [to_dev(t) for t in to_tiled(*w)]}
        self.p = torch.from_numpy(va @ vw.T).cuda()
        g = torch.Generator().manual_seed(seed)
        self.bias = (torch.randint(-64, 65, (N,), generator=g) / 16.0).float().cuda()
        self.res = {dt: (torch.randn((M, N), generator=g) * 40).to(dt).cuda() for dt in (F32, BF16)}

    def want(self, bias, act, res, dt, scale=1.0):
        """(exact result, tolerance; 0: bit for bit)"""
        t = self.p if not bias else self.p + self.bias.double()
        r = None if res is None else self.res[res]
        if act in (None, "relu"):
            t = t.clamp(min=0) if act else t
            f = t.float()
            assert torch.equal(f.double(), t)
            return ((f if r is None else f + r.float()).to(dt)).double(), torch.zeros((), dtype=torch.float64, device="cuda")
        if act == "silu":
            y = t / (1 + (-t).exp())
            tol = (8 + 2 * t.abs()) * U * y.abs() + 2.0 ** -119 * t.abs()
        else:
            y = 0.5 * t * torch.special.erfc(-t / math.sqrt(2.0))
            tol = (16 + 2 * t.square()) * U * y.abs() + 2.0 ** -118
        if r is not None:
            y = y + r.double()
            tol = tol + U * y.abs()
        return y, tol + (2.0 ** -8 if dt == BF16 else U) * y.abs() + 2.0 ** -126

    def check(self, call, bias, act, res, dt, pad=0, in_place=False):
        M, N = self.M, self.N
        buf = torch.full((M + 2, N + pad), GUARD, dtype=dt, device="cuda")
        out = buf[:M, :N]
        r = None
        if res is not None:
            if in_place:
                out.copy_(self.res[res])
                r = out
            else:                                       # a residual of another pitch
                wide = torch.zeros((M, N + 3), dtype=res, device="cuda")
                wide[:, :N] = self.res[res]
                r = wide[:, :N]
        y = call(out, self.bias if bias else None, act, r)
        assert y is out
        assert bool((buf[M:] == GUARD).all()) and bool((buf[:, N:] == GUARD).all()), "wrote outside the M x N block"
        want, tol = self.want(bias, act, res, dt)
        err = (out.double() - want).abs()
        assert bool((err <= tol).all()), "%d off, worst %g (at %g)" % (int((err > tol).sum()), float((err - tol).max()), float(want.flatten()[(err - tol).argmax()]))
        return out


FORMS = [(True, None, BF16, BF16), (True, "gelu", None, BF16), (False, "silu", F32, F32), (True, "relu", BF16, F32), (False, None, F32, BF16), (True, "gelu", F32, F32),
         (False, "relu", None, F32), (True, "silu", BF16, BF16), (False, None, None, BF16)]


def on_route(brq, route, c, la, lw):
    return lambda out, bias, act, res: brq.diag_mxfp4_gemm_epilogue_on(route, *c.a[la], *c.w[lw], out, c.K, bias=bias, activation=act, residual=res, a_layout=la, w_layout=lw)


TILE = {r: tuple(int(d) for d in r.split("x")) for r in ("64x128", "128x128", "192x128", "192x256", "320x128", "256x128")}


@pytest.mark.parametrize("route", sorted(TILE))
def test_one_tile_kernels(brq, route):
    tm, tn = TILE[route]
    # one past the tile and its columns by 3; short by one; one row; several tiles; both kinds of stages (K up to 1024: single ones where a tile has them)
    for dm, dn, K in ((1, 3, 512), (-1, -1, 1024), (1 - tm, 9 - tn, 2048), (tm + 17, tn + 72, 1536)):
        c = Case(tm + dm, tn + dn, K, seed=tm + K)
        for i, (la, lw) in enumerate(LAYOUTS):
            for j, (bias, act, res, dt) in enumerate(FORMS):
                if (i + j) % 2:
                    continue
                for pad in (0, 8 if dt == BF16 else 5):
                    print("case", route, c.M, c.N, K, la, lw, bias, act, res, dt, pad, flush=True)
                    c.check(on_route(brq, route, c, la, lw), bias, act, res, dt, pad, in_place=res == dt and pad == 0)


@pytest.mark.parametrize("route", ["256x256", "128x256"])
def test_wide_tiles(brq, route):
    """Rows and columns that end anywhere in a tile that their alignment allows, K of one superstage and of more, more tiles than a round of the chip."""
    for M, N, K in ((1, 8, 512), (63, 264, 1024), (65, 248, 512), (129, 136, 1536), (255, 512, 2048), (321, 776, 512), (2049, 8200, 1024)):
        c = Case(M, N, K, seed=M + N)
        for i, (la, lw) in enumerate(LAYOUTS):
            for j, (bias, act, res, dt) in enumerate(FORMS):
                if M > 2000 and (i + j) % 4:
                    continue
                for pad in (0, 8):
                    print("case", route, M, N, K, la, lw, bias, act, res, dt, pad, flush=True)
                    c.check(on_route(brq, route, c, la, lw), bias, act, res, dt, pad, in_place=res == dt and pad == 0)
    c = Case(70, 132, 1024, seed=9)                      # whole 16 bytes of fp32 only
    for bias, act, res, dt in FORMS:
        if dt == F32:
            c.check(on_route(brq, route, c, "tiled", "tiled"), bias, act, res, dt, 4)


@pytest.mark.parametrize("route,shapes", [("stream", [(1, 96, 512), (16, 33, 1536), (5, 700, 2560), (3, 4, 4096)]), ("skinny", [(1, 40, 96), (16, 17, 544), (7, 300, 32)]),
                                          ("general", [(1, 1, 32), (33, 65, 96), (70, 130, 544)]), ("few", [(1, 5, 512), (16, 33, 512 * 9), (5, 100, 512 * 13), (3, 70, 544), (7, 16, 512 * 2 + 96), (2, 1, 4096)]), ("any_k", [(1, 5, 256), (64, 129, 1056), (65, 128, 288), (200, 300, 4000)])])
def test_other_kernels(brq, route, shapes):
    for M, N, K in shapes:
        c = Case(M, N, K, seed=M + N)
        for la, lw in LAYOUTS:
            if route in ("stream", "few") and K % 512 and (la, lw) != ("tiled", "tiled"):
                continue
            for bias, act, res, dt in FORMS:
                for pad in (0, 8):
                    print("case", route, M, N, K, la, lw, bias, act, res, dt, pad, flush=True)
                    c.check(on_route(brq, route, c, la, lw), bias, act, res, dt, pad, in_place=res == dt and pad == 8)


# N: a ragged tile of 16, 32 and 48 columns (which of the three is by N); K: 1 to 4 superstages a wavefront, the last one's not all there, tiled ones that end inside a superstage
@pytest.mark.parametrize("N", [1, 100, 4099, 8213])
@pytest.mark.parametrize("M,Ks", [(17, (512, 4096 + 32, 8192 + 512, 16384)), (32, (4096, 8192, 12288 + 512)), (33, (512 + 96, 4096, 8192, 12288)), (48, (4096 + 512, 8192 + 512)),
                                  (49, (512, 4096, 4096 + 512)), (64, (4096 - 32, 8192))])
def test_up_to_64_rows(brq, M, Ks, N):
    for i, K in enumerate(Ks):
        c = Case(M, N, K, seed=M + N)
        for j, (la, lw) in enumerate(LAYOUTS):
            if K % 512 and (la, lw) != ("tiled", "tiled"):
                continue
            for k, (bias, act, res, dt) in enumerate(FORMS):
                if (i + j + k) % 3:
                    continue
                pad = 8 * (k % 2)
                print("case", M, N, K, la, lw, bias, act, res, dt, pad, flush=True)
                c.check(on_route(brq, "few", c, la, lw), bias, act, res, dt, pad, in_place=res == dt and pad == 8)


def test_few_rows_refuse_longer_k(brq):
    """What the kernels for up to 64 rows do not take is refused by name, and taken by the call."""
    for M, K in ((17, 16384 + 512), (33, 12288 + 512), (49, 8192 + 512), (65, 512)):
        c = Case(M, 40, K, seed=K)
        with pytest.raises(RuntimeError, match="shape"):
            c.check(on_route(brq, "few", c, "tiled", "tiled"), True, None, None, BF16)
        c.check(lambda out, bias, act, res: brq.mxfp4_gemm_epilogue(*c.a["tiled"], *c.w["tiled"], out=out, bias=bias, a_layout="tiled", w_layout="tiled", M=M, N=40, K=K), True, None, None, BF16)


@pytest.mark.parametrize("route", ["64x128", "128x128"])
def test_split_along_k(brq, route):
    """Slices of equal and unequal length, to 16; row-major K that ends inside the last slice's last superstage."""
    for M, N, K, slices in ((1, 3, 1024 * 2, 2), (65, 130, 512 * 7, 3), (130, 72, 6144, 5), (40, 300, 512 * 13, 6), (70, 129, 128 * 27, 3), (20, 4, 128 * 17, 2), (129, 140, 7168, 7)):
        c = Case(M, N, K, seed=K)
        for la, lw in LAYOUTS:
            if K % 512 and (la, lw) not in (("tiled", "tiled"), ("rowmajor", "rowmajor")):
                continue
            for bias, act, res, dt in FORMS:
                for pad in (0, 8):
                    print("case", route, M, N, K, slices, la, lw, bias, act, res, dt, pad, flush=True)

                    def call(out, b, a, r):
                        return brq.diag_mxfp4_gemm_epilogue_on(route, *c.a[la], *c.w[lw], out, c.K, bias=b, activation=a, residual=r, a_layout=la, w_layout=lw, slices=slices)
                    c.check(call, bias, act, res, dt, pad, in_place=res == dt and pad == 8)
    long_k(brq, route, 33, 68, 1024 * 16, slices=16)


def long_k(brq, route, rows, columns, K, **kw):
    (a, va), (w, vw) = operand(1, rows, K), operand(2, columns, K)           # partial sums are no longer all exact
    a, w = ([to_dev(t) for t in to_tiled(*o)] for o in (a, w))
    out = torch.empty((rows, columns), device="cuda")
    brq.diag_mxfp4_gemm_epilogue_on(route, *a, *w, out, K, a_layout="tiled", w_layout="tiled", **kw)
    want, scale = torch.from_numpy(va @ vw.T).cuda(), torch.from_numpy(np.abs(va) @ np.abs(vw).T).cuda()
    assert bool(((out.double() - want).abs() <= 1e-5 * scale).all())


def test_long_k_of_few_rows(brq):
    for K in (512 * 61, 512 * 64, 512 * 79):             # 8 to 10 superstages a wavefront
        long_k(brq, "few", 16, 40, K)


def test_the_call(brq):
    """Through the dispatcher, both ways of the binding; what the call makes, takes and returns."""
    for M, N, K in ((1, 256, 512), (16, 200, 544), (40, 72, 96), (100, 520, 1024), (300, 136, 2048), (130, 1000, 1056), (700, 260, 512), (48, 260, 7168), (130, 260, 7168)):
        c = Case(M, N, K, seed=K)
        for la, lw in LAYOUTS:
            kw = dict(a_layout=la, w_layout=lw, M=M, N=N, K=K)
            for bias, act, res, dt in FORMS:
                for stream in (None, torch.cuda.current_stream()):
                    print("case", M, N, K, la, lw, bias, act, res, dt, stream, flush=True)

                    def call(out, b, a, r):
                        return brq.mxfp4_gemm_epilogue(*c.a[la], *c.w[lw], bias=b, activation=a, residual=r, out=out, stream=stream, **kw)
                    got = c.check(call, bias, act, res, dt, pad=8)
                    new = brq.mxfp4_gemm_epilogue(*c.a[la], *c.w[lw], bias=c.bias if bias else None, activation=act, residual=None if res is None else c.res[res], out_dtype=dt,
                                                  stream=stream, **kw)
                    assert new.dtype == dt and torch.equal(new, got)
        need = brq.mxfp4_gemm_epilogue_workspace(M, N, K, "tiled", "tiled")
        assert (need > 0) == ((M, K) == (130, 7168))
        if need:                                         # few tiles and a long K: split, in a workspace of the caller's too
            assert need % (M * N * 4) == 0
            kw = dict(a_layout="tiled", w_layout="tiled", M=M, N=N, K=K)
            got = brq.mxfp4_gemm_epilogue(*c.a["tiled"], *c.w["tiled"], bias=c.bias, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), **kw)
            assert torch.equal(got, brq.mxfp4_gemm_epilogue(*c.a["tiled"], *c.w["tiled"], bias=c.bias, **kw))
            for stream in (None, torch.cuda.current_stream()):
                with pytest.raises(brq.BrqError):
                    brq.mxfp4_gemm_epilogue(*c.a["tiled"], *c.w["tiled"], bias=c.bias, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"), stream=stream, **kw)
        nothing = brq.mxfp4_gemm_epilogue(*c.a["tiled"], *c.w["tiled"], a_layout="tiled", w_layout="tiled", M=M, N=N, K=K)
        assert torch.equal(nothing, brq.mxfp4_gemm(*c.a["tiled"], *c.w["tiled"], a_layout="tiled", w_layout="tiled", M=M, N=N, K=K))


def test_special_values(brq):
    """NaN and infinities in the bias and the residual stay in their column and element; activations at large arguments."""
    c = Case(20, 40, 96, seed=3)
    bias, res = c.bias.clone(), c.res[F32].clone()
    bias[3], bias[5] = float("nan"), float("inf")
    bias[7], bias[9], bias[11] = 1e30, -1e30, -2000.0
    res[4, 20], res[6, 21] = float("nan"), float("-inf")
    for act in (None, "relu", "silu", "gelu"):
        y = brq.mxfp4_gemm_epilogue(*c.a["rowmajor"], *c.w["rowmajor"], bias=bias, activation=act, residual=res)
        odd = torch.zeros((20, 40), dtype=torch.bool, device="cuda")
        odd[:, 3] = odd[4, 20] = True
        assert torch.equal(y.isnan(), odd), act
        fine = torch.zeros(40, dtype=torch.bool, device="cuda")
        fine[5] = True
        infinite = fine.expand(20, 40).clone()
        infinite[6, 21] = True
        assert torch.equal(y.isinf(), infinite), act
        if act:
            assert torch.equal(y[:, 9], res[:, 9]) and torch.equal(y[:, 11], res[:, 11])       # nothing is left of -1e30 and -2000
            assert bool((y[:, 7] == 1e30).all())


def test_empty(brq):
    e = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    assert brq.mxfp4_gemm_epilogue(e(0, 32), e(0, 2), e(5, 32), e(5, 2), bias=torch.zeros(5, device="cuda")).shape == (0, 5)
    assert brq.mxfp4_gemm_epilogue(e(5, 32), e(5, 2), e(0, 32), e(0, 2), activation="silu").shape == (5, 0)


def test_refused_tensors(brq):
    c = Case(4, 64, 64)
    a, w = c.a["rowmajor"], c.w["rowmajor"]
    for stream in (None, torch.cuda.current_stream()):
        with pytest.raises(ValueError, match="activation"):
            brq.mxfp4_gemm_epilogue(*a, *w, activation="tanh", stream=stream)
        with pytest.raises(ValueError):
            brq.mxfp4_gemm_epilogue(*a, *w, activation=2, stream=stream)
        with pytest.raises(ValueError):
            brq.mxfp4_gemm_epilogue(*a, *w, bias=c.bias[:32], stream=stream)
        with pytest.raises(TypeError):
            brq.mxfp4_gemm_epilogue(*a, *w, bias=c.bias.bfloat16(), stream=stream)
        with pytest.raises(ValueError):
            brq.mxfp4_gemm_epilogue(*a, *w, residual=c.res[F32][:3], stream=stream)
        with pytest.raises(TypeError):
            brq.mxfp4_gemm_epilogue(*a, *w, residual=c.res[F32].half(), stream=stream)
        with pytest.raises(brq.BrqError):
            brq.mxfp4_gemm_epilogue(*a, *w, residual=c.res[F32][:1].expand(4, 64), stream=stream)       # rows on top of one another
        with pytest.raises(ValueError):
            brq.mxfp4_gemm_epilogue(*a, *w, residual=c.res[F32].t().contiguous().t(), stream=stream)    # columns apart
        with pytest.raises(ValueError):
            brq.mxfp4_gemm_epilogue(*a, *w, out=torch.empty((3, 64), device="cuda"), stream=stream)
