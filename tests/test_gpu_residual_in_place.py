"""The norm and its gradients with an output in an input's place, every place that the header allows: the bits of the call with buffers of its own, and what
else was there left alone.  Rows of every split over wavefronts and lanes, with ragged ends (lanes behind a row's end load its last chunk again, maybe
after it was written); rows enough that a workgroup of the backward pass goes on to another row, and a last group of rows that is not all there."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def brq():
    import paper_2511_04214_amd as b
    b.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return b


def rand(g, M, K, dtype):
    return torch.randn((M, K), generator=g).to(dtype).cuda()


def placed(t, pitch):
    """A copy of t as rows of a wider buffer, and the buffer."""
    buf = torch.full((t.shape[0] + 2, t.shape[1] + pitch), 3.0, dtype=t.dtype, device="cuda")
    rows = buf[1: t.shape[0] + 1, : t.shape[1]]
    rows.copy_(t)
    return rows, buf


def untouched(buf, K):
    return bool((buf[0] == 3).all()) and bool((buf[-1] == 3).all()) and bool((buf[:, K:] == 3).all())


SIZES = [(1, 32), (5, 480), (2050, 480), (7, 992), (1030, 1024), (3, 2016), (601, 2048), (2, 4064), (600, 4096), (300, 8160), (2, 16352), (300, 12320), (270, 24608), (1, 32768)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", SIZES)
def test_gradient_over_an_input(brq, M, K, dtype):
    g = torch.Generator().manual_seed(M + K)
    t = {n: rand(g, M, K, dtype) for n in ("h", "gy", "gh")}
    w = 1 + 0.3 * torch.randn(K, generator=g).cuda()
    want, wdw = brq.add_rms_norm_backward(t["h"], t["gy"], gh=t["gh"], weight=w)
    for place in ("h", "gy", "gh"):
        for pitch in (0, 24):
            for stream in (None, torch.cuda.current_stream()):
                print("case", M, K, dtype, place, pitch, stream, flush=True)
                there, buf = placed(t[place], pitch)
                a = dict(t, **{place: there})
                dh, dw = brq.add_rms_norm_backward(a["h"], a["gy"], gh=a["gh"], weight=w, dh=there, stream=stream)
                assert dh is there and torch.equal(dh, want) and torch.equal(dw, wdw) and untouched(buf, K)
    if dtype == BF16:                                   # of another type than the output's: not its place
        gy = t["gy"].float()
        with pytest.raises(brq.BrqError):
            brq.add_rms_norm_backward(t["h"], gy, weight=w, dh=gy.view(BF16)[:, :K])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", SIZES)
def test_norm_over_an_input(brq, M, K, dtype):
    g = torch.Generator().manual_seed(M + K + 1)
    x0, r0 = rand(g, M, K, dtype), rand(g, M, K, dtype)
    w = 1 + 0.3 * torch.randn(K, generator=g).cuda()
    y0, h0 = brq.add_rms_norm(x0, residual=r0, weight=w)
    q0 = brq.add_rms_norm_rotate_quantize_fused(x0, 32, residual=r0, weight=w)
    for sum_at, out_at in (("x", None), ("r", None), (None, "x"), (None, "r"), ("x", "r"), ("r", "x")):
        for pitch in (0, 24):
            print("case", M, K, dtype, sum_at, out_at, pitch, flush=True)
            (x, bx), (r, br) = placed(x0, pitch), placed(r0, pitch)
            at = {"x": x, "r": r, None: None}
            y, h = brq.add_rms_norm(x, residual=r, weight=w, h_out=at[sum_at], out=at[out_at])
            assert torch.equal(y, y0) and torch.equal(h, h0) and untouched(bx, K) and untouched(br, K)
            if out_at is None:
                (x, bx), (r, br) = placed(x0, pitch), placed(r0, pitch)
                c, s, h = brq.add_rms_norm_rotate_quantize_fused(x, 32, residual=r, weight=w, h_out=x if sum_at == "x" else r)
                assert torch.equal(c, q0[0]) and torch.equal(s, q0[1]) and torch.equal(h, h0) and untouched(bx, K) and untouched(br, K)
    x, bx = placed(x0, 24)                              # no residual: the norm over its input
    want, _ = brq.add_rms_norm(x0, weight=w)
    y, _ = brq.add_rms_norm(x, weight=w, out=x)
    assert y is x and torch.equal(x, want) and untouched(bx, K)
