"""What the residual side refuses, on the host and before anything is launched (no GPU)."""
import ctypes
from ctypes import byref

import pytest
import torch

import paper_2511_04214_amd as brq

OK, NULL, SHAPE, BLOCK, ALIGN, DTYPE, LAYOUT, ACTIVATION = 0, 1, 2, 3, 4, 5, 7, 9
P = 0x1000          # never dereferenced: P, Q, R, S are buffers of their own
Q, R, S = 2 * P, 3 * P, 4 * P


@pytest.fixture(scope="module")
def L():
    return brq.lib()


def norm_refusals(f):
    """What both forms of the norm share."""
    assert f(M=0) == OK and f(M=0, x=None, res=None, h=None) == OK
    assert f(x=None) == f(h=P + 0x100, res=None) == NULL
    assert f(xdt=2) == f(rdt=-1) == DTYPE
    assert f(M=-1) == f(M=1 << 31) == f(K=0) == f(K=-32) == f(K=48) == f(K=32768 + 32) == f(M=1 << 29, K=64) == SHAPE
    assert f(ldx=32) == f(ldr=32) == f(ldh=32) == f(ldx=1 << 30) == f(ldr=1 << 62) == f(ldh=(1 << 63) - 1) == SHAPE
    assert f(eps=-1e-6) == f(eps=float("nan")) == f(eps=-float("inf")) == SHAPE
    assert f(x=P + 8) == f(res=Q + 2) == f(h=R + 4) == f(w=P + 4) == f(ldx=68) == f(ldr=66) == f(ldh=70) == ALIGN
    # a sum in a summand's place: the same rows, or none of it
    assert f(h=Q, ldh=72) == f(h=P, ldh=72) == f(h=P, xdt=0) == SHAPE
    assert f(M=0, h=Q, ldh=72) == OK


def test_add_rms_norm(L):
    def f(x=P, xdt=1, ldx=64, res=Q, rdt=1, ldr=64, M=3, K=64, w=P, eps=1e-6, h=R, ldh=64, y=S, ydt=1, ldy=64):
        return L.brq_add_rms_norm(x, xdt, ldx, res, rdt, ldr, M, K, w, eps, h, ldh, y, ydt, ldy, None)
    norm_refusals(f)
    assert f(y=None) == NULL and f(ydt=5) == DTYPE and f(ldy=32) == SHAPE and f(y=S + 2) == f(ldy=65) == ALIGN
    assert f(y=R) == f(y=P, ldy=72) == f(y=Q, ydt=0) == SHAPE          # the sum and its norm in one place; another pitch; another type


def test_fused(L):
    def f(x=P, xdt=1, ldx=64, res=Q, rdt=1, ldr=64, M=3, K=64, w=P, eps=1e-6, h=R, ldh=64, ydt=0, B=32, signs=None, codes=S, scales=S, layout=0):
        return L.brq_add_rms_norm_rotate_quantize_fused(x, xdt, ldx, res, rdt, ldr, M, K, w, eps, h, ldh, ydt, B, signs, codes, scales, layout, None)
    norm_refusals(f)
    for B in (0, 2, 4, 24, 128, 1024, -8, 1 << 40):
        assert f(B=B) == BLOCK, B
    assert f(B=1024, K=1024, ldx=1024, ldr=1024, ldh=1024) == BLOCK and f(B=1, signs=P) == BLOCK
    assert f(codes=None) == f(scales=None) == NULL and f(ydt=2) == DTYPE and f(layout=2) == f(layout=-1) == LAYOUT
    assert f(codes=S + 4) == f(scales=S + 8) == f(signs=P + 1) == ALIGN
    assert f(M=0, codes=None, scales=None) == OK


def test_backward(L):
    def f(h=P, hdt=1, ldh=64, gy=Q, gdt=1, ldgy=64, gh=R, ldgh=64, M=3, K=64, w=P, eps=1e-6, dh=S, lddh=64, dw=P, ws=P, n=1 << 20):
        return L.brq_add_rms_norm_backward(h, hdt, ldh, gy, gdt, ldgy, gh, ldgh, M, K, w, eps, dh, lddh, dw, ws, n, None)
    assert f(h=None) == f(gy=None) == f(dh=None) == f(ws=None) == f(w=None) == NULL           # (w: a gradient of a weight that is not there)
    assert f(hdt=3) == f(gdt=9) == DTYPE
    assert f(M=-1) == f(K=40) == f(K=1 << 16) == f(ldh=32) == f(ldgy=32) == f(ldgh=32) == f(lddh=32) == f(eps=float("nan")) == f(n=16) == f(n=-1) == SHAPE
    assert f(dh=R, lddh=72) == f(dh=P, lddh=72) == f(dh=Q, gdt=0) == f(dh=Q, lddh=72) == SHAPE
    assert f(h=P + 2) == f(gy=Q + 4) == f(gh=R + 8) == f(dh=S + 2) == f(w=P + 4) == f(dw=P + 2) == f(ws=P + 8) == f(ldgh=68) == ALIGN
    assert f(M=0, w=None, dw=None, ws=None, n=0, h=None, gy=None, gh=None, dh=None) == OK
    n = ctypes.c_int64()
    assert L.brq_add_rms_norm_backward_workspace(3, 64, None) == NULL
    assert L.brq_add_rms_norm_backward_workspace(-1, 64, byref(n)) == L.brq_add_rms_norm_backward_workspace(1, 65, byref(n)) == SHAPE
    assert brq.add_rms_norm_backward_workspace(0, 64) == 0 < brq.add_rms_norm_backward_workspace(1, 64)


def test_gemm_epilogue(L):
    def f(aq=P, as_=P, la=0, wq=P, ws=P, lw=0, M=4, N=6, K=64, bias=P, act=2, res=Q, rdt=1, ldr=6, y=R, ydt=1, ldy=6, space=S, n=1 << 30, call=None):
        return (call or L.brq_mxfp4_gemm_epilogue)(aq, as_, la, wq, ws, lw, M, N, K, bias, act, res, rdt, ldr, y, ydt, ldy, space, n, None)
    assert f(M=0) == f(N=0, ldr=0, ldy=0) == OK and f(M=0, aq=None, y=None, res=None) == OK

    def on(route, slices=1):
        return lambda *a: L.brq_diag_mxfp4_gemm_epilogue_on(route, slices, *a)
    for call in (None, on(0)):
        assert f(aq=None, call=call) == f(ws=None, call=call) == f(y=None, call=call) == NULL
        assert f(ydt=2, call=call) == f(rdt=2, call=call) == DTYPE and f(la=3, call=call) == LAYOUT
        for act in (-1, 4, 1 << 30):
            assert f(act=act, call=call) == ACTIVATION
        assert f(M=-1, call=call) == f(K=40, call=call) == f(ldy=5, call=call) == f(ldr=5, call=call) == f(ldr=1 << 30, call=call) == SHAPE
        assert f(y=Q, ldy=8, call=call) == f(y=Q, ydt=0, call=call) == SHAPE                  # a sum in the residual's place: the same rows
        assert f(bias=P + 2, call=call) == f(res=Q + 1, call=call) == f(res=Q + 2, rdt=0, call=call) == f(y=R + 8, call=call) == f(space=S + 8, call=call) == ALIGN
    assert f(M=0, call=on(0)) == SHAPE
    for route in (3, 4, 12, -1, 1, 2, 5, 11):            # persistent kernels; no kernels; kernels that do not take 20 rows of K = 64
        assert f(M=20, call=on(route)) == SHAPE
    big = dict(M=70, N=130, K=4096, la=1, lw=1, ldr=130, ldy=130)
    assert f(**big, space=None, call=on(5, 2)) == NULL and f(**big, n=2 * 70 * 132 * 4 - 1, call=on(6, 2)) == SHAPE
    for route, slices in ((5, 0), (5, -1), (5, 5), (6, 17), (7, 2), (0, 2), (2, 2)):     # no slices; slices below 1024; too many; kernels that are not split
        assert f(**big, call=on(route, slices)) == SHAPE
    n = ctypes.c_int64()
    space = L.brq_mxfp4_gemm_epilogue_workspace
    assert space(0, 0, 4, 6, 64, None) == NULL and space(2, 0, 4, 6, 64, byref(n)) == LAYOUT
    assert space(0, 0, -1, 6, 64, byref(n)) == space(0, 0, 4, 1 << 40, 64, byref(n)) == space(0, 0, 4, 6, 65, byref(n)) == SHAPE
    assert space(0, 0, 0, 6, 64, byref(n)) == OK and n.value == 0
    assert "activation" in brq.lib().brq_strerror(ACTIVATION).decode()


def test_python_refuses_before_the_library():
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    with pytest.raises(ValueError, match="GPU tensor"):
        brq.add_rms_norm(t(3, 64))
    with pytest.raises(ValueError, match="GPU tensor"):
        brq.add_rms_norm_backward(t(3, 64), t(3, 64))
    with pytest.raises(ValueError, match="GPU tensor"):
        brq.add_rms_norm_rotate_quantize_fused(t(3, 64), 32)
    with pytest.raises(ValueError, match="GPU tensor"):
        brq.mxfp4_gemm_epilogue(*(t(3, 32, dtype=torch.uint8) for _ in range(4)))
    with pytest.raises(TypeError):
        brq.add_rms_norm(t(3, 64), None, None, 1e-6, None, None, None, True, None, 0)
