"""Python binding of the residual side of libbrq (include/brq_residual.h): the RMS norm with the residual's addition, its gradients, the
same in front of the online step, and the product with bias, activation and residual.  Argument marshalling only, as in __init__.py.

Matrices are 2-D tensors with contiguous rows of any pitch of whole 16 bytes (the product's result and residual: any pitch).  What a call
allocates (outputs, workspaces) is allocated on the stream that the work goes to.
"""
import ctypes

import torch

import paper_2511_04214_amd as _brq
from .attention import _array, _on, _same_device, _size

ACTIVATIONS = {None: 0, "relu": 1, "silu": 2, "gelu": 3}
# the kernels of mxfp4_gemm_epilogue (include/brq_diag.h), by their numbers there
EPILOGUE_ROUTES = _brq.GEMM_ROUTES + ("few",)
# the entry points that the compiled marshalling calls, in its order
NATIVE = ("brq_add_rms_norm", "brq_add_rms_norm_backward", "brq_add_rms_norm_backward_workspace", "brq_add_rms_norm_rotate_quantize_fused",
          "brq_mxfp4_gemm_epilogue", "brq_mxfp4_gemm_epilogue_workspace")


def declare(L):
    """Argument types of the entry points of brq_residual.h."""
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    for name, args in (
            ("add_rms_norm", [vp, i32, i64, vp, i32, i64, i64, i64, vp, f32, vp, i64, vp, i32, i64, vp]),
            ("add_rms_norm_backward", [vp, i32, i64, vp, i32, i64, vp, i64, i64, i64, vp, f32, vp, i64, vp, vp, i64, vp]),
            ("add_rms_norm_backward_workspace", [i64, i64, ctypes.POINTER(i64)]),
            ("add_rms_norm_rotate_quantize_fused", [vp, i32, i64, vp, i32, i64, i64, i64, vp, f32, vp, i64, i32, i64, vp, vp, vp, i32, vp]),
            ("diag_mxfp4_gemm_epilogue_on", [i32, i32, vp, vp, i32, vp, vp, i32, i64, i64, i64, vp, i32, vp, i32, i64, vp, i32, i64, vp, i64, vp]),
            ("diag_mxfp4_gemm_epilogue_route", [i32, i32, i64, i64, i64, i32, i32, i32, i32, i64, i64, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]),
            ("mxfp4_gemm_epilogue", [vp, vp, i32, vp, vp, i32, i64, i64, i64, vp, i32, vp, i32, i64, vp, i32, i64, vp, i64, vp]),
            ("mxfp4_gemm_epilogue_workspace", [i32, i32, i64, i64, i64, ctypes.POINTER(i64)])):
        f = getattr(L, "brq_" + name)
        f.argtypes, f.restype = args, i32


def _native(name, stream, *args):
    """What the compiled marshalling answers: None where it leaves the call to Python."""
    if stream is not None or _brq._native is None:
        return None
    r = getattr(_brq._native, name)(*args)
    if type(r) is int:
        _brq._check(r)
    return r


def _matrix(t, name, shape=None, dtype=None):
    """(address, dtype code, pitch) of a matrix; t None: nothing."""
    if t is None:
        return None, 0, 0
    M, K, ld = _brq._rows(t, name)
    if shape is not None and (M, K) != tuple(shape):
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return t.data_ptr(), _brq._dtype_code(t), ld


def _sum(x, residual, h_out, want_h, stream):
    """The tensor for the sum, None where there is none or it is not wanted."""
    if residual is None:
        if h_out is not None:
            raise ValueError("h_out without a residual: the sum is x itself")
        return None
    if h_out is None and want_h:
        with _on(stream):
            h_out = torch.empty(x.shape, dtype=residual.dtype, device=x.device)
    return h_out


def add_rms_norm(x, residual=None, weight=None, eps=1e-6, out_dtype=None, out=None, h_out=None, want_h=True, stream=None):
    """(y, h): h = x + residual in the residual's dtype, y = h / sqrt(mean h^2 + eps) * weight, a row at a time (brq_add_rms_norm).

    x, residual [M, K]; weight fp32 [K] (None: none).  y is of out_dtype (None: x's).  h is None without a residual, and where neither
    h_out nor want_h asks for it.  h_out and out may each be x or the residual itself, where dtypes agree (not both the same)."""
    r = _native("add_rms_norm", stream, x, residual, weight, eps, out_dtype, out, h_out, want_h)
    if r is not None:
        return r
    px, dx, ldx = _matrix(x, "x")
    M, K = x.shape
    pr, dr, ldr = _matrix(residual, "residual", (M, K))
    _same_device(x, residual, weight, out, h_out)
    pw = _array(weight, "weight", torch.float32, (K,), True)
    h = _sum(x, residual, h_out, want_h, stream)
    with _on(stream):
        y = torch.empty((M, K), dtype=out_dtype or x.dtype, device=x.device) if out is None else out
    ph, _, ldh = _matrix(h, "h_out", (M, K), None if residual is None else residual.dtype)
    py, dy, ldy = _matrix(y, "out", (M, K))
    _brq._check(_brq.lib().brq_add_rms_norm(px, dx, ldx, pr, dr, ldr, M, K, pw, eps, ph, ldh, py, dy, ldy, _brq._stream(stream)))
    return y, h


def add_rms_norm_backward_workspace(M, K):
    """Bytes of the workspace of add_rms_norm_backward (brq_add_rms_norm_backward_workspace)."""
    return _size(_brq.lib().brq_add_rms_norm_backward_workspace, M, K)


def add_rms_norm_backward(h, gy, gh=None, weight=None, eps=1e-6, dh=None, workspace=None, stream=None):
    """(dh, dw) from the sum h of add_rms_norm (x where there was no residual), the gradient gy of its y and the gradient gh that h has
    from elsewhere (None: none) (brq_add_rms_norm_backward).  dh, of h's dtype, is the gradient of x and of the residual; it may be h, gh, or gy where
    dtypes agree.  dw is fp32 [K], None without a weight."""
    r = _native("add_rms_norm_backward", stream, h, gy, gh, weight, eps, dh, workspace)
    if r is not None:
        return r
    ph, dt, ldh = _matrix(h, "h")
    M, K = h.shape
    pg, dg, ldg = _matrix(gy, "gy", (M, K))
    pgh, _, ldgh = _matrix(gh, "gh", (M, K), h.dtype)
    _same_device(h, gy, gh, weight, dh, workspace)
    pw = _array(weight, "weight", torch.float32, (K,), True)
    need = add_rms_norm_backward_workspace(M, K) if weight is not None else 0
    with _on(stream):
        dh = torch.empty((M, K), dtype=h.dtype, device=h.device) if dh is None else dh
        dw = None if weight is None else torch.empty_like(weight)
        if workspace is None and need:
            workspace = torch.empty((need,), dtype=torch.uint8, device=h.device)
    pd, _, ldd = _matrix(dh, "dh", (M, K), h.dtype)
    _brq._check(_brq.lib().brq_add_rms_norm_backward(
        ph, dt, ldh, pg, dg, ldg, pgh, ldgh, M, K, pw, eps, pd, ldd, None if dw is None else dw.data_ptr(),
        _array(workspace, "workspace", torch.uint8, (None,), True), 0 if workspace is None else workspace.numel(), _brq._stream(stream)))
    return dh, dw


def add_rms_norm_rotate_quantize_fused(x, B, residual=None, weight=None, eps=1e-6, y_dtype=torch.float32, h_out=None, want_h=True,
                                       codes=None, scales=None, stream=None, layout="rowmajor", signs=None):
    """(codes, scales, h): add_rms_norm and rotate_quantize_fused of its y in one pass, B = 1 (no rotation) or 8 ... 512
    (brq_add_rms_norm_rotate_quantize_fused).  y_dtype: torch.bfloat16 rounds y to bf16 before the rotation, torch.float32 keeps it."""
    r = _native("add_rms_norm_rotate_quantize", stream, x, B, residual, weight, eps, y_dtype, h_out, want_h, codes, scales, layout, signs)
    if r is not None:
        return r
    px, dx, ldx = _matrix(x, "x")
    M, K = x.shape
    pr, dr, ldr = _matrix(residual, "residual", (M, K))
    if y_dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("y_dtype must be torch.float32 or torch.bfloat16")
    _same_device(x, residual, weight, h_out, codes, scales, signs)
    lc = _brq._layout_code(layout)
    pw = _array(weight, "weight", torch.float32, (K,), True)
    h = _sum(x, residual, h_out, want_h, stream)
    with _on(stream):
        codes, scales = _brq._alloc_q(x, M, K, codes, scales, layout)
    ph, _, ldh = _matrix(h, "h_out", (M, K), None if residual is None else residual.dtype)
    _brq._check(_brq.lib().brq_add_rms_norm_rotate_quantize_fused(
        px, dx, ldx, pr, dr, ldr, M, K, pw, eps, ph, ldh, _brq.BRQ_BF16 if y_dtype == torch.bfloat16 else _brq.BRQ_F32, B,
        _brq._signs_ptr(signs, K), codes.data_ptr(), scales.data_ptr(), lc, _brq._stream(stream)))
    return codes, scales, h


def _activation(name):
    code = ACTIVATIONS.get(name) if name is None or isinstance(name, str) else None
    if code is None:
        raise ValueError("activation must be one of %s" % list(ACTIVATIONS))
    return code


def mxfp4_gemm_epilogue_workspace(M, N, K, a_layout="rowmajor", w_layout="rowmajor"):
    """Bytes of the workspace of mxfp4_gemm_epilogue (brq_mxfp4_gemm_epilogue_workspace)."""
    return _size(_brq.lib().brq_mxfp4_gemm_epilogue_workspace, _brq._layout_code(a_layout), _brq._layout_code(w_layout), M, N, K)


def mxfp4_gemm_epilogue(aq, as_, wq, ws, bias=None, activation=None, residual=None, out_dtype=torch.float32, out=None, stream=None,
                        a_layout="rowmajor", w_layout="rowmajor", M=None, N=None, K=None, workspace=None):
    """Y = act(deq(aq, as) @ deq(wq, ws)^T + bias) + residual, rounded once (brq_mxfp4_gemm_epilogue).

    Operands as in mxfp4_gemm.  bias: fp32 [N]; activation: None, "relu", "silu" or "gelu" (with erfc); residual: [M, N], float32 or bfloat16,
    which may be `out`."""
    r = _native("gemm_epilogue", stream, aq, as_, wq, ws, bias, activation, residual, out_dtype, out, a_layout, w_layout, M, N, K, workspace)
    if r is not None:
        return r
    la, lw, M, N, K = _brq._operands(aq, as_, wq, ws, a_layout, w_layout, M, N, K)
    act = _activation(activation)
    _same_device(aq, as_, wq, ws, bias, residual, out, workspace)
    pb = _array(bias, "bias", torch.float32, (N,), True)
    pr, dr, ldr = _matrix(residual, "residual", (M, N))
    need = 0 if bias is None and not act and residual is None else mxfp4_gemm_epilogue_workspace(M, N, K, a_layout, w_layout)
    with _on(stream):
        y, ldy = _brq._result(out, M, N, out_dtype, aq.device)
        if workspace is None and need:
            workspace = torch.empty((need,), dtype=torch.uint8, device=aq.device)
    _brq._check(_brq.lib().brq_mxfp4_gemm_epilogue(aq.data_ptr(), as_.data_ptr(), la, wq.data_ptr(), ws.data_ptr(), lw, M, N, K, pb, act,
                                                   pr, dr, ldr, y.data_ptr(), _brq._dtype_code(y), ldy,
                                                   _array(workspace, "workspace", torch.uint8, (None,), True),
                                                   0 if workspace is None else workspace.numel(), _brq._stream(stream)))
    return y


def diag_mxfp4_gemm_epilogue_route(M, N, K, a_layout="rowmajor", w_layout="rowmajor", bias=False, activation=None, residual=False, out_dtype=torch.float32,
                                   ldy=None, cus=256):
    """(kernel, slices) that mxfp4_gemm_epilogue takes on a device of `cus` compute units: one of EPILOGUE_ROUTES, split along K into so many
    (brq_diag_mxfp4_gemm_epilogue_route; needs no GPU)."""
    r, n = ctypes.c_int32(), ctypes.c_int32()
    _brq._check(_brq.lib().brq_diag_mxfp4_gemm_epilogue_route(
        _brq._layout_code(a_layout), _brq._layout_code(w_layout), M, N, K, bool(bias), _activation(activation), bool(residual),
        _brq.BRQ_BF16 if out_dtype == torch.bfloat16 else _brq.BRQ_F32, N if ldy is None else ldy, cus, ctypes.byref(r), ctypes.byref(n)))
    return EPILOGUE_ROUTES[r.value], n.value


def diag_mxfp4_gemm_epilogue_on(route, aq, as_, wq, ws, out, K, bias=None, activation=None, residual=None, a_layout="rowmajor",
                                w_layout="rowmajor", slices=1, stream=None):
    """out[M, N] = mxfp4_gemm_epilogue on the kernel `route`, one of EPILOGUE_ROUTES, in so many slices of K (brq_diag_mxfp4_gemm_epilogue_on)."""
    M, N, ldy = _brq._rows(out, "out")
    la, lw, _, _, _ = _brq._operands(aq, as_, wq, ws, a_layout, w_layout, M, N, K)
    pb = _array(bias, "bias", torch.float32, (N,), True)
    pr, dr, ldr = _matrix(residual, "residual", (M, N))
    with _on(stream):
        space = torch.empty((slices * M * ((N + 3) // 4 * 16) if slices > 1 else 0,), dtype=torch.uint8, device=out.device)
    _brq._check(_brq.lib().brq_diag_mxfp4_gemm_epilogue_on(
        EPILOGUE_ROUTES.index(route), slices, aq.data_ptr(), as_.data_ptr(), la, wq.data_ptr(), ws.data_ptr(), lw, M, N, K, pb, _activation(activation),
        pr, dr, ldr, out.data_ptr(), _brq._dtype_code(out), ldy, space.data_ptr(), space.numel(), _brq._stream(stream)))
    return out
