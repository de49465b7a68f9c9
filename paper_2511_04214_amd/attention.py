"""Python binding of the attention side of libbrq (include/brq_attn.h): head norms with position rotation, the MXFP4
cache, attention over it, its pages.  Argument marshalling only, as in __init__.py.

Heads are 3-D tensors [T, H, D] with contiguous channels and any strides of whole 16 bytes (views of a packed
projection).  A cache is a uint8 tensor [num_pages, kv4_page_bytes(Hk, D)]; a page holds KV4_PAGE tokens.  What a
call allocates (outputs, workspaces) is allocated on the stream that the work goes to.
"""
import contextlib
import ctypes

import torch

import paper_2511_04214_amd as _brq

KV4_PAGE = 64
# the entry points that the compiled marshalling calls, in its order
NATIVE = ("brq_qk_norm_rope", "brq_qk_norm_rope_backward", "brq_qk_norm_rope_backward_workspace", "brq_kv4_append", "brq_kv4_read", "brq_kv4_attention",
          "brq_kv4_attention_workspace", "brq_kv4_pages_workspace", "brq_kv4_pages_copy", "brq_kv4_pages_fork", "brq_kv4_pages_free", "brq_kv4_pages_reserve",
          "brq_kv4_pages_compact")


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("heads", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Rope(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("rot", ctypes.c_int64), ("interleaved", ctypes.c_int32)]


def declare(L):
    """Argument types of the entry points of brq_attn.h."""
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    h, r, n = ctypes.POINTER(_Heads), ctypes.POINTER(_Rope), ctypes.POINTER(i64)
    for name, args in (
            ("qk_norm_rope", [h, h, i32, i64, i64, vp, vp, f32, r, i64, h, h, i32, vp]),
            ("qk_norm_rope_backward", [h, h, i32, i64, i64, vp, vp, f32, r, i64, h, h, i32, h, h, vp, vp, vp, i64, vp]),
            ("qk_norm_rope_backward_workspace", [i64, i64, i64, i64, n]),
            ("kv4_page_bytes", [i64, i64, n]),
            ("kv4_append", [h, h, h, i32, i64, i64, vp, vp, f32, r, i64, i64, vp, vp, i64, h, vp]),
            ("kv4_read", [vp, i64, i64, i64, vp, h, h, i32, vp]),
            ("kv4_attention", [h, i64, i64, vp, i64, i64, vp, i64, vp, vp, i64, f32, i32, i64, i64, i64, h, vp, vp, i64, vp]),
            ("diag_kv4_attention_route", [i64, i64, i64, i64, i64, i64, i64, i32, i64, i64, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]),
            ("kv4_attention_workspace", [i64, i64, i64, i64, i64, i64, i64, n]),
            ("kv4_pages_workspace", [i64, i64, n]),
            ("kv4_pages_copy", [vp, i64, i64, vp, vp, i64, vp]),
            ("kv4_pages_fork", [vp, i64, i64, vp, i64, i64, vp, vp, vp, vp, i64, vp, vp, vp]),
            ("kv4_pages_free", [vp, i64, i64, vp, vp, i64, vp, i64, vp]),
            ("kv4_pages_reserve", [vp, i64, i64, vp, i64, vp, vp, i64, vp, vp, vp]),
            ("kv4_pages_compact", [vp, i64, i64, vp, i64, i64, vp, vp, vp, vp])):
        f = getattr(L, "brq_" + name)
        f.argtypes, f.restype = args, i32


def _heads(t, name, shape=None):
    """[T, H, D] tensor -> _Heads; `shape`: what it has to have, None where any will do."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor (libbrq has no CPU path)" % name)
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError("%s must be [tokens, heads, channels] with contiguous channels" % name)
    if shape is not None and any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    return _Heads(t.data_ptr(), t.shape[1], t.stride(0), t.stride(1))


def _same_device(like, *tensors):
    if like.is_cuda and like.device.index != torch.cuda.current_device():
        raise ValueError("tensors on %s, which is not the current device" % like.device)
    for t in tensors:
        if t is not None and t.device != like.device:
            raise ValueError("tensors on several devices: %s and %s" % (like.device, t.device))


def _array(t, name, dtype, shape, optional=False):
    """The address of a contiguous GPU tensor of `dtype` and `shape` (None: any length)."""
    if t is None:
        if optional:
            return None
        raise ValueError("%s must be given" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor (libbrq has no CPU path)" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous() or t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError("%s must be contiguous and %s, got %s" % (name, list(shape), list(t.shape)))
    return t.data_ptr()


def _rope(cos, sin, positions, interleaved, T):
    if cos is None and sin is None and positions is None:
        return None
    c = _array(cos, "cos", torch.float32, (None, None))
    return _Rope(c, _array(sin, "sin", torch.float32, tuple(cos.shape)), _array(positions, "positions", torch.int64, (T,)), cos.shape[0],
                 cos.shape[1] * 2, int(bool(interleaved)))


def _on(stream):
    """What is allocated in here belongs to `stream`."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _native(name, stream, *args):
    """What the compiled marshalling answers: None where it leaves the call to Python."""
    if stream is not None or _brq._native is None:
        return None
    r = getattr(_brq._native, name)(*args)
    if type(r) is int:
        _brq._check(r)
    return r


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _size(call, *args):
    n = ctypes.c_int64()
    _brq._check(call(*args, ctypes.byref(n)))
    return n.value


def qk_norm_rope(q, k=None, wq=None, wk=None, eps=1e-6, cos=None, sin=None, positions=None, interleaved=False, B=1, out_dtype=None,
                 q_out=None, k_out=None, stream=None):
    """(q', k') of queries [T, Hq, D] and keys [T, Hk, D]: RMS norm of every head with weights wq, wk (fp32 [D]; None: no norm),
    rotation by position (cos, sin fp32 [rows, rot / 2], positions int64 [T]; None: none), block rotation (B = 1: none)
    (brq_qk_norm_rope).  Without `k` the second result is None."""
    r = _native("qk_norm_rope", stream, q, k, wq, wk, eps, cos, sin, positions, interleaved, B, out_dtype, q_out, k_out)
    if r is not None:
        return r
    hq, hk = _heads(q, "q"), _heads(k, "k", None if k is None else (q.shape[0], None, q.shape[2]))
    T, _, D = q.shape
    if k is not None and k.dtype != q.dtype:
        raise ValueError("q and k must agree in dtype")
    _same_device(q, k, wq, wk, cos, sin, positions, q_out, k_out)
    rope = _rope(cos, sin, positions, interleaved, T)
    with _on(stream):
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
        if k is not None and k_out is None:
            k_out = torch.empty(k.shape, dtype=q_out.dtype, device=q.device)
    if k is None:
        k_out = None
    elif k_out.dtype != q_out.dtype:
        raise ValueError("q_out and k_out must agree in dtype")
    ho, hko = _heads(q_out, "q_out", q.shape), _heads(k_out, "k_out", None if k is None else k.shape)
    _brq._check(_brq.lib().brq_qk_norm_rope(_ref(hq), _ref(hk), _brq._dtype_code(q), T, D, _array(wq, "wq", torch.float32, (D,), True),
                                            _array(wk, "wk", torch.float32, (D,), True), eps, _ref(rope), B, _ref(ho), _ref(hko),
                                            _brq._dtype_code(q_out), _brq._stream(stream)))
    return q_out, k_out


def qk_norm_rope_backward_workspace(T, Hq, Hk, D):
    """Bytes of the workspace of qk_norm_rope_backward (brq_qk_norm_rope_backward_workspace)."""
    return _size(_brq.lib().brq_qk_norm_rope_backward_workspace, T, Hq, Hk, D)


def qk_norm_rope_backward(q, k, gq, gk, wq=None, wk=None, eps=1e-6, cos=None, sin=None, positions=None, interleaved=False, B=1, dq=None,
                          dk=None, workspace=None, stream=None):
    """(dq, dk, dwq, dwk) from the inputs of qk_norm_rope and the gradients gq, gk of its results (brq_qk_norm_rope_backward).
    dwq, dwk are fp32 [D], None where the weight is."""
    r = _native("qk_norm_rope_backward", stream, q, k, gq, gk, wq, wk, eps, cos, sin, positions, interleaved, B, dq, dk, workspace)
    if r is not None:
        return r
    T, Hq, D = q.shape if q.dim() == 3 else (0, 0, 0)
    hq, hk = _heads(q, "q"), _heads(k, "k", None if k is None else (T, None, D))
    if (k is None) != (gk is None):
        raise ValueError("k and gk go together")
    hgq, hgk = _heads(gq, "gq", q.shape), _heads(gk, "gk", None if k is None else k.shape)
    if (k is not None and k.dtype != q.dtype) or (gk is not None and gk.dtype != gq.dtype):
        raise ValueError("q and k, and gq and gk, must agree in dtype")
    _same_device(q, k, gq, gk, wq, wk, cos, sin, positions, dq, dk, workspace)
    rope = _rope(cos, sin, positions, interleaved, T)
    pwq, pwk = _array(wq, "wq", torch.float32, (D,), True), _array(wk, "wk", torch.float32, (D,), True)
    sums = wq is not None or (wk is not None and k is not None)
    need = qk_norm_rope_backward_workspace(T, Hq, 0 if k is None else k.shape[1], D) if sums else 0
    with _on(stream):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=k.dtype, device=q.device) if dk is None and k is not None else dk
        dwq = None if wq is None else torch.empty_like(wq)
        dwk = None if wk is None or k is None else torch.empty_like(wk)
        if workspace is None and need:
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
    if dq.dtype != q.dtype or (dk is not None and dk.dtype != q.dtype):
        raise ValueError("dq and dk must have the dtype of q and k")
    hdq, hdk = _heads(dq, "dq", q.shape), _heads(dk if k is not None else None, "dk", None if k is None else k.shape)
    _brq._check(_brq.lib().brq_qk_norm_rope_backward(
        _ref(hq), _ref(hk), _brq._dtype_code(q), T, D, pwq, pwk, eps, _ref(rope), B, _ref(hgq), _ref(hgk), _brq._dtype_code(gq), _ref(hdq),
        _ref(hdk), None if dwq is None else dwq.data_ptr(), None if dwk is None else dwk.data_ptr(),
        _array(workspace, "workspace", torch.uint8, (None,), True), 0 if workspace is None else workspace.numel(), _brq._stream(stream)))
    return dq, dk if k is not None else None, dwq, dwk


def kv4_page_bytes(Hk, D):
    """Bytes of a cache page of KV4_PAGE tokens with Hk heads of D channels (brq_kv4_page_bytes)."""
    return _size(_brq.lib().brq_kv4_page_bytes, Hk, D)


def _pool(pool, Hk=None, D=None):
    """(address, pages, heads) of a cache; Hk: the heads it has to have."""
    p = _array(pool, "pool", torch.uint8, (None, None))
    if D is None:
        return p, pool.shape[0], None
    if Hk is None:
        Hk = pool.shape[1] // (68 * D) if D else 0
    if pool.shape[1] != Hk * 68 * D or Hk < 1:
        raise ValueError("pool must be [pages, kv4_page_bytes(%s, %s)], got %s" % (Hk, D, list(pool.shape)))
    return p, pool.shape[0], Hk


def kv4_append(pool, slots, k, v, q=None, wq=None, wk=None, eps=1e-6, cos=None, sin=None, positions=None, interleaved=False, B=1, Bv=1,
               q_out=None, stream=None):
    """Writes keys and values [T, Hk, D] to slots (int64 [T], page * KV4_PAGE + place) of the cache: keys as qk_norm_rope makes
    them, values rotated by Bv, both as MXFP4 (brq_kv4_append).  With q the queries come along: returns q', else None."""
    r = _native("kv4_append", stream, pool, slots, k, v, q, wq, wk, eps, cos, sin, positions, interleaved, B, Bv, q_out)
    if r is not None:
        return None if r is True else r
    hk = _heads(k, "k")
    T, Hk, D = k.shape
    hv, hq = _heads(v, "v", k.shape), _heads(q, "q", (T, None, D))
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise ValueError("q, k and v must agree in dtype")
    _same_device(k, pool, slots, v, q, wq, wk, cos, sin, positions, q_out)
    p, pages, _ = _pool(pool, Hk, D)
    rope = _rope(cos, sin, positions, interleaved, T)
    sl = _array(slots, "slots", torch.int64, (T,))
    if q is not None and q_out is None:
        with _on(stream):
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if q_out is not None and (q is None or q_out.dtype != q.dtype):
        raise ValueError("q_out must have the dtype of q")
    ho = _heads(q_out, "q_out", None if q is None else q.shape)
    _brq._check(_brq.lib().brq_kv4_append(_ref(hq), _ref(hk), _ref(hv), _brq._dtype_code(k), T, D, _array(wq, "wq", torch.float32, (D,), True),
                                          _array(wk, "wk", torch.float32, (D,), True), eps, _ref(rope), B, Bv, sl, p, pages, _ref(ho),
                                          _brq._stream(stream)))
    return q_out


def kv4_read(pool, slots, D, out_dtype=torch.bfloat16, k_out=None, v_out=None, stream=None):
    """(k, v), each [T, Hk, D]: the values that stand at slots (int64 [T]) of the cache (brq_kv4_read)."""
    r = _native("kv4_read", stream, pool, slots, D, out_dtype, k_out, v_out)
    if r is not None:
        return r
    p, pages, Hk = _pool(pool, None, D)
    sl = _array(slots, "slots", torch.int64, (None,))
    shape = (slots.shape[0], Hk, D)
    _same_device(pool, slots, k_out, v_out)
    with _on(stream):
        k_out = torch.empty(shape, dtype=out_dtype, device=pool.device) if k_out is None else k_out
        v_out = torch.empty(shape, dtype=k_out.dtype, device=pool.device) if v_out is None else v_out
    if v_out.dtype != k_out.dtype:
        raise ValueError("k_out and v_out must agree in dtype")
    hk, hv = _heads(k_out, "k_out", shape), _heads(v_out, "v_out", shape)
    _brq._check(_brq.lib().brq_kv4_read(p, pages, shape[0], D, sl, _ref(hk), _ref(hv), _brq._dtype_code(k_out), _brq._stream(stream)))
    return k_out, v_out


def kv4_attention_workspace(T, S, Hq, Hk, D, max_q, max_kv):
    """Bytes of the workspace of kv4_attention (brq_kv4_attention_workspace)."""
    return _size(_brq.lib().brq_kv4_attention_workspace, T, S, Hq, Hk, D, max_q, max_kv)


def kv4_attention(q, pool, table, kv_lens, scale=None, causal=True, window=0, cu_q=None, max_q=None, max_kv=None, out=None, lse=None,
                  want_lse=False, workspace=None, stream=None):
    """Attention of query rows q [T, Hq, D] (bfloat16) over the cache (brq_kv4_attention).

    table int32 [S, columns], kv_lens int32 [S]; cu_q int32 [S + 1] says which rows are whose (None: one row a sequence,
    T = S).  max_q: the longest sequence's rows (None: 1 without cu_q, else T); max_kv: the longest context (None: what the
    table has room for).  scale: None for D ** -0.5.  Returns out, or (out, lse) where lse is given or wanted."""
    r = _native("kv4_attention", stream, q, pool, table, kv_lens, scale, causal, window, cu_q, max_q, max_kv, out, lse, want_lse, workspace)
    if r is not None:
        return r
    hq = _heads(q, "q")
    T, Hq, D = q.shape
    if q.dtype != torch.bfloat16 or (out is not None and out.dtype != torch.bfloat16):
        raise TypeError("q and out must be torch.bfloat16")
    _same_device(q, pool, table, kv_lens, cu_q, out, lse, workspace)
    p, pages, Hk = _pool(pool, None, D)
    pt = _array(table, "table", torch.int32, (None, None))
    S, cols = table.shape
    pl, pc = _array(kv_lens, "kv_lens", torch.int32, (S,)), _array(cu_q, "cu_q", torch.int32, (S + 1,), True)
    if cu_q is None and T != S:
        raise ValueError("cu_q must be given where the number of rows is not that of the sequences")
    max_q = (1 if cu_q is None else max(1, T)) if max_q is None else max_q
    max_kv = cols * KV4_PAGE if max_kv is None else max_kv
    need = kv4_attention_workspace(T, S, Hq, Hk, D, max_q, max_kv)
    scale = D ** -0.5 if scale is None else scale
    with _on(stream):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        if lse is None and want_lse:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device)
        if workspace is None and need:
            workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
    ho = _heads(out, "out", q.shape)
    _brq._check(_brq.lib().brq_kv4_attention(
        _ref(hq), T, D, p, pages, Hk, pt, cols, pl, pc, S, scale, int(bool(causal)), window, max_q, max_kv,
        _ref(ho), _array(lse, "lse", torch.float32, (T, Hq), True), _array(workspace, "workspace", torch.uint8, (None,), True),
        0 if workspace is None else workspace.numel(), _brq._stream(stream)))
    return out if lse is None else (out, lse)


# the kernels of kv4_attention (include/brq_diag.h), by their numbers there
KV4_ROUTES = ("few_16", "few_32", "one", "pair", "tall")


def diag_kv4_attention_route(T, S, Hq, Hk, D, max_q, max_kv, causal=True, window=0, cus=256):
    """(kernel, parts): the kernel that kv4_attention takes for a call of these sizes on a device of `cus` compute units, one of
    KV4_ROUTES, and into how many parts it cuts a context (brq_diag_kv4_attention_route; needs no GPU)."""
    r, n = ctypes.c_int32(), ctypes.c_int32()
    _brq._check(_brq.lib().brq_diag_kv4_attention_route(T, S, Hq, Hk, D, max_q, max_kv, int(bool(causal)), window, cus, ctypes.byref(r), ctypes.byref(n)))
    return KV4_ROUTES[r.value], n.value


def kv4_pages_workspace(n, num_pages):
    """Bytes of the workspace of kv4_pages_fork, _reserve (n: their lists' length) and _compact (n = 0) (brq_kv4_pages_workspace)."""
    return _size(_brq.lib().brq_kv4_pages_workspace, n, num_pages)


def _state(table, lens, refs, num_pages):
    pt = _array(table, "table", torch.int32, (None, None))
    pl = None if lens is None else _array(lens, "lens", torch.int32, (table.shape[0],))
    return pt, table.shape[0], table.shape[1], pl, _array(refs, "refs", torch.int32, (num_pages,))


def _lists(a, b, what):
    pa = _array(a, what[0], torch.int32, (None,))
    return pa, None if b is None else _array(b, what[1], torch.int32, (a.shape[0],)), a.shape[0]


def _space(n, num_pages, workspace, like, stream):
    """(result int32 [1], workspace)"""
    need = kv4_pages_workspace(n, num_pages)
    with _on(stream):
        result = torch.empty((1,), dtype=torch.int32, device=like.device)
        workspace = torch.empty((need,), dtype=torch.uint8, device=like.device) if workspace is None else workspace
    p = _array(workspace, "workspace", torch.uint8, (None,))
    if workspace.numel() < need:
        raise ValueError("workspace must have at least %d bytes" % need)
    return result, p, workspace


def kv4_pages_copy(pool, src, dst, stream=None):
    """Page dst[i] = page src[i] of the cache; src, dst int32 (brq_kv4_pages_copy)."""
    if _native("kv4_pages_copy", stream, pool, src, dst) is not None:
        return
    p, pages, _ = _pool(pool)
    ps, pd, n = _lists(src, dst, ("src", "dst"))
    _same_device(pool, src, dst)
    _brq._check(_brq.lib().brq_kv4_pages_copy(p, pool.shape[1], pages, ps, pd, n, _brq._stream(stream)))


def kv4_pages_fork(pool, table, lens, refs, parents, children, workspace=None, stream=None):
    """Sequences children[i] become copies of parents[i] (int32 lists): full pages shared, a last one that is not full copied
    (brq_kv4_pages_fork).  Returns failed, int32 [1]: pairs for which no free page was left."""
    r = _native("kv4_pages_fork", stream, pool, table, lens, refs, parents, children, workspace)
    if r is not None:
        return r
    p, pages, _ = _pool(pool)
    pt, S, cols, pl, pr = _state(table, lens, refs, pages)
    pp, pc, n = _lists(parents, children, ("parents", "children"))
    _same_device(pool, table, lens, refs, parents, children, workspace)
    failed, pw, workspace = _space(n, pages, workspace, pool, stream)
    _brq._check(_brq.lib().brq_kv4_pages_fork(p, pool.shape[1], pages, pt, S, cols, pl, pr, pp, pc, n, failed.data_ptr(), pw, _brq._stream(stream)))
    return failed


def kv4_pages_free(table, lens, refs, seqs, stream=None):
    """The pages of sequences seqs (int32) are given up (brq_kv4_pages_free)."""
    if _native("kv4_pages_free", stream, table, lens, refs, seqs) is not None:
        return
    pt, S, cols, pl, pr = _state(table, lens, refs, None)
    ps, _, n = _lists(seqs, None, ("seqs",))
    _same_device(table, lens, refs, seqs)
    _brq._check(_brq.lib().brq_kv4_pages_free(pt, S, cols, pl, pr, refs.shape[0], ps, n, _brq._stream(stream)))


def kv4_pages_reserve(table, refs, seqs, tokens, workspace=None, stream=None):
    """Sequences seqs[i] get pages for tokens[i] tokens (int32 lists) (brq_kv4_pages_reserve).  Returns failed, int32 [1]:
    sequences that got none for want of pages or columns."""
    r = _native("kv4_pages_reserve", stream, table, refs, seqs, tokens, workspace)
    if r is not None:
        return r
    pt, S, cols, _, pr = _state(table, None, refs, None)
    ps, pk, n = _lists(seqs, tokens, ("seqs", "tokens"))
    _same_device(table, refs, seqs, tokens, workspace)
    failed, pw, workspace = _space(n, refs.shape[0], workspace, table, stream)
    _brq._check(_brq.lib().brq_kv4_pages_reserve(pt, S, cols, pr, refs.shape[0], ps, pk, n, failed.data_ptr(), pw, _brq._stream(stream)))
    return failed


def kv4_pages_compact(pool, table, refs, workspace=None, stream=None):
    """The live pages move to the lowest numbers, table and refs follow (brq_kv4_pages_compact).  Returns live, int32 [1]."""
    r = _native("kv4_pages_compact", stream, pool, table, refs, workspace)
    if r is not None:
        return r
    p, pages, _ = _pool(pool)
    pt, S, cols, _, pr = _state(table, None, refs, pages)
    _same_device(pool, table, refs, workspace)
    live, pw, workspace = _space(0, pages, workspace, pool, stream)
    _brq._check(_brq.lib().brq_kv4_pages_compact(p, pool.shape[1], pages, pt, S, cols, pr, live.data_ptr(), pw, _brq._stream(stream)))
    return live
