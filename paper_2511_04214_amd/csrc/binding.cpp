// The calls that a layer and an analysis make, without the interpreter's share of them: arguments are read from the tensors here, checked
// as __init__.py checks them, and handed to the C ABI.  With Python and ctypes in between a call cost the host 6 to 9 us, of
// which the launch is 3: a small layer (16 x 256 x 256, two calls and a result tensor) took 15.0 us, the GPU 6.7.
//
// Only what is plainly right is done here: tensors of torch's own type on the GPU with no other dispatch key than that,
// plain integers, the current stream.  Anything else (a subclass, a traced or batched tensor, an argument that does not
// fit, buffers that are to be made) returns None, and the caller goes its way through Python, which accepts or refuses it
// as it always did.  Otherwise a call returns the library's status, 0 or not, or the result tensor.
#include <Python.h>

#include <algorithm>
#include <cmath>

#include <ATen/core/Tensor.h>
#include <ATen/ops/_foreach_zero.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/brq.h"
#include "../../include/brq_attn.h"
#include "../../include/brq_residual.h"

namespace {

// The interpreter's lock is not held while one of these lives (an exception gives it back too).
struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// The library's entry points, set by bind() when it is loaded.
decltype(&brq_rotate_quantize_fused) f_rotate_quantize;
decltype(&brq_swiglu_rotate_quantize_fused) f_swiglu;
decltype(&brq_matrix_rotate_quantize_fused) f_matrix;
decltype(&brq_mxfp4_gemm) f_gemm;
decltype(&brq_rotate_quantize_gemm_fused) f_decode;
decltype(&brq_block_stats) f_stats;
decltype(&brq_block_stats_summary) f_summary;

// A tensor of torch's own type, on the GPU, that nothing watches or stands in for: beside the dispatch keys that every such
// tensor has (autograd's, autocast's) it has the device's alone.
bool on_gpu(const at::Tensor& t) {
    return t.defined() && t.key_set() - c10::autograd_dispatch_keyset_with_ADInplaceOrView - c10::autocast_dispatch_keyset ==
                              c10::DispatchKeySet(c10::DispatchKey::CUDA);
}
const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return on_gpu(t) ? &t : nullptr;
}

const at::Tensor* bytes(PyObject* o) {
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == at::kByte && t->is_contiguous() ? t : nullptr;
}

bool dtype_of(at::ScalarType s, brq_dtype* d) {
    *d = s == at::kFloat ? BRQ_F32 : BRQ_BF16;
    return s == at::kFloat || s == at::kBFloat16;
}

bool dtype_arg(PyObject* o, at::ScalarType* s, brq_dtype* d) {
    if (!THPDtype_Check(o)) return false;
    *s = reinterpret_cast<THPDtype*>(o)->scalar_type;
    return dtype_of(*s, d);
}

// A matrix with contiguous rows.
struct Rows {
    const at::Tensor* t;
    int64_t M, K, ld;
    brq_dtype dt;
};
bool rows(PyObject* o, Rows* r) {
    r->t = plain(o);
    if (!r->t || r->t->dim() != 2 || !dtype_of(r->t->scalar_type(), &r->dt)) return false;
    r->M = r->t->size(0);
    r->K = r->t->size(1);
    if (r->K > 1 && r->t->stride(1) != 1) return false;
    r->ld = r->M > 1 ? r->t->stride(0) : r->K;
    return true;
}

bool integer(PyObject* o, int64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}

PyObject *s_rowmajor, *s_tiled;
bool layout(PyObject* o, brq_layout* l) {
    if (!PyUnicode_CheckExact(o)) return false;
    const bool rm = o == s_rowmajor || PyUnicode_Compare(o, s_rowmajor) == 0;
    *l = rm ? BRQ_LAYOUT_ROWMAJOR : BRQ_LAYOUT_TILED;
    return rm || o == s_tiled || PyUnicode_Compare(o, s_tiled) == 0;
}

// Bytes of a quantized [rows][K] operand; sizes that are no operand's are left to Python.
bool operand_size(int64_t n, int64_t K, brq_layout l, int64_t* codes, int64_t* scales) {
    if (n < 0 || K <= 0 || K % 32 != 0 || n >= int64_t(1) << 31 || K >= int64_t(1) << 31) return false;
    if (l == BRQ_LAYOUT_TILED) {
        n = (n + 63) / 64 * 64;
        K = (K + 511) / 512 * 512;
    }
    *codes = n * (K / 2);
    *scales = n * (K / 32);
    return true;
}

bool signs_arg(PyObject* o, int64_t K, const int8_t** p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o);
    if (!t || !t->is_contiguous() || t->scalar_type() != at::kChar || t->numel() != K) return false;
    *p = static_cast<const int8_t*>(t->const_data_ptr());
    return true;
}

// Buffers that a quantizing call fills.
bool buffers(PyObject* c, PyObject* s, int64_t M, int64_t K, brq_layout l, uint8_t** codes, uint8_t** scales) {
    int64_t nc, ns;
    const at::Tensor *tc = bytes(c), *ts = bytes(s);
    if (!tc || !ts || !operand_size(M, K, l, &nc, &ns) || tc->numel() < nc || ts->numel() < ns) return false;
    *codes = static_cast<uint8_t*>(tc->data_ptr());
    *scales = static_cast<uint8_t*>(ts->data_ptr());
    return true;
}

// An operand of a product: codes and scales, `n` rows of K (either may be -1: not given; a row-major operand says).
bool operand(PyObject* c, PyObject* s, brq_layout l, int64_t* n, int64_t* K) {
    const at::Tensor *tc = bytes(c), *ts = bytes(s);
    if (!tc || !ts) return false;
    if (l == BRQ_LAYOUT_ROWMAJOR) {
        if (tc->dim() != 2 || (*n >= 0 && *n != tc->size(0)) || (*K >= 0 && *K != tc->size(1) * 2)) return false;
        *n = tc->size(0);
        *K = tc->size(1) * 2;
        if (ts->dim() != 2 || ts->size(0) != *n || ts->size(1) != *K / 32) return false;
    }
    return true;
}
const uint8_t* data(PyObject* o) { return static_cast<const uint8_t*>(THPVariable_Unpack(o).const_data_ptr()); }
bool operand_fits(PyObject* c, PyObject* s, brq_layout l, int64_t n, int64_t K) {
    int64_t nc, ns;
    return operand_size(n, K, l, &nc, &ns) && THPVariable_Unpack(c).numel() >= nc && THPVariable_Unpack(s).numel() >= ns;
}

// None or a size
bool size_arg(PyObject* o, int64_t* v) {
    *v = -1;
    return o == Py_None || (integer(o, v) && *v >= 0);
}

// The product's result: `out`, or a new tensor on the device of `like`.  The allocator may have to wait for the GPU, and the GPU
// for work that another thread has yet to launch: the lock is not held meanwhile, and addresses are read after it.
bool result(PyObject* out, PyObject* dtype, const at::Tensor& like, int64_t M, int64_t N, at::Tensor* y, brq_dtype* dt, int64_t* ldy) {
    if (out != Py_None) {
        Rows r;
        if (!rows(out, &r) || r.M != M || r.K != N) return false;
        *y = *r.t;
        *dt = r.dt;
        *ldy = r.ld;
        return true;
    }
    at::ScalarType s;
    if (!dtype_arg(dtype, &s, dt)) return false;
    const at::TensorOptions options = at::TensorOptions().dtype(s).device(like.device());
    {
        const Unlocked u;
        *y = at::empty({M, N}, options);
    }
    *ldy = N;
    return on_gpu(*y);
}

void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Nobody looks at what is done with tensors from outside (a function mode sees every look at a shape).
bool quiet() { return !at::impl::torch_function_mode_enabled(); }

template <class F>
brq_status released(F call) {
    const Unlocked u;
    return call();
}

PyObject* status(brq_status st) { return PyLong_FromLong((long)st); }
PyObject* result_or(brq_status st, PyObject* out, at::Tensor& y) {
    if (st != BRQ_OK) return status(st);
    if (out == Py_None) return THPVariable_Wrap(std::move(y));
    Py_INCREF(out);
    return out;
}

// rotate_quantize(x, B, codes, scales, layout, signs)
PyObject* rotate_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Rows x;
    int64_t B;
    brq_layout l;
    const int8_t* signs;
    uint8_t *codes, *scales;
    if (n != 6 || !f_rotate_quantize || !quiet() || !rows(a[0], &x) || !integer(a[1], &B) || !layout(a[4], &l) || !buffers(a[2], a[3], x.M, x.K, l, &codes, &scales) ||
        !signs_arg(a[5], x.K, &signs)) Py_RETURN_NONE;
    const void* p = x.t->const_data_ptr();
    void* s = current_stream();
    return status(released([&] { return f_rotate_quantize(p, x.dt, x.M, x.K, x.ld, B, signs, codes, scales, l, s); }));
    END_HANDLE_TH_ERRORS
}

// swiglu_rotate_quantize(gate, up, B, h_dtype, codes, scales, layout, signs)
PyObject* swiglu_rotate_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Rows g, u;
    int64_t B;
    brq_layout l;
    brq_dtype hd;
    at::ScalarType hs;
    const int8_t* signs;
    uint8_t *codes, *scales;
    if (n != 8 || !f_swiglu || !quiet() || !rows(a[0], &g) || !rows(a[1], &u) || g.M != u.M || g.K != u.K || g.dt != u.dt || !integer(a[2], &B) ||
        !dtype_arg(a[3], &hs, &hd) || !layout(a[6], &l) || !buffers(a[4], a[5], g.M, g.K, l, &codes, &scales) ||
        !signs_arg(a[7], g.K, &signs)) Py_RETURN_NONE;
    const void *pg = g.t->const_data_ptr(), *pu = u.t->const_data_ptr();
    void* s = current_stream();
    return status(released([&] { return f_swiglu(pg, pu, g.dt, g.M, g.K, g.ld, u.ld, hd, B, signs, codes, scales, l, s); }));
    END_HANDLE_TH_ERRORS
}

// matrix_rotate_quantize(x, R, codes, scales, layout)
PyObject* matrix_rotate_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Rows x;
    brq_layout l;
    uint8_t *codes, *scales;
    const at::Tensor* R = n == 5 && f_matrix && quiet() ? plain(a[1]) : nullptr;
    if (!R || !R->is_contiguous() || R->scalar_type() != at::kFloat || R->dim() < 2 || R->dim() > 3 || R->size(-1) != 32 || R->size(-2) != 32 ||
        !rows(a[0], &x) || !layout(a[4], &l) || !buffers(a[2], a[3], x.M, x.K, l, &codes, &scales)) Py_RETURN_NONE;
    const int64_t nR = R->dim() == 3 ? R->size(0) : 1;
    const void* p = x.t->const_data_ptr();
    const float* r = static_cast<const float*>(R->const_data_ptr());
    void* s = current_stream();
    return status(released([&] { return f_matrix(p, x.dt, x.M, x.K, x.ld, r, nR, codes, scales, l, s); }));
    END_HANDLE_TH_ERRORS
}

// gemm(aq, as, wq, ws, out_dtype, out, a_layout, w_layout, M, N, K)
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    brq_layout la, lw;
    int64_t M, N, K, ldy;
    at::Tensor y;
    brq_dtype dt;
    if (n != 11 || !f_gemm || !quiet() || !layout(a[6], &la) || !layout(a[7], &lw) || !size_arg(a[8], &M) || !size_arg(a[9], &N) || !size_arg(a[10], &K) ||
        !operand(a[0], a[1], la, &M, &K) || !operand(a[2], a[3], lw, &N, &K) || M < 0 || N < 0 || K < 0 ||
        !operand_fits(a[0], a[1], la, M, K) || !operand_fits(a[2], a[3], lw, N, K) ||
        !result(a[5], a[4], THPVariable_Unpack(a[0]), M, N, &y, &dt, &ldy)) Py_RETURN_NONE;
    const uint8_t *ac = data(a[0]), *as = data(a[1]), *wc = data(a[2]), *ws = data(a[3]);
    void *p = y.data_ptr(), *s = current_stream();
    return result_or(released([&] { return f_gemm(ac, as, la, wc, ws, lw, M, N, K, p, dt, ldy, s); }), a[5], y);
    END_HANDLE_TH_ERRORS
}

// rotate_quantize_gemm(x, B, wq, ws, N, out_dtype, out, w_layout, signs)
PyObject* rotate_quantize_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Rows x;
    brq_layout l;
    int64_t B, N, ldy;
    const int8_t* signs;
    at::Tensor y;
    brq_dtype dt;
    if (n != 9 || !f_decode || !quiet() || !rows(a[0], &x) || !integer(a[1], &B) || !bytes(a[2]) || !bytes(a[3]) || !integer(a[4], &N) || !layout(a[7], &l) ||
        !signs_arg(a[8], x.K, &signs) || !operand_fits(a[2], a[3], l, N, x.K) || !result(a[6], a[5], *x.t, x.M, N, &y, &dt, &ldy)) Py_RETURN_NONE;
    const void* p = x.t->const_data_ptr();
    if (signs) signs = reinterpret_cast<const int8_t*>(data(a[8]));
    const uint8_t *wc = data(a[2]), *ws = data(a[3]);
    void *q = y.data_ptr(), *s = current_stream();
    return result_or(released([&] { return f_decode(p, x.dt, x.M, x.K, x.ld, B, signs, wc, ws, l, N, q, dt, ldy, s); }), a[6], y);
    END_HANDLE_TH_ERRORS
}

// ---- the analysis: the two statistics calls and the summary of a comparison of up to 8 M values took 45 us, all of it the
// host; 33 now (six launches, seven new tensors).

// Numbers as float32, as ctypes makes them of float(t): up to `most`.
bool number(PyObject* o, double* v) {
    if (PyFloat_CheckExact(o)) *v = PyFloat_AS_DOUBLE(o);
    else if (PyLong_CheckExact(o)) *v = PyLong_AsDouble(o);
    else return false;
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}
bool numbers(PyObject* o, float* v, int most, int* n) {
    if (!PyTuple_CheckExact(o) && !PyList_CheckExact(o)) return false;
    const Py_ssize_t len = PySequence_Fast_GET_SIZE(o);
    if (len > most) return false;
    *n = (int)len;
    for (int i = 0; i < *n; ++i) {
        double d;
        if (!number(PySequence_Fast_GET_ITEM(o, i), &d)) return false;
        v[i] = (float)d;
    }
    return true;
}

// An output or input of one type: None (`*t` stays undefined), or contiguous with its sizes.
bool array(PyObject* o, at::ScalarType s, at::IntArrayRef sizes, at::Tensor* t) {
    if (o == Py_None) return true;
    const at::Tensor* p = plain(o);
    if (!p || p->scalar_type() != s || !p->is_contiguous() || p->sizes() != sizes) return false;
    *t = *p;
    return true;
}
bool flat_array(PyObject* o, at::ScalarType s, int64_t n, at::Tensor* t) {
    if (o == Py_None) return true;
    const at::Tensor* p = plain(o);
    if (!p || p->scalar_type() != s || !p->is_contiguous() || p->numel() != n) return false;
    *t = *p;
    return true;
}
template <class T>
T* address(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }
// the caller's own object, or the new tensor, or None
PyObject* handed(PyObject* given, at::Tensor& t) {
    if (given == Py_None && t.defined()) return THPVariable_Wrap(std::move(t));
    Py_INCREF(given);
    return given;
}
PyObject* three(PyObject* a, PyObject* b, PyObject* c) {
    PyObject* r = a && b && c ? PyTuple_Pack(3, a, b, c) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    Py_XDECREF(c);
    return r;
}

// block_stats(x, B, thresholds, signs, counts, want_amax, want_sqerr, amax, sqerr)
PyObject* block_stats(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Rows x;
    int64_t B;
    float th[8];
    int nt;
    const int8_t* signs;
    at::Tensor counts, amax, sqerr;
    if (n != 9 || !f_stats || !quiet() || !rows(a[0], &x) || x.M <= 0 || x.K <= 0 || x.K % 32 != 0 || !integer(a[1], &B) || !numbers(a[2], th, 8, &nt) ||
        !signs_arg(a[3], x.K, &signs) || !flat_array(a[4], at::kLong, nt, &counts) || !PyBool_Check(a[5]) || !PyBool_Check(a[6])) Py_RETURN_NONE;
    const int64_t shape[2] = {x.M, x.K / 32};
    if (!array(a[7], at::kFloat, shape, &amax) || !array(a[8], at::kFloat, shape, &sqerr)) Py_RETURN_NONE;
    const at::TensorOptions f32 = at::TensorOptions().dtype(at::kFloat).device(x.t->device());
    {
        const Unlocked u;
        if (!amax.defined() && a[5] == Py_True) amax = at::empty(shape, f32);
        if (!sqerr.defined() && a[6] == Py_True) sqerr = at::empty(shape, f32);
        if (!counts.defined() && nt) counts = at::zeros({nt}, f32.dtype(at::kLong));
    }
    for (const at::Tensor* t : {&amax, &sqerr, &counts})
        if (t->defined() && !on_gpu(*t)) Py_RETURN_NONE;
    const void* p = x.t->const_data_ptr();
    if (signs) signs = reinterpret_cast<const int8_t*>(data(a[3]));
    float *pa = address<float>(amax), *ps = address<float>(sqerr);
    uint64_t* pc = address<uint64_t>(counts);
    void* s = current_stream();
    const brq_status st = released([&] { return f_stats(p, x.dt, x.M, x.K, x.ld, B, signs, th, nt, pa, pc, ps, nullptr, s); });
    return st != BRQ_OK ? status(st) : three(handed(a[7], amax), handed(a[4], counts), handed(a[8], sqerr));
    END_HANDLE_TH_ERRORS
}

// block_stats_summary(amax, sqerr, amax_ref, outlier_threshold, edges, hist, counts, sums)
PyObject* block_stats_summary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor* amax = n == 8 && f_summary && quiet() ? plain(a[0]) : nullptr;
    if (!amax || amax->scalar_type() != at::kFloat || !amax->is_contiguous() || amax->numel() == 0) Py_RETURN_NONE;
    const int64_t blocks = amax->numel();
    at::Tensor sqerr, ref, hist, counts, sums;
    double outlier;
    float edges[32];
    int ne;
    if (!flat_array(a[1], at::kFloat, blocks, &sqerr) || !flat_array(a[2], at::kFloat, blocks, &ref) || !number(a[3], &outlier) || !numbers(a[4], edges, 32, &ne) ||
        !flat_array(a[5], at::kLong, ne + 1, &hist) || !flat_array(a[6], at::kLong, 4, &counts) || !flat_array(a[7], at::kDouble, 4, &sums)) Py_RETURN_NONE;
    const at::TensorOptions i64 = at::TensorOptions().dtype(at::kLong).device(amax->device());
    {
        const Unlocked u;
        std::vector<at::Tensor> made;                          // each a tensor of its own, cleared by one launch
        if (!hist.defined()) made.push_back(hist = at::empty({ne + 1}, i64));
        if (!counts.defined()) made.push_back(counts = at::empty({4}, i64));
        if (!sums.defined()) made.push_back((sums = at::empty({4}, i64.dtype(at::kDouble))).view(at::kLong));
        if (!made.empty()) at::_foreach_zero_(made);
    }
    for (const at::Tensor* t : {&hist, &counts, &sums})
        if (!on_gpu(*t)) Py_RETURN_NONE;
    const float *pa = static_cast<const float*>(THPVariable_Unpack(a[0]).const_data_ptr()), *pq = address<float>(sqerr), *pr = address<float>(ref);
    uint64_t *ph = address<uint64_t>(hist), *pc = address<uint64_t>(counts);
    double* pd = address<double>(sums);
    void* s = current_stream();
    const brq_status st = released([&] { return f_summary(pa, pq, pr, blocks, (float)outlier, edges, ne, ph, pc, pd, s); });
    return st != BRQ_OK ? status(st) : three(handed(a[5], hist), handed(a[6], counts), handed(a[7], sums));
    END_HANDLE_TH_ERRORS
}

// bind_stats(addresses of brq_block_stats and brq_block_stats_summary)
PyObject* bind_stats(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[2];
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "bind_stats takes the addresses of two entry points");
        return nullptr;
    }
    for (int i = 0; i < 2; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point's address is NULL");
            return nullptr;
        }
    }
    f_stats = reinterpret_cast<decltype(f_stats)>(p[0]);
    f_summary = reinterpret_cast<decltype(f_summary)>(p[1]);
    Py_RETURN_NONE;
}

// bind(addresses of the entry points of a layer, in the order above)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[5];
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind takes the addresses of five entry points");
        return nullptr;
    }
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point's address is NULL");
            return nullptr;
        }
    }
    f_rotate_quantize = reinterpret_cast<decltype(f_rotate_quantize)>(p[0]);
    f_swiglu = reinterpret_cast<decltype(f_swiglu)>(p[1]);
    f_matrix = reinterpret_cast<decltype(f_matrix)>(p[2]);
    f_gemm = reinterpret_cast<decltype(f_gemm)>(p[3]);
    f_decode = reinterpret_cast<decltype(f_decode)>(p[4]);
    Py_RETURN_NONE;
}

// ---- the attention side: through Python and ctypes a call took 9 to 20 us of the host (a decoding step's two 41), the GPU 5 to 8.
// `o`: None where that is allowed, else a tensor that fits, or the call is left to Python.

decltype(&brq_qk_norm_rope) f_norm;
decltype(&brq_qk_norm_rope_backward) f_norm_back;
decltype(&brq_qk_norm_rope_backward_workspace) f_norm_back_space;
decltype(&brq_kv4_append) f_append;
decltype(&brq_kv4_read) f_read;
decltype(&brq_kv4_attention) f_attention;
decltype(&brq_kv4_attention_workspace) f_attention_space;
decltype(&brq_kv4_pages_workspace) f_pages_space;
decltype(&brq_kv4_pages_copy) f_copy;
decltype(&brq_kv4_pages_fork) f_fork;
decltype(&brq_kv4_pages_free) f_free;
decltype(&brq_kv4_pages_reserve) f_reserve;
decltype(&brq_kv4_pages_compact) f_compact;
bool g_attention;                    // bind_attention() was called

// The tensors of a call: on one device, the current one.
struct Call {
    c10::DeviceIndex device = -1;
    const at::Tensor* take(PyObject* o) {
        const at::Tensor* t = plain(o);
        if (!t) return nullptr;
        if (device < 0) {
            if (t->device().index() != c10::hip::current_device()) return nullptr;
            device = t->device().index();
        }
        return t->device().index() == device ? t : nullptr;
    }
    at::TensorOptions options(at::ScalarType s) const { return at::TensorOptions().dtype(s).device(c10::DeviceType::CUDA, device); }
};

struct HeadSet {
    at::Tensor t;                    // undefined: None
    brq_heads h{};
    int64_t T = 0, D = 0;
    brq_dtype dt = BRQ_F32;
    const brq_heads* get() const { return t.defined() ? &h : nullptr; }
    void fill() { h = brq_heads{t.data_ptr(), t.size(1), t.stride(0), t.stride(1)}; }
};
bool head_set(Call& c, PyObject* o, HeadSet* x, bool optional = false) {
    if (optional && o == Py_None) return true;
    const at::Tensor* t = c.take(o);
    if (!t || t->dim() != 3 || (t->size(2) > 1 && t->stride(2) != 1) || !dtype_of(t->scalar_type(), &x->dt)) return false;
    x->t = *t;
    x->T = t->size(0);
    x->D = t->size(2);
    x->fill();
    return true;
}
bool same_tokens(const HeadSet& a, const HeadSet& b) { return !b.t.defined() || (a.T == b.T && a.D == b.D && a.dt == b.dt); }
// An output: given, of `like`'s sizes and type `s`, or to be made.
bool head_out(Call& c, PyObject* o, const HeadSet& like, at::ScalarType s, HeadSet* x) {
    if (!like.t.defined()) return o == Py_None;
    if (o == Py_None) return true;
    return head_set(c, o, x) && x->t.sizes() == like.t.sizes() && x->t.scalar_type() == s;
}
bool make(const Call& c, at::IntArrayRef sizes, at::ScalarType s, at::Tensor* t) {
    if (!t->defined()) {
        const Unlocked u;
        *t = at::empty(sizes, c.options(s));
    }
    return on_gpu(*t);
}
bool make_heads(const Call& c, const HeadSet& like, at::ScalarType s, HeadSet* x) {
    if (!like.t.defined()) return true;
    if (!make(c, like.t.sizes(), s, &x->t)) return false;
    x->fill();
    return true;
}
at::ScalarType scalar_of(brq_dtype d) { return d == BRQ_BF16 ? at::kBFloat16 : at::kFloat; }

// A contiguous array of one type; sizes of -1 are any.
bool array_of(Call& c, PyObject* o, at::ScalarType s, std::initializer_list<int64_t> sizes, at::Tensor* t, bool optional = false) {
    if (optional && o == Py_None) return true;
    const at::Tensor* p = c.take(o);
    if (!p || p->scalar_type() != s || !p->is_contiguous() || p->dim() != (int64_t)sizes.size()) return false;
    int i = 0;
    for (int64_t n : sizes)
        if (const int64_t m = p->size(i++); n >= 0 && n != m) return false;
    *t = *p;
    return true;
}

// wq, wk, eps, cos, sin, positions, interleaved, B: the arguments a[0] ... a[7] of the passes over heads
struct NormArgs {
    at::Tensor wq, wk, cos, sin, pos;
    double eps;
    int64_t B;
    brq_rope r{};
    const brq_rope* rope() const { return cos.defined() ? &r : nullptr; }
};
bool norm_args(Call& c, PyObject* const* a, int64_t T, int64_t D, NormArgs* n) {
    if (!array_of(c, a[0], at::kFloat, {D}, &n->wq, true) || !array_of(c, a[1], at::kFloat, {D}, &n->wk, true) || !number(a[2], &n->eps) ||
        !PyBool_Check(a[6]) || !integer(a[7], &n->B)) return false;
    if (a[3] == Py_None) return a[4] == Py_None && a[5] == Py_None;
    if (!array_of(c, a[3], at::kFloat, {-1, -1}, &n->cos) || !array_of(c, a[4], at::kFloat, {n->cos.size(0), n->cos.size(1)}, &n->sin) ||
        !array_of(c, a[5], at::kLong, {T}, &n->pos)) return false;
    n->r = brq_rope{address<float>(n->cos), address<float>(n->sin), address<int64_t>(n->pos), n->cos.size(0), n->cos.size(1) * 2, a[6] == Py_True};
    return true;
}

PyObject* wrapped(PyObject* given, at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return handed(given, t);
}
template <int N>
PyObject* tuple_of(PyObject* (&items)[N]) {
    bool fine = true;
    for (PyObject* o : items) fine = fine && o;
    PyObject* r = fine ? PyTuple_New(N) : nullptr;
    for (int i = 0; i < N; ++i) {
        if (r) PyTuple_SET_ITEM(r, i, items[i]);
        else Py_XDECREF(items[i]);
    }
    return r;
}

// qk_norm_rope(q, k, wq, wk, eps, cos, sin, positions, interleaved, B, out_dtype, q_out, k_out)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    HeadSet q, k, qo, ko;
    NormArgs m;
    at::ScalarType s;
    brq_dtype dt;
    if (n != 13 || !g_attention || !quiet() || !head_set(c, a[0], &q) || !head_set(c, a[1], &k, true) || !same_tokens(q, k) || !norm_args(c, a + 2, q.T, q.D, &m)) Py_RETURN_NONE;
    if (a[11] != Py_None) {
        if (!head_set(c, a[11], &qo)) Py_RETURN_NONE;
        s = qo.t.scalar_type();
    } else if (a[10] == Py_None) {
        s = q.t.scalar_type();
    } else if (!dtype_arg(a[10], &s, &dt)) {
        Py_RETURN_NONE;
    }
    if (!head_out(c, a[11], q, s, &qo) || !head_out(c, a[12], k, s, &ko) || !make_heads(c, q, s, &qo) || !make_heads(c, k, s, &ko) || !dtype_of(s, &dt)) Py_RETURN_NONE;
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_norm(q.get(), k.get(), q.dt, q.T, q.D, address<float>(m.wq), address<float>(m.wk), (float)m.eps, m.rope(), m.B, qo.get(), ko.get(), dt, st);
    });
    if (r != BRQ_OK) return status(r);
    PyObject* items[2] = {wrapped(a[11], qo.t), wrapped(a[12], ko.t)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

// qk_norm_rope_backward(q, k, gq, gk, wq, wk, eps, cos, sin, positions, interleaved, B, dq, dk, workspace)
PyObject* qk_norm_rope_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    HeadSet q, k, gq, gk, dq, dk;
    NormArgs m;
    at::Tensor dwq, dwk, space;
    if (n != 15 || !g_attention || !quiet() || !head_set(c, a[0], &q) || !head_set(c, a[1], &k, true) || !same_tokens(q, k) || !head_set(c, a[2], &gq) || !head_set(c, a[3], &gk, true) ||
        gq.t.sizes() != q.t.sizes() || k.t.defined() != gk.t.defined() || (k.t.defined() && (gk.t.sizes() != k.t.sizes() || gk.dt != gq.dt)) ||
        !norm_args(c, a + 4, q.T, q.D, &m) || !array_of(c, a[14], at::kByte, {-1}, &space, true)) Py_RETURN_NONE;
    const at::ScalarType s = q.t.scalar_type();
    if (!head_out(c, a[12], q, s, &dq) || !head_out(c, a[13], k, s, &dk) || !make_heads(c, q, s, &dq) || !make_heads(c, k, s, &dk)) Py_RETURN_NONE;
    int64_t need = 0;
    if (m.wq.defined() || (m.wk.defined() && k.t.defined())) {
        if (const brq_status r = f_norm_back_space(q.T, q.h.heads, k.t.defined() ? k.h.heads : 0, q.D, &need); r != BRQ_OK) return status(r);
        if (need && !make(c, {need}, at::kByte, &space)) Py_RETURN_NONE;
    }
    if ((m.wq.defined() && !make(c, {q.D}, at::kFloat, &dwq)) || (m.wk.defined() && k.t.defined() && !make(c, {q.D}, at::kFloat, &dwk))) Py_RETURN_NONE;
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_norm_back(q.get(), k.get(), q.dt, q.T, q.D, address<float>(m.wq), address<float>(m.wk), (float)m.eps, m.rope(), m.B, gq.get(), gk.get(), gq.dt, dq.get(),
                           dk.get(), address<float>(dwq), address<float>(dwk), address<void>(space), space.defined() ? space.numel() : 0, st);
    });
    if (r != BRQ_OK) return status(r);
    PyObject* items[4] = {wrapped(a[12], dq.t), wrapped(a[13], dk.t), wrapped(Py_None, dwq), wrapped(Py_None, dwk)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

// A cache of heads of D channels; *Hk: its heads, to be found where negative.
bool cache(Call& c, PyObject* o, int64_t D, int64_t* Hk, at::Tensor* t) {
    if (!array_of(c, o, at::kByte, {-1, -1}, t) || D <= 0 || t->size(1) % (68 * D) != 0 || t->size(1) < 68 * D) return false;
    if (*Hk < 0) *Hk = t->size(1) / (68 * D);
    return *Hk * 68 * D == t->size(1);
}

// kv4_append(pool, slots, k, v, q, wq, wk, eps, cos, sin, positions, interleaved, B, Bv, q_out); True: there is no q
PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    HeadSet q, k, v, qo;
    NormArgs m;
    at::Tensor pool, slots;
    int64_t Bv;
    if (n != 15 || !g_attention || !quiet() || !head_set(c, a[2], &k) || !head_set(c, a[3], &v) || v.t.sizes() != k.t.sizes() || v.dt != k.dt || !head_set(c, a[4], &q, true) ||
        !same_tokens(k, q) || !norm_args(c, a + 5, k.T, k.D, &m) || !integer(a[13], &Bv) || !array_of(c, a[1], at::kLong, {k.T}, &slots)) Py_RETURN_NONE;
    int64_t Hk = k.h.heads;
    if (!cache(c, a[0], k.D, &Hk, &pool) || !head_out(c, a[14], q, scalar_of(k.dt), &qo) || !make_heads(c, q, scalar_of(k.dt), &qo)) Py_RETURN_NONE;
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_append(q.get(), k.get(), v.get(), k.dt, k.T, k.D, address<float>(m.wq), address<float>(m.wk), (float)m.eps, m.rope(), m.B, Bv, address<int64_t>(slots),
                        address<uint8_t>(pool), pool.size(0), qo.get(), st);
    });
    if (r != BRQ_OK) return status(r);
    if (!q.t.defined()) Py_RETURN_TRUE;
    return wrapped(a[14], qo.t);
    END_HANDLE_TH_ERRORS
}

// kv4_read(pool, slots, D, out_dtype, k_out, v_out)
PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    HeadSet k, v;
    at::Tensor pool, slots;
    int64_t D, Hk = -1;
    at::ScalarType s;
    brq_dtype dt;
    if (n != 6 || !g_attention || !quiet() || !integer(a[2], &D) || !cache(c, a[0], D, &Hk, &pool) || !array_of(c, a[1], at::kLong, {-1}, &slots) || !dtype_arg(a[3], &s, &dt)) Py_RETURN_NONE;
    const int64_t shape[3] = {slots.size(0), Hk, D};
    const at::IntArrayRef sizes(shape);
    if (!head_set(c, a[4], &k, true) || (k.t.defined() && k.t.sizes() != sizes)) Py_RETURN_NONE;
    if (k.t.defined()) s = k.t.scalar_type();
    if (!head_set(c, a[5], &v, true) || (v.t.defined() && (v.t.sizes() != sizes || v.t.scalar_type() != s)) || !make(c, sizes, s, &k.t) || !make(c, sizes, s, &v.t)) Py_RETURN_NONE;
    k.fill();
    v.fill();
    dtype_of(s, &dt);
    void* st = current_stream();
    const brq_status r = released([&] { return f_read(address<uint8_t>(pool), pool.size(0), sizes[0], D, address<int64_t>(slots), k.get(), v.get(), dt, st); });
    if (r != BRQ_OK) return status(r);
    PyObject* items[2] = {wrapped(a[4], k.t), wrapped(a[5], v.t)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

// kv4_attention(q, pool, table, kv_lens, scale, causal, window, cu_q, max_q, max_kv, out, lse, want_lse, workspace); scale, max_q and max_kv may be None
PyObject* kv4_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    HeadSet q, out;
    at::Tensor pool, table, lens, cu, lse, space;
    double scale = 0.0;
    int64_t Hk = -1, window, max_q = 0, max_kv = 0, need = 0;
    if (n != 14 || !g_attention || !quiet() || !head_set(c, a[0], &q) || q.dt != BRQ_BF16 || !cache(c, a[1], q.D, &Hk, &pool) || !array_of(c, a[2], at::kInt, {-1, -1}, &table) ||
        !array_of(c, a[3], at::kInt, {table.size(0)}, &lens) || !array_of(c, a[7], at::kInt, {table.size(0) + 1}, &cu, true) || (!cu.defined() && q.T != table.size(0)) ||
        (a[4] != Py_None && !number(a[4], &scale)) || !PyBool_Check(a[5]) || !integer(a[6], &window) || (a[8] != Py_None && !integer(a[8], &max_q)) ||
        (a[9] != Py_None && !integer(a[9], &max_kv)) ||
        !head_out(c, a[10], q, at::kBFloat16, &out) || !array_of(c, a[11], at::kFloat, {q.T, q.h.heads}, &lse, true) || !PyBool_Check(a[12]) ||
        !array_of(c, a[13], at::kByte, {-1}, &space, true)) Py_RETURN_NONE;
    const int64_t S = table.size(0);
    if (a[4] == Py_None) scale = 1.0 / std::sqrt((double)q.D);
    if (a[8] == Py_None) max_q = cu.defined() ? std::max<int64_t>(1, q.T) : 1;
    if (a[9] == Py_None) max_kv = table.size(1) * BRQ_KV4_PAGE;
    if (const brq_status r = f_attention_space(q.T, S, q.h.heads, Hk, q.D, max_q, max_kv, &need); r != BRQ_OK) return status(r);
    if (!make_heads(c, q, at::kBFloat16, &out) || (a[12] == Py_True && !make(c, {q.T, q.h.heads}, at::kFloat, &lse)) || (need && !make(c, {need}, at::kByte, &space))) Py_RETURN_NONE;
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_attention(q.get(), q.T, q.D, address<uint8_t>(pool), pool.size(0), Hk, address<int32_t>(table), table.size(1), address<int32_t>(lens), address<int32_t>(cu), S,
                           (float)scale, a[5] == Py_True, window, max_q, max_kv, out.get(), address<float>(lse), address<void>(space), space.defined() ? space.numel() : 0, st);
    });
    if (r != BRQ_OK) return status(r);
    if (!lse.defined()) return wrapped(a[10], out.t);
    PyObject* items[2] = {wrapped(a[10], out.t), wrapped(a[11], lse)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

// A scheduler's state and two lists of one length
struct PageState {
    at::Tensor table, lens, refs, x, y, space, result;
    bool state(Call& c, PyObject* t, PyObject* l, PyObject* r, int64_t pages) {
        return array_of(c, t, at::kInt, {-1, -1}, &table) && (!l || array_of(c, l, at::kInt, {table.size(0)}, &lens)) && array_of(c, r, at::kInt, {pages}, &refs);
    }
    bool lists(Call& c, PyObject* a, PyObject* b) { return array_of(c, a, at::kInt, {-1}, &x) && (!b || array_of(c, b, at::kInt, {x.size(0)}, &y)); }
    bool room(Call& c, PyObject* o, int64_t n) {
        int64_t need = 0;
        return array_of(c, o, at::kByte, {-1}, &space, true) && f_pages_space(n, refs.size(0), &need) == BRQ_OK && make(c, {need}, at::kByte, &space) &&
               space.numel() >= need && make(c, {1}, at::kInt, &result);
    }
    PyObject* answer(brq_status r) { return r != BRQ_OK ? status(r) : THPVariable_Wrap(std::move(result)); }
};

// kv4_pages_copy(pool, src, dst) -> status
PyObject* kv4_pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    PageState p;
    at::Tensor pool;
    if (n != 3 || !g_attention || !quiet() || !array_of(c, a[0], at::kByte, {-1, -1}, &pool) || !p.lists(c, a[1], a[2])) Py_RETURN_NONE;
    void* st = current_stream();
    return status(released([&] { return f_copy(address<uint8_t>(pool), pool.size(1), pool.size(0), address<int32_t>(p.x), address<int32_t>(p.y), p.x.size(0), st); }));
    END_HANDLE_TH_ERRORS
}

// kv4_pages_fork(pool, table, lens, refs, parents, children, workspace) -> failed
PyObject* kv4_pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    PageState p;
    at::Tensor pool;
    if (n != 7 || !g_attention || !quiet() || !array_of(c, a[0], at::kByte, {-1, -1}, &pool) || !p.state(c, a[1], a[2], a[3], pool.size(0)) || !p.lists(c, a[4], a[5]) ||
        !p.room(c, a[6], p.x.size(0))) Py_RETURN_NONE;
    void* st = current_stream();
    return p.answer(released([&] {
        return f_fork(address<uint8_t>(pool), pool.size(1), pool.size(0), address<int32_t>(p.table), p.table.size(0), p.table.size(1), address<int32_t>(p.lens), address<int32_t>(p.refs),
                      address<int32_t>(p.x), address<int32_t>(p.y), p.x.size(0), address<int32_t>(p.result), address<void>(p.space), st);
    }));
    END_HANDLE_TH_ERRORS
}

// kv4_pages_free(table, lens, refs, seqs) -> status
PyObject* kv4_pages_free(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    PageState p;
    if (n != 4 || !g_attention || !quiet() || !p.state(c, a[0], a[1], a[2], -1) || !p.lists(c, a[3], nullptr)) Py_RETURN_NONE;
    void* st = current_stream();
    return status(released([&] {
        return f_free(address<int32_t>(p.table), p.table.size(0), p.table.size(1), address<int32_t>(p.lens), address<int32_t>(p.refs), p.refs.size(0), address<int32_t>(p.x), p.x.size(0), st);
    }));
    END_HANDLE_TH_ERRORS
}

// kv4_pages_reserve(table, refs, seqs, tokens, workspace) -> failed
PyObject* kv4_pages_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    PageState p;
    if (n != 5 || !g_attention || !quiet() || !p.state(c, a[0], nullptr, a[1], -1) || !p.lists(c, a[2], a[3]) || !p.room(c, a[4], p.x.size(0))) Py_RETURN_NONE;
    void* st = current_stream();
    return p.answer(released([&] {
        return f_reserve(address<int32_t>(p.table), p.table.size(0), p.table.size(1), address<int32_t>(p.refs), p.refs.size(0), address<int32_t>(p.x), address<int32_t>(p.y), p.x.size(0),
                         address<int32_t>(p.result), address<void>(p.space), st);
    }));
    END_HANDLE_TH_ERRORS
}

// kv4_pages_compact(pool, table, refs, workspace) -> live
PyObject* kv4_pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    PageState p;
    at::Tensor pool;
    if (n != 4 || !g_attention || !quiet() || !array_of(c, a[0], at::kByte, {-1, -1}, &pool) || !p.state(c, a[1], nullptr, a[2], pool.size(0)) || !p.room(c, a[3], 0)) Py_RETURN_NONE;
    void* st = current_stream();
    return p.answer(released([&] {
        return f_compact(address<uint8_t>(pool), pool.size(1), pool.size(0), address<int32_t>(p.table), p.table.size(0), p.table.size(1), address<int32_t>(p.refs),
                         address<int32_t>(p.result), address<void>(p.space), st);
    }));
    END_HANDLE_TH_ERRORS
}

// bind_attention(addresses of the entry points of the attention side, in the order of their declaration above)
PyObject* bind_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[13];
    if (n != 13) {
        PyErr_SetString(PyExc_TypeError, "bind_attention takes the addresses of thirteen entry points");
        return nullptr;
    }
    for (int i = 0; i < 13; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point's address is NULL");
            return nullptr;
        }
    }
    int i = 0;
    auto set = [&](auto& f) { f = reinterpret_cast<std::decay_t<decltype(f)>>(p[i++]); };
    set(f_norm), set(f_norm_back), set(f_norm_back_space), set(f_append), set(f_read), set(f_attention), set(f_attention_space), set(f_pages_space), set(f_copy), set(f_fork),
        set(f_free), set(f_reserve), set(f_compact);
    g_attention = true;
    Py_RETURN_NONE;
}

// ---- the residual side (brq_residual.h)

decltype(&brq_add_rms_norm) f_add_norm;
decltype(&brq_add_rms_norm_backward) f_add_norm_back;
decltype(&brq_add_rms_norm_backward_workspace) f_add_norm_back_space;
decltype(&brq_add_rms_norm_rotate_quantize_fused) f_add_norm_quantize;
decltype(&brq_mxfp4_gemm_epilogue) f_gemm_epilogue;
decltype(&brq_mxfp4_gemm_epilogue_workspace) f_gemm_epilogue_space;
bool g_residual;                     // bind_residual() was called

// A matrix of a call, or one to be made: rows of any pitch.
struct Matrix {
    at::Tensor t;                    // undefined: None
    int64_t ld = 0;
    brq_dtype dt = BRQ_F32;
    void fill() { ld = t.size(0) > 1 ? t.stride(0) : t.size(1); }
    void* p() const { return t.defined() ? t.data_ptr() : nullptr; }
};
bool matrix(Call& c, PyObject* o, Matrix* x, bool optional = false) {
    if (optional && o == Py_None) return true;
    const at::Tensor* t = c.take(o);
    if (!t || t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1) || !dtype_of(t->scalar_type(), &x->dt)) return false;
    x->t = *t;
    x->fill();
    return true;
}
bool same_sizes(const Matrix& a, const Matrix& b) { return !b.t.defined() || a.t.sizes() == b.t.sizes(); }
// `o`, of `like`'s sizes and type `s`, or a new one.
bool matrix_out(Call& c, PyObject* o, const Matrix& like, at::ScalarType s, Matrix* x) {
    if (o != Py_None) return matrix(c, o, x) && same_sizes(like, *x) && x->t.scalar_type() == s;
    if (!make(c, like.t.sizes(), s, &x->t)) return false;
    x->fill();
    return dtype_of(s, &x->dt);
}
// The sum of x and the residual: none without a residual, and where nobody asks for it.
bool sum_out(Call& c, PyObject* h_out, PyObject* want, const Matrix& x, const Matrix& res, Matrix* h) {
    if (!PyBool_Check(want)) return false;
    if (!res.t.defined()) return h_out == Py_None;
    return (h_out == Py_None && want == Py_False) || matrix_out(c, h_out, x, res.t.scalar_type(), h);
}

// add_rms_norm(x, residual, weight, eps, out_dtype, out, h_out, want_h)
PyObject* add_rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    Matrix x, res, y, h;
    at::Tensor w;
    double eps;
    at::ScalarType s;
    brq_dtype dt;
    if (n != 8 || !g_residual || !quiet() || !matrix(c, a[0], &x) || !matrix(c, a[1], &res, true) || !same_sizes(x, res) ||
        !array_of(c, a[2], at::kFloat, {x.t.size(1)}, &w, true) || !number(a[3], &eps)) Py_RETURN_NONE;
    if (a[5] != Py_None) {
        const at::Tensor* t = c.take(a[5]);
        if (!t) Py_RETURN_NONE;
        s = t->scalar_type();
    } else if (a[4] == Py_None) {
        s = x.t.scalar_type();
    } else if (!dtype_arg(a[4], &s, &dt)) {
        Py_RETURN_NONE;
    }
    if (!matrix_out(c, a[5], x, s, &y) || !sum_out(c, a[6], a[7], x, res, &h)) Py_RETURN_NONE;
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_add_norm(x.p(), x.dt, x.ld, res.p(), res.dt, res.ld, x.t.size(0), x.t.size(1), address<float>(w), (float)eps, h.p(), h.ld, y.p(), y.dt, y.ld, st);
    });
    if (r != BRQ_OK) return status(r);
    PyObject* items[2] = {wrapped(a[5], y.t), wrapped(a[6], h.t)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

// add_rms_norm_backward(h, gy, gh, weight, eps, dh, workspace)
PyObject* add_rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    Matrix h, gy, gh, dh;
    at::Tensor w, dw, space;
    double eps;
    if (n != 7 || !g_residual || !quiet() || !matrix(c, a[0], &h) || !matrix(c, a[1], &gy) || !matrix(c, a[2], &gh, true) || !same_sizes(h, gy) || !same_sizes(h, gh) ||
        (gh.t.defined() && gh.dt != h.dt) || !array_of(c, a[3], at::kFloat, {h.t.size(1)}, &w, true) || !number(a[4], &eps) ||
        !array_of(c, a[6], at::kByte, {-1}, &space, true) || !matrix_out(c, a[5], h, h.t.scalar_type(), &dh)) Py_RETURN_NONE;
    const int64_t M = h.t.size(0), K = h.t.size(1);
    if (w.defined()) {
        int64_t need = 0;
        if (const brq_status r = f_add_norm_back_space(M, K, &need); r != BRQ_OK) return status(r);
        if ((need && !make(c, {need}, at::kByte, &space)) || !make(c, {K}, at::kFloat, &dw)) Py_RETURN_NONE;
    }
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_add_norm_back(h.p(), h.dt, h.ld, gy.p(), gy.dt, gy.ld, gh.p(), gh.ld, M, K, address<float>(w), (float)eps, dh.p(), dh.ld, address<float>(dw),
                               address<void>(space), space.defined() ? space.numel() : 0, st);
    });
    if (r != BRQ_OK) return status(r);
    PyObject* items[2] = {wrapped(a[5], dh.t), wrapped(Py_None, dw)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

// add_rms_norm_rotate_quantize(x, B, residual, weight, eps, y_dtype, h_out, want_h, codes, scales, layout, signs)
PyObject* add_rms_norm_rotate_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    Matrix x, res, h;
    at::Tensor w;
    double eps;
    int64_t B;
    at::ScalarType s;
    brq_dtype dt;
    brq_layout l;
    const int8_t* signs;
    uint8_t *codes, *scales;
    if (n != 12 || !g_residual || !quiet() || !matrix(c, a[0], &x) || !integer(a[1], &B) || !matrix(c, a[2], &res, true) || !same_sizes(x, res) ||
        !array_of(c, a[3], at::kFloat, {x.t.size(1)}, &w, true) || !number(a[4], &eps) || !dtype_arg(a[5], &s, &dt) || a[8] == Py_None || a[9] == Py_None ||
        !c.take(a[8]) || !c.take(a[9]) || (a[11] != Py_None && !c.take(a[11])) || !layout(a[10], &l) || !signs_arg(a[11], x.t.size(1), &signs) ||
        !buffers(a[8], a[9], x.t.size(0), x.t.size(1), l, &codes, &scales) || !sum_out(c, a[6], a[7], x, res, &h)) Py_RETURN_NONE;
    if (signs) signs = reinterpret_cast<const int8_t*>(data(a[11]));
    codes = const_cast<uint8_t*>(data(a[8]));
    scales = const_cast<uint8_t*>(data(a[9]));
    void* st = current_stream();
    const brq_status r = released([&] {
        return f_add_norm_quantize(x.p(), x.dt, x.ld, res.p(), res.dt, res.ld, x.t.size(0), x.t.size(1), address<float>(w), (float)eps, h.p(), h.ld, dt, B, signs, codes,
                                   scales, l, st);
    });
    if (r != BRQ_OK) return status(r);
    Py_INCREF(a[8]);
    Py_INCREF(a[9]);
    PyObject* items[3] = {a[8], a[9], wrapped(a[6], h.t)};
    return tuple_of(items);
    END_HANDLE_TH_ERRORS
}

PyObject *s_relu, *s_silu, *s_gelu;
bool activation(PyObject* o, brq_activation* v) {
    *v = BRQ_ACT_NONE;
    if (o == Py_None) return true;
    if (!PyUnicode_CheckExact(o)) return false;
    auto is = [&](PyObject* s) { return o == s || PyUnicode_Compare(o, s) == 0; };
    *v = is(s_relu) ? BRQ_ACT_RELU : is(s_silu) ? BRQ_ACT_SILU : is(s_gelu) ? BRQ_ACT_GELU : BRQ_ACT_NONE;
    return *v != BRQ_ACT_NONE;
}

// gemm_epilogue(aq, as, wq, ws, bias, activation, residual, out_dtype, out, a_layout, w_layout, M, N, K, workspace)
PyObject* gemm_epilogue(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c;
    brq_layout la, lw;
    int64_t M, N, K;
    at::Tensor bias, y, space;
    Matrix res;
    brq_activation act;
    brq_dtype dt;
    int64_t ldy;
    if (n != 15 || !g_residual || !quiet() || !c.take(a[0]) || !c.take(a[1]) || !c.take(a[2]) || !c.take(a[3]) || (a[8] != Py_None && !c.take(a[8])) || !layout(a[9], &la) ||
        !layout(a[10], &lw) || !size_arg(a[11], &M) || !size_arg(a[12], &N) || !size_arg(a[13], &K) || !operand(a[0], a[1], la, &M, &K) ||
        !operand(a[2], a[3], lw, &N, &K) || M < 0 || N < 0 || K < 0 || !operand_fits(a[0], a[1], la, M, K) || !operand_fits(a[2], a[3], lw, N, K) ||
        !array_of(c, a[4], at::kFloat, {N}, &bias, true) || !activation(a[5], &act) || !matrix(c, a[6], &res, true) ||
        (res.t.defined() && (res.t.size(0) != M || res.t.size(1) != N)) || !array_of(c, a[14], at::kByte, {-1}, &space, true) ||
        !result(a[8], a[7], THPVariable_Unpack(a[0]), M, N, &y, &dt, &ldy)) Py_RETURN_NONE;
    if (!space.defined() && (bias.defined() || act != BRQ_ACT_NONE || res.t.defined())) {
        int64_t need = 0;
        if (const brq_status r = f_gemm_epilogue_space(la, lw, M, N, K, &need); r != BRQ_OK) return status(r);
        if (need && !make(c, {need}, at::kByte, &space)) Py_RETURN_NONE;
    }
    const uint8_t *ac = data(a[0]), *as = data(a[1]), *wc = data(a[2]), *ws = data(a[3]);
    void *p = y.data_ptr(), *s = current_stream();
    return result_or(released([&] { return f_gemm_epilogue(ac, as, la, wc, ws, lw, M, N, K, address<float>(bias), act, res.p(), res.dt, res.ld, p, dt, ldy, address<void>(space), space.defined() ? space.numel() : 0, s); }), a[8], y);
    END_HANDLE_TH_ERRORS
}

PyObject* bind_residual(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "bind_residual takes the addresses of six entry points");
        return nullptr;
    }
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point's address is NULL");
            return nullptr;
        }
    }
    int i = 0;
    auto set = [&](auto& f) { f = reinterpret_cast<std::decay_t<decltype(f)>>(p[i++]); };
    set(f_add_norm), set(f_add_norm_back), set(f_add_norm_back_space), set(f_add_norm_quantize), set(f_gemm_epilogue), set(f_gemm_epilogue_space);
    g_residual = true;
    Py_RETURN_NONE;
}

#define BRQ_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BRQ_METHOD(bind), BRQ_METHOD(rotate_quantize), BRQ_METHOD(swiglu_rotate_quantize), BRQ_METHOD(matrix_rotate_quantize),
                         BRQ_METHOD(gemm), BRQ_METHOD(rotate_quantize_gemm), BRQ_METHOD(bind_stats), BRQ_METHOD(block_stats), BRQ_METHOD(block_stats_summary),
                         BRQ_METHOD(bind_attention), BRQ_METHOD(qk_norm_rope), BRQ_METHOD(qk_norm_rope_backward), BRQ_METHOD(kv4_append), BRQ_METHOD(kv4_read), BRQ_METHOD(kv4_attention),
                         BRQ_METHOD(kv4_pages_copy), BRQ_METHOD(kv4_pages_fork), BRQ_METHOD(kv4_pages_free), BRQ_METHOD(kv4_pages_reserve), BRQ_METHOD(kv4_pages_compact),
                         BRQ_METHOD(bind_residual), BRQ_METHOD(add_rms_norm), BRQ_METHOD(add_rms_norm_backward), BRQ_METHOD(add_rms_norm_rotate_quantize), BRQ_METHOD(gemm_epilogue), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
    s_rowmajor = PyUnicode_InternFromString("rowmajor");
    s_tiled = PyUnicode_InternFromString("tiled");
    s_relu = PyUnicode_InternFromString("relu");
    s_silu = PyUnicode_InternFromString("silu");
    s_gelu = PyUnicode_InternFromString("gelu");
    if (!s_rowmajor || !s_tiled || !s_relu || !s_silu || !s_gelu) return nullptr;
    PyObject* m = PyModule_Create(&module);
    // The torch whose headers this was built with: tensors are read through them, so no other will do.
    if (m && PyModule_AddStringConstant(m, "TORCH", BRQ_TORCH) != 0) Py_CLEAR(m);
    return m;
}
