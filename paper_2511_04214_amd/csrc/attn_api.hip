// extern "C" boundary of the attention side (include/brq_attn.h): argument validation on the host, then launches on the
// caller's stream.
#include <cmath>
#include <limits>

#include "../../include/brq_attn.h"
#include "brq_attn.h"
#include "brq_launch.h"

namespace {

constexpr int64_t kMax = int64_t(1) << 31;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int size_of(brq_dtype d) { return d == BRQ_F32 ? 4 : d == BRQ_BF16 ? 2 : 0; }
brq_status launched(hipError_t e) { return e == hipSuccess ? BRQ_OK : BRQ_ERR_LAUNCH; }

// A set of heads; outputs must not overlap themselves.  `need`: the number of heads, or -1 for any.
brq_status check_heads(const brq_heads* x, int es, int64_t T, int64_t D, int64_t need, bool out) {
    if (!x) return BRQ_ERR_NULL;
    if (es == 0) return BRQ_ERR_DTYPE;
    if (x->heads < 1 || x->heads >= kMax || (need >= 0 && x->heads != need)) return BRQ_ERR_SHAPE;
    if (T >= kMax || T * x->heads >= kMax / 64) return BRQ_ERR_SHAPE;
    if (x->token_stride < 0 || x->head_stride < 0 || x->token_stride >= kMax * 16 || x->head_stride >= kMax * 16) return BRQ_ERR_SHAPE;
    if (out && T > 0) {
        const int64_t ts = T > 1 ? x->token_stride : 0, hs = x->heads > 1 ? x->head_stride : 0;
        const bool rows = (x->heads == 1 || hs >= D) && (T == 1 || ts >= (x->heads - 1) * hs + D);
        const bool columns = (T == 1 || ts >= D) && (x->heads == 1 || hs >= (T - 1) * ts + D);
        if (!rows && !columns) return BRQ_ERR_SHAPE;
    }
    if (T > 0 && !x->data) return BRQ_ERR_NULL;
    if (!aligned(x->data, 16) || (T > 1 && (x->token_stride * es) % 16 != 0) || (x->heads > 1 && (x->head_stride * es) % 16 != 0)) return BRQ_ERR_ALIGN;
    return BRQ_OK;
}

brq_status check_rope(const brq_rope* r, int64_t T, int64_t D) {
    if (!r) return BRQ_OK;
    if (r->rot <= 0 || r->rot > D || r->rot % 16 != 0 || r->rows < 1 || r->rows >= kMax) return BRQ_ERR_SHAPE;
    if (T > 0 && (!r->cos || !r->sin || !r->positions)) return BRQ_ERR_NULL;
    if (!aligned(r->cos, 16) || !aligned(r->sin, 16) || !aligned(r->positions, 8)) return BRQ_ERR_ALIGN;
    return BRQ_OK;
}

// log2 of a rotation block inside a head, 0 for none, -1 if it is none
int block_of(int64_t B, int64_t D) {
    if (B == 1) return 0;
    if (B < 8 || B > D || (B & (B - 1)) != 0) return -1;
    int l = 0;
    while ((int64_t(1) << l) < B) ++l;
    return l;
}

brq::Heads view(const brq_heads* x, int es) {
    if (!x) return brq::Heads{nullptr, 0, 0, 0};
    return brq::Heads{static_cast<uint8_t*>(x->data), x->token_stride * es, x->head_stride * es, (int)x->heads};
}

brq::Rope view(const brq_rope* r) {
    if (!r) return brq::Rope{nullptr, nullptr, nullptr, 0, 0, 0};
    return brq::Rope{r->cos, r->sin, r->positions, r->rows, (int)r->rot, r->interleaved != 0};
}

#define BRQ_CHECK(expr) do { if (const brq_status st_ = (expr); st_ != BRQ_OK) return st_; } while (0)

// What the passes over heads share.
brq_status check_common(const brq_heads* q, const brq_heads* k, brq_dtype xdt, int64_t T, int64_t D, const float* wq,
                        const float* wk, float eps, const brq_rope* rope) {
    if (size_of(xdt) == 0) return BRQ_ERR_DTYPE;
    if (T < 0 || !(eps >= 0.0f)) return BRQ_ERR_SHAPE;
    if (q) BRQ_CHECK(check_heads(q, size_of(xdt), T, D, -1, false));
    if (k) BRQ_CHECK(check_heads(k, size_of(xdt), T, D, -1, false));
    BRQ_CHECK(check_rope(rope, T, D));
    if (!aligned(wq, 4) || !aligned(wk, 4)) return BRQ_ERR_ALIGN;
    return BRQ_OK;
}

brq_status check_cache(const uint8_t* pool, int64_t num_pages, int64_t Hk, int64_t D) {
    if (D != 64 && D != 128) return BRQ_ERR_SHAPE;
    if (num_pages < 0 || num_pages >= kMax || Hk < 1 || Hk >= 65536) return BRQ_ERR_SHAPE;
    if (num_pages > 0 && !pool) return BRQ_ERR_NULL;
    return aligned(pool, 16) ? BRQ_OK : BRQ_ERR_ALIGN;
}

brq_status check_attention_sizes(int64_t T, int64_t S, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q, int64_t max_kv) {
    if (D != 64 && D != 128) return BRQ_ERR_SHAPE;
    if (T < 0 || S < 0 || S >= kMax || Hk < 1 || Hk >= 65536 || Hq < 1 || Hq % Hk != 0 || Hq >= 65536 || T >= kMax || T * Hq >= kMax / 64) return BRQ_ERR_SHAPE;
    if (max_q < 1 || max_q >= kMax / 64 || max_kv < 0 || max_kv >= kMax - 64) return BRQ_ERR_SHAPE;
    // a workgroup of up to 512 threads to each, and to every 128 rows besides, in one grid; max_q, a bound alone, adds none
    if (S * Hk >= kMax / 512) return BRQ_ERR_SHAPE;
    return BRQ_OK;
}

brq_status check_pages(int64_t num_pages, int64_t S, int64_t cols, int64_t n) {
    if (num_pages < 0 || num_pages >= kMax / 4 || S < 0 || cols < 0 || cols >= kMax / 64 || S >= kMax || S * cols >= kMax || n < 0 || n >= kMax / 1024) return BRQ_ERR_SHAPE;
    return BRQ_OK;
}
brq_status check_pool(const uint8_t* pool, int64_t page_bytes, int64_t num_pages) {
    if (page_bytes <= 0 || page_bytes % 16 != 0 || page_bytes >= kMax) return BRQ_ERR_SHAPE;
    if (num_pages > 0 && !pool) return BRQ_ERR_NULL;
    return aligned(pool, 16) ? BRQ_OK : BRQ_ERR_ALIGN;
}
template <class... P>
brq_status check_ints(P... p) {
    if ((... || !p)) return BRQ_ERR_NULL;
    return (... && aligned(p, 4)) ? BRQ_OK : BRQ_ERR_ALIGN;
}

}  // namespace

extern "C" {

brq_status brq_qk_norm_rope(const brq_heads* q, const brq_heads* k, brq_dtype xdt, int64_t T, int64_t D, const float* wq,
                            const float* wk, float eps, const brq_rope* rope, int64_t B, const brq_heads* q_out,
                            const brq_heads* k_out, brq_dtype ydt, void* stream) {
    if (!q || (k == nullptr) != (k_out == nullptr)) return BRQ_ERR_NULL;
    if (D != 64 && D != 128 && D != 256) return BRQ_ERR_SHAPE;
    BRQ_CHECK(check_common(q, k, xdt, T, D, wq, wk, eps, rope));
    BRQ_CHECK(check_heads(q_out, size_of(ydt), T, D, q->heads, true));
    if (k) BRQ_CHECK(check_heads(k_out, size_of(ydt), T, D, k->heads, true));
    const int l2b = block_of(B, D);
    if (l2b < 0) return BRQ_ERR_BLOCK;
    if (T == 0) return BRQ_OK;
    brq::HeadsArgs a{};
    a.q = view(q, size_of(xdt));
    a.k = view(k, size_of(xdt));
    a.qo = view(q_out, size_of(ydt));
    a.ko = view(k_out, size_of(ydt));
    a.wq = wq;
    a.wk = wk;
    a.eps = eps;
    a.rope = view(rope);
    a.T = T;
    a.l2b = l2b;
    return launched(brq::launch_heads((int)D, xdt == BRQ_BF16, ydt == BRQ_BF16, false, a, static_cast<hipStream_t>(stream)));
}

brq_status brq_qk_norm_rope_backward_workspace(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t* bytes) {
    if (!bytes) return BRQ_ERR_NULL;
    if ((D != 64 && D != 128 && D != 256) || T < 0 || T >= kMax || Hq < 1 || Hk < 0 || Hq >= kMax || Hk >= kMax || T * Hq >= kMax / 64 || T * Hk >= kMax / 64) return BRQ_ERR_SHAPE;
    *bytes = T == 0 ? 0 : brq::heads_backward_workgroups(T, (int)Hq, (int)Hk, (int)D) * 2 * D * 4;
    return BRQ_OK;
}

brq_status brq_qk_norm_rope_backward(const brq_heads* q, const brq_heads* k, brq_dtype xdt, int64_t T, int64_t D, const float* wq,
                                     const float* wk, float eps, const brq_rope* rope, int64_t B, const brq_heads* gq,
                                     const brq_heads* gk, brq_dtype gdt, const brq_heads* dq, const brq_heads* dk, float* dwq,
                                     float* dwk, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!q || (k == nullptr) != (gk == nullptr) || (k == nullptr) != (dk == nullptr)) return BRQ_ERR_NULL;
    if ((dwq && !wq) || (dwk && (!wk || !k))) return BRQ_ERR_NULL;
    if (D != 64 && D != 128 && D != 256) return BRQ_ERR_SHAPE;
    BRQ_CHECK(check_common(q, k, xdt, T, D, wq, wk, eps, rope));
    BRQ_CHECK(check_heads(gq, size_of(gdt), T, D, q->heads, false));
    BRQ_CHECK(check_heads(dq, size_of(xdt), T, D, q->heads, true));
    if (k) {
        BRQ_CHECK(check_heads(gk, size_of(gdt), T, D, k->heads, false));
        BRQ_CHECK(check_heads(dk, size_of(xdt), T, D, k->heads, true));
    }
    const int l2b = block_of(B, D);
    if (l2b < 0) return BRQ_ERR_BLOCK;
    if (!aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    const bool sums = dwq || dwk;
    if (T == 0)                                     // (sums over nothing)
        return sums ? launched(brq::launch_heads_weight_grads(nullptr, 0, (int)D, dwq, dwk, static_cast<hipStream_t>(stream))) : BRQ_OK;
    int64_t need = 0;
    BRQ_CHECK(brq_qk_norm_rope_backward_workspace(T, q->heads, k ? k->heads : 0, D, &need));
    if (sums && !workspace) return BRQ_ERR_NULL;
    if (sums && workspace_bytes < need) return BRQ_ERR_SHAPE;
    brq::HeadsArgs a{};
    a.q = view(q, size_of(xdt));
    a.k = view(k, size_of(xdt));
    a.gq = view(gq, size_of(gdt));
    a.gk = view(gk, size_of(gdt));
    a.qo = view(dq, size_of(xdt));
    a.ko = view(dk, size_of(xdt));
    a.wq = wq;
    a.wk = wk;
    a.eps = eps;
    a.rope = view(rope);
    a.T = T;
    a.l2b = l2b;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    a.dwq = dwq;
    a.dwk = dwk;
    return launched(brq::launch_heads_backward((int)D, xdt == BRQ_BF16, gdt == BRQ_BF16, a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_page_bytes(int64_t Hk, int64_t D, int64_t* bytes) {
    if (!bytes) return BRQ_ERR_NULL;
    if ((D != 64 && D != 128) || Hk < 1 || Hk >= 65536) return BRQ_ERR_SHAPE;
    *bytes = Hk * brq::kv4_head_bytes((int)D);
    return BRQ_OK;
}

brq_status brq_kv4_append(const brq_heads* q, const brq_heads* k, const brq_heads* v, brq_dtype xdt, int64_t T, int64_t D,
                          const float* wq, const float* wk, float eps, const brq_rope* rope, int64_t B, int64_t Bv,
                          const int64_t* slots, uint8_t* pool, int64_t num_pages, const brq_heads* q_out, void* stream) {
    if (!k || !v || (q == nullptr) != (q_out == nullptr)) return BRQ_ERR_NULL;
    if (D != 64 && D != 128) return BRQ_ERR_SHAPE;
    BRQ_CHECK(check_common(q, k, xdt, T, D, wq, wk, eps, rope));
    BRQ_CHECK(check_heads(v, size_of(xdt), T, D, k->heads, false));
    if (q) BRQ_CHECK(check_heads(q_out, size_of(xdt), T, D, q->heads, true));
    BRQ_CHECK(check_cache(pool, num_pages, k->heads, D));
    const int l2b = block_of(B, D), l2bv = block_of(Bv, D);
    if (l2b < 0 || l2bv < 0) return BRQ_ERR_BLOCK;
    if (T == 0) return BRQ_OK;
    if (!slots) return BRQ_ERR_NULL;
    if (!aligned(slots, 8)) return BRQ_ERR_ALIGN;
    brq::HeadsArgs a{};
    a.q = view(q, size_of(xdt));
    a.k = view(k, size_of(xdt));
    a.v = view(v, size_of(xdt));
    a.qo = view(q_out, size_of(xdt));
    a.wq = wq;
    a.wk = wk;
    a.eps = eps;
    a.rope = view(rope);
    a.T = T;
    a.l2b = l2b;
    a.l2bv = l2bv;
    a.slots = slots;
    a.pool = pool;
    a.num_slots = num_pages * BRQ_KV4_PAGE;
    a.Hk = (int)k->heads;
    return launched(brq::launch_heads((int)D, xdt == BRQ_BF16, xdt == BRQ_BF16, true, a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_read(const uint8_t* pool, int64_t num_pages, int64_t T, int64_t D, const int64_t* slots, const brq_heads* k_out,
                        const brq_heads* v_out, brq_dtype ydt, void* stream) {
    if (T < 0 || (D != 64 && D != 128)) return BRQ_ERR_SHAPE;
    BRQ_CHECK(check_heads(k_out, size_of(ydt), T, D, -1, true));
    BRQ_CHECK(check_heads(v_out, size_of(ydt), T, D, k_out->heads, true));
    BRQ_CHECK(check_cache(pool, num_pages, k_out->heads, D));
    if (T == 0) return BRQ_OK;
    if (!slots) return BRQ_ERR_NULL;
    if (!aligned(slots, 8)) return BRQ_ERR_ALIGN;
    return launched(brq::launch_kv4_read((int)D, pool, num_pages * BRQ_KV4_PAGE, (int)k_out->heads, T, slots, view(k_out, size_of(ydt)),
                                         view(v_out, size_of(ydt)), ydt == BRQ_BF16, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_attention_workspace(int64_t T, int64_t S, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q, int64_t max_kv,
                                       int64_t* bytes) {
    if (!bytes) return BRQ_ERR_NULL;
    BRQ_CHECK(check_attention_sizes(T, S, Hq, Hk, D, max_q, max_kv));
    *bytes = 0;
    if (T == 0 || S == 0) return BRQ_OK;
    int cus = 0;
    if (brq::device_cus(&cus) != hipSuccess) return BRQ_ERR_DEVICE;
    *bytes = brq::kv4_attention_workspace(T, S, (int)Hq, (int)Hk, (int)D, max_q, max_kv, cus);
    return BRQ_OK;
}

brq_status brq_kv4_attention(const brq_heads* q, int64_t T, int64_t D, const uint8_t* pool, int64_t num_pages, int64_t Hk,
                             const int32_t* table, int64_t table_cols, const int32_t* kv_lens, const int32_t* cu_q, int64_t S,
                             float scale, int causal, int64_t window, int64_t max_q, int64_t max_kv, const brq_heads* out,
                             float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!q || !out) return BRQ_ERR_NULL;
    if (T < 0 || !(std::fabs(scale) <= std::numeric_limits<float>::max())) return BRQ_ERR_SHAPE;
    BRQ_CHECK(check_attention_sizes(T, S, q->heads, Hk, D, max_q, max_kv));
    BRQ_CHECK(check_heads(q, 2, T, D, -1, false));
    BRQ_CHECK(check_heads(out, 2, T, D, q->heads, true));
    BRQ_CHECK(check_cache(pool, num_pages, Hk, D));
    if (table_cols < 0 || table_cols >= kMax / 64 || window < 0 || window >= kMax || (window > 0 && !causal) || (!cu_q && T != S)) return BRQ_ERR_SHAPE;
    if (!aligned(lse, 4) || !aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    if (T == 0 || S == 0) return BRQ_OK;
    BRQ_CHECK(check_ints(kv_lens));
    if ((table_cols > 0 && !table)) return BRQ_ERR_NULL;
    if (!aligned(table, 4) || !aligned(cu_q, 4)) return BRQ_ERR_ALIGN;
    int64_t need = 0;
    BRQ_CHECK(brq_kv4_attention_workspace(T, S, q->heads, Hk, D, max_q, max_kv, &need));
    if (need > 0 && !workspace) return BRQ_ERR_NULL;
    if (workspace_bytes < need) return BRQ_ERR_SHAPE;
    brq::AttnArgs a{};
    a.q = view(q, 2);
    a.o = view(out, 2);
    a.T = T;
    a.pool = pool;
    a.num_pages = num_pages;
    a.Hk = (int)Hk;
    a.G = (int)(q->heads / Hk);
    a.table = table;
    a.kv_lens = kv_lens;
    a.cu_q = cu_q;
    a.table_cols = (int)table_cols;
    a.S = (int)S;
    a.scale = scale;
    a.causal = causal != 0;
    a.window = (int)window;
    a.max_q = (int)max_q;
    a.max_kv = (int)max_kv;
    a.lse = lse;
    a.workspace = workspace;
    return launched(brq::launch_kv4_attention((int)D, a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_pages_workspace(int64_t n, int64_t num_pages, int64_t* bytes) {
    if (!bytes) return BRQ_ERR_NULL;
    BRQ_CHECK(check_pages(num_pages, 0, 0, n));
    *bytes = (8 + n + 2 * num_pages) * 4;
    return BRQ_OK;
}

brq_status brq_kv4_pages_copy(uint8_t* pool, int64_t page_bytes, int64_t num_pages, const int32_t* src, const int32_t* dst, int64_t n,
                              void* stream) {
    BRQ_CHECK(check_pages(num_pages, 0, 0, n));
    BRQ_CHECK(check_pool(pool, page_bytes, num_pages));
    if (n == 0 || num_pages == 0) return BRQ_OK;
    if (n * ((page_bytes + 16383) / 16384) >= kMax) return BRQ_ERR_SHAPE;
    BRQ_CHECK(check_ints(src, dst));
    brq::PagesArgs a{};
    a.pool = pool;
    a.page_bytes = page_bytes;
    a.num_pages = (int)num_pages;
    a.a = src;
    a.b = dst;
    a.n = (int)n;
    return launched(brq::launch_pages_copy(a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_pages_fork(uint8_t* pool, int64_t page_bytes, int64_t num_pages, int32_t* table, int64_t S, int64_t table_cols,
                              int32_t* lens, int32_t* refs, const int32_t* parent, const int32_t* child, int64_t n, int32_t* failed,
                              void* workspace, void* stream) {
    BRQ_CHECK(check_pages(num_pages, S, table_cols, n));
    BRQ_CHECK(check_pool(pool, page_bytes, num_pages));
    BRQ_CHECK(check_ints(failed));
    if (n * ((page_bytes + 16383) / 16384) >= kMax) return BRQ_ERR_SHAPE;
    if (n > 0 && S > 0) BRQ_CHECK(check_ints(table_cols ? table : lens, lens, num_pages ? refs : lens, parent, child));
    if (!workspace) return BRQ_ERR_NULL;
    if (!aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    brq::PagesArgs a{};
    a.pool = pool;
    a.page_bytes = page_bytes;
    a.num_pages = (int)num_pages;
    a.table = table;
    a.S = (int)S;
    a.cols = (int)table_cols;
    a.lens = lens;
    a.refs = refs;
    a.a = parent;
    a.b = child;
    a.n = S > 0 ? (int)n : 0;
    a.result = failed;
    a.workspace = static_cast<int32_t*>(workspace);
    return launched(brq::launch_pages_fork(a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_pages_free(int32_t* table, int64_t S, int64_t table_cols, int32_t* lens, int32_t* refs, int64_t num_pages,
                              const int32_t* seq, int64_t n, void* stream) {
    BRQ_CHECK(check_pages(num_pages, S, table_cols, n));
    if (n == 0 || S == 0) return BRQ_OK;
    BRQ_CHECK(check_ints(table_cols ? table : lens, lens, num_pages ? refs : lens, seq));
    brq::PagesArgs a{};
    a.num_pages = (int)num_pages;
    a.table = table;
    a.S = (int)S;
    a.cols = (int)table_cols;
    a.lens = lens;
    a.refs = refs;
    a.a = seq;
    a.n = (int)n;
    return launched(brq::launch_pages_free(a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_pages_reserve(int32_t* table, int64_t S, int64_t table_cols, int32_t* refs, int64_t num_pages,
                                 const int32_t* seq, const int32_t* tokens, int64_t n, int32_t* failed, void* workspace, void* stream) {
    BRQ_CHECK(check_pages(num_pages, S, table_cols, n));
    BRQ_CHECK(check_ints(failed));
    if (n > 0 && S > 0) BRQ_CHECK(check_ints(table_cols ? table : failed, num_pages ? refs : failed, seq, tokens));
    if (!workspace) return BRQ_ERR_NULL;
    if (!aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    brq::PagesArgs a{};
    a.num_pages = (int)num_pages;
    a.table = table;
    a.S = (int)S;
    a.cols = (int)table_cols;
    a.refs = refs;
    a.a = seq;
    a.b = tokens;
    a.n = S > 0 ? (int)n : 0;
    a.result = failed;
    a.workspace = static_cast<int32_t*>(workspace);
    return launched(brq::launch_pages_reserve(a, static_cast<hipStream_t>(stream)));
}

brq_status brq_kv4_pages_compact(uint8_t* pool, int64_t page_bytes, int64_t num_pages, int32_t* table, int64_t S, int64_t table_cols,
                                 int32_t* refs, int32_t* live, void* workspace, void* stream) {
    BRQ_CHECK(check_pages(num_pages, S, table_cols, 0));
    BRQ_CHECK(check_pool(pool, page_bytes, num_pages));
    BRQ_CHECK(check_ints(live, num_pages ? refs : live, S * table_cols ? table : live));
    if (!workspace) return BRQ_ERR_NULL;
    if (!aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    brq::PagesArgs a{};
    a.pool = pool;
    a.page_bytes = page_bytes;
    a.num_pages = (int)num_pages;
    a.table = table;
    a.S = (int)S;
    a.cols = (int)table_cols;
    a.refs = refs;
    a.result = live;
    a.workspace = static_cast<int32_t*>(workspace);
    return launched(brq::launch_pages_compact(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
