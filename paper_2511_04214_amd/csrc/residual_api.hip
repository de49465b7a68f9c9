// extern "C" boundary of the residual side (include/brq_residual.h): argument validation on the host, then launches on the
// caller's stream.
#include "../../include/brq_diag.h"
#include "../../include/brq_residual.h"
#include "brq_launch.h"
#include "brq_residual.h"

namespace {

constexpr int64_t kMax = int64_t(1) << 31;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int size_of(brq_dtype d) { return d == BRQ_F32 ? 4 : d == BRQ_BF16 ? 2 : 0; }
brq_status launched(hipError_t e) { return e == hipSuccess ? BRQ_OK : BRQ_ERR_LAUNCH; }

#define BRQ_CHECK(expr) do { if (const brq_status st_ = (expr); st_ != BRQ_OK) return st_; } while (0)

brq_status check_sizes(int64_t M, int64_t K) {
    if (M < 0 || K <= 0 || K % 32 != 0 || K > brq::NORM_MAX_K) return BRQ_ERR_SHAPE;
    return M >= kMax || M * (K / 8) >= kMax ? BRQ_ERR_SHAPE : BRQ_OK;
}

// A matrix of M rows of K.  A pitch is below 2^30 elements: no product of it in bytes and a row's number overflows.
brq_status check_rows(const void* x, brq_dtype dt, int64_t M, int64_t K, int64_t ld) {
    const int es = size_of(dt);
    if (es == 0) return BRQ_ERR_DTYPE;
    if (ld < K || ld >= kMax / 2) return BRQ_ERR_SHAPE;
    if (M > 0 && !x) return BRQ_ERR_NULL;
    return aligned(x, 16) && ld * es % 16 == 0 ? BRQ_OK : BRQ_ERR_ALIGN;
}

// An output at an input's address has to be that input's rows.
brq_status check_place(const void* out, brq_dtype odt, int64_t ldo, const void* in, brq_dtype idt, int64_t ldi, int64_t M) {
    return out && out == in && (odt != idt || (M > 1 && ldo != ldi)) ? BRQ_ERR_SHAPE : BRQ_OK;
}

brq_status check_weight(const float* w, float eps) {
    if (!(eps >= 0.0f)) return BRQ_ERR_SHAPE;
    return aligned(w, 16) ? BRQ_OK : BRQ_ERR_ALIGN;
}

brq::RowSet rows(const void* p, brq_dtype dt, int64_t ld) { return {static_cast<uint8_t*>(const_cast<void*>(p)), ld * size_of(dt), dt == BRQ_BF16}; }

// What both forms of the norm share: inputs and the sum.
brq_status check_norm(const void* x, brq_dtype xdt, int64_t ldx, const void* res, brq_dtype rdt, int64_t ldr, int64_t M, int64_t K,
                      const float* w, float eps, const void* h, int64_t ldh) {
    BRQ_CHECK(check_sizes(M, K));
    BRQ_CHECK(check_rows(x, xdt, M, K, ldx));
    if (res) BRQ_CHECK(check_rows(res, rdt, M, K, ldr));
    if (h) {
        if (!res && M > 0) return BRQ_ERR_NULL;
        BRQ_CHECK(check_rows(h, rdt, M, K, ldh));
        BRQ_CHECK(check_place(h, rdt, ldh, res, rdt, ldr, M));
        BRQ_CHECK(check_place(h, rdt, ldh, x, xdt, ldx, M));
    }
    return check_weight(w, eps);
}

brq::NormArgs norm_args(const void* x, brq_dtype xdt, int64_t ldx, const void* res, brq_dtype rdt, int64_t ldr, int64_t M, int64_t K,
                        const float* w, float eps, void* h, int64_t ldh) {
    brq::NormArgs a{};
    a.x = rows(x, xdt, ldx);
    if (res) a.res = rows(res, rdt, ldr);
    if (h) a.h = rows(h, rdt, ldh);
    a.w = w;
    a.eps = eps;
    a.M = M;
    a.K = K;
    return a;
}

brq_status check_epilogue(int64_t M, int64_t N, const float* bias, brq_activation act, const void* residual, brq_dtype rdt, int64_t ldr,
                          const void* y, brq_dtype ydt, int64_t ldy) {
    if (act < BRQ_ACT_NONE || act > BRQ_ACT_GELU) return BRQ_ERR_ACTIVATION;
    if (!aligned(bias, 4)) return BRQ_ERR_ALIGN;
    if (!residual) return BRQ_OK;
    if (size_of(rdt) == 0) return BRQ_ERR_DTYPE;
    if (ldr < N || ldr >= kMax / 2) return BRQ_ERR_SHAPE;
    if (!aligned(residual, (uintptr_t)size_of(rdt))) return BRQ_ERR_ALIGN;
    return check_place(y, ydt, ldy, residual, rdt, ldr, M);
}
brq::Epilogue epilogue(const float* bias, brq_activation act, const void* residual, brq_dtype rdt, int64_t ldr, brq_dtype ydt) {
    return {bias, static_cast<const uint8_t*>(residual), residual ? ldr * size_of(rdt) : 0, rdt == BRQ_BF16, (int)act, ydt == BRQ_BF16};
}

}  // namespace

extern "C" {

brq_status brq_add_rms_norm(const void* x, brq_dtype xdt, int64_t ldx, const void* res, brq_dtype rdt, int64_t ldr, int64_t M,
                            int64_t K, const float* w, float eps, void* h, int64_t ldh, void* y, brq_dtype ydt, int64_t ldy,
                            void* stream) {
    BRQ_CHECK(check_norm(x, xdt, ldx, res, rdt, ldr, M, K, w, eps, h, ldh));
    BRQ_CHECK(check_rows(y, ydt, M, K, ldy));
    BRQ_CHECK(check_place(y, ydt, ldy, x, xdt, ldx, M));
    if (res) BRQ_CHECK(check_place(y, ydt, ldy, res, rdt, ldr, M));
    if (h && h == y && M > 0) return BRQ_ERR_SHAPE;
    if (M == 0) return BRQ_OK;
    brq::NormArgs a = norm_args(x, xdt, ldx, res, rdt, ldr, M, K, w, eps, h, ldh);
    a.y = rows(y, ydt, ldy);
    return launched(brq::launch_add_rms_norm(a, false, static_cast<hipStream_t>(stream)));
}

brq_status brq_add_rms_norm_rotate_quantize_fused(const void* x, brq_dtype xdt, int64_t ldx, const void* res, brq_dtype rdt,
                                                  int64_t ldr, int64_t M, int64_t K, const float* w, float eps, void* h,
                                                  int64_t ldh, brq_dtype ydt, int64_t B, const int8_t* signs, uint8_t* codes,
                                                  uint8_t* scales, brq_layout layout, void* stream) {
    BRQ_CHECK(check_norm(x, xdt, ldx, res, rdt, ldr, M, K, w, eps, h, ldh));
    if (size_of(ydt) == 0) return BRQ_ERR_DTYPE;
    if (layout != BRQ_LAYOUT_ROWMAJOR && layout != BRQ_LAYOUT_TILED) return BRQ_ERR_LAYOUT;
    int l2b = 0;
    if (B != 1) {
        if (B < 8 || B > 512 || (B & (B - 1)) != 0 || K % B != 0) return BRQ_ERR_BLOCK;
        while ((int64_t(1) << l2b) < B) ++l2b;
    } else if (signs) {
        return BRQ_ERR_BLOCK;
    }
    if (M > 0 && (!codes || !scales)) return BRQ_ERR_NULL;
    if (!aligned(signs, 16) || !aligned(codes, 16) || !aligned(scales, 16)) return BRQ_ERR_ALIGN;
    if (M == 0) return BRQ_OK;
    brq::NormArgs a = norm_args(x, xdt, ldx, res, rdt, ldr, M, K, w, eps, h, ldh);
    a.y.bf16 = ydt == BRQ_BF16;
    a.codes = codes;
    a.scales = scales;
    a.tiled = layout == BRQ_LAYOUT_TILED;
    a.l2b = l2b;
    a.signs = signs;
    return launched(brq::launch_add_rms_norm(a, true, static_cast<hipStream_t>(stream)));
}

brq_status brq_add_rms_norm_backward_workspace(int64_t M, int64_t K, int64_t* bytes) {
    if (!bytes) return BRQ_ERR_NULL;
    BRQ_CHECK(check_sizes(M, K));
    *bytes = brq::norm_backward_parts(M, K) * K * 4;
    return BRQ_OK;
}

brq_status brq_add_rms_norm_backward(const void* h, brq_dtype hdt, int64_t ldh, const void* gy, brq_dtype gdt, int64_t ldgy,
                                     const void* gh, int64_t ldgh, int64_t M, int64_t K, const float* w, float eps, void* dh,
                                     int64_t lddh, float* dw, void* workspace, int64_t workspace_bytes, void* stream) {
    BRQ_CHECK(check_sizes(M, K));
    BRQ_CHECK(check_rows(h, hdt, M, K, ldh));
    BRQ_CHECK(check_rows(gy, gdt, M, K, ldgy));
    if (gh) BRQ_CHECK(check_rows(gh, hdt, M, K, ldgh));
    BRQ_CHECK(check_rows(dh, hdt, M, K, lddh));
    if (gh) BRQ_CHECK(check_place(dh, hdt, lddh, gh, hdt, ldgh, M));
    BRQ_CHECK(check_place(dh, hdt, lddh, h, hdt, ldh, M));
    BRQ_CHECK(check_place(dh, hdt, lddh, gy, gdt, ldgy, M));
    BRQ_CHECK(check_weight(w, eps));
    if (dw && !w) return BRQ_ERR_NULL;
    if (!aligned(dw, 4) || !aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    const int64_t need = dw ? brq::norm_backward_parts(M, K) * K * 4 : 0;
    if (need > 0 && !workspace) return BRQ_ERR_NULL;
    if (need > workspace_bytes) return BRQ_ERR_SHAPE;
    if (M == 0 && !dw) return BRQ_OK;
    brq::NormBackwardArgs a{};
    a.h = rows(h, hdt, ldh);
    a.gy = rows(gy, gdt, ldgy);
    if (gh) a.gh = rows(gh, hdt, ldgh);
    a.dh = rows(dh, hdt, lddh);
    a.w = w;
    a.eps = eps;
    a.M = M;
    a.K = K;
    a.partial = dw ? static_cast<float*>(workspace) : nullptr;
    a.dw = dw;
    return launched(brq::launch_add_rms_norm_backward(a, static_cast<hipStream_t>(stream)));
}

brq_status brq_mxfp4_gemm_epilogue_workspace(brq_layout a_layout, brq_layout w_layout, int64_t M, int64_t N, int64_t K, int64_t* bytes) {
    alignas(16) static const uint8_t operand[16] = {};      // (nothing is launched: any aligned address will do)
    if (!bytes) return BRQ_ERR_NULL;
    BRQ_CHECK(brq::check_gemm(operand, operand, a_layout, operand, operand, w_layout, M, N, K, operand, BRQ_F32, N));
    *bytes = 0;
    if (M == 0 || N == 0) return BRQ_OK;
    int cus = 0;
    if (brq::device_cus(&cus) != hipSuccess) return BRQ_ERR_DEVICE;
    const brq::GemmShape g{M, N, K, a_layout == BRQ_LAYOUT_TILED, w_layout == BRQ_LAYOUT_TILED, true, N, 0, true};
    *bytes = brq::split_gemm_workspace(g, brq::gemm_split(g, cus));
    return BRQ_OK;
}

brq_status brq_mxfp4_gemm_epilogue(const uint8_t* aq, const uint8_t* as, brq_layout a_layout, const uint8_t* wq, const uint8_t* ws,
                                   brq_layout w_layout, int64_t M, int64_t N, int64_t K, const float* bias, brq_activation act,
                                   const void* residual, brq_dtype rdt, int64_t ldr, void* y, brq_dtype ydt, int64_t ldy, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
    BRQ_CHECK(brq::check_gemm(aq, as, a_layout, wq, ws, w_layout, M, N, K, y, ydt, ldy));
    BRQ_CHECK(check_epilogue(M, N, bias, act, residual, rdt, ldr, y, ydt, ldy));
    if (!aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    if (M == 0 || N == 0) return BRQ_OK;
    const brq::Operand a{aq, as, a_layout == BRQ_LAYOUT_TILED}, w{wq, ws, w_layout == BRQ_LAYOUT_TILED};
    brq::GemmShape g{M, N, K, a.tiled, w.tiled, ydt == BRQ_BF16, ldy, reinterpret_cast<uintptr_t>(y)};
    if (!bias && act == BRQ_ACT_NONE && !residual) return launched(brq::launch_mxfp4_gemm(a, w, g, y, static_cast<hipStream_t>(stream)));
    g.epilogue = true;
    g.exponential = act == BRQ_ACT_SILU || act == BRQ_ACT_GELU;
    g.residual = residual != nullptr;
    int cus = 0;
    if (brq::device_cus(&cus) != hipSuccess) return BRQ_ERR_LAUNCH;
    const int64_t need = brq::split_gemm_workspace(g, brq::gemm_split(g, cus));
    if (need > 0 && !workspace) return BRQ_ERR_NULL;
    if (need > workspace_bytes) return BRQ_ERR_SHAPE;
    const brq::Epilogue e = epilogue(bias, act, residual, rdt, ldr, ydt);
    return launched(brq::launch_mxfp4_gemm(a, w, g, y, static_cast<hipStream_t>(stream), &e, workspace));
}

brq_status brq_diag_mxfp4_gemm_epilogue_on(int32_t route, int32_t slices, const uint8_t* aq, const uint8_t* as, brq_layout a_layout, const uint8_t* wq, const uint8_t* ws,
                                           brq_layout w_layout, int64_t M, int64_t N, int64_t K, const float* bias, int32_t act,
                                           const void* residual, brq_dtype rdt, int64_t ldr, void* y, brq_dtype ydt, int64_t ldy, void* workspace,
                                           int64_t workspace_bytes, void* stream) {
    BRQ_CHECK(brq::check_gemm(aq, as, a_layout, wq, ws, w_layout, M, N, K, y, ydt, ldy));
    BRQ_CHECK(check_epilogue(M, N, bias, (brq_activation)act, residual, rdt, ldr, y, ydt, ldy));
    if (!aligned(workspace, 16)) return BRQ_ERR_ALIGN;
    const brq::Operand a{aq, as, a_layout == BRQ_LAYOUT_TILED}, w{wq, ws, w_layout == BRQ_LAYOUT_TILED};
    brq::GemmShape g{M, N, K, a.tiled, w.tiled, ydt == BRQ_BF16, ldy, reinterpret_cast<uintptr_t>(y)};
    g.epilogue = true;
    if (M == 0 || N == 0 || slices < 1 || !brq::gemm_route_supported(route, g)) return BRQ_ERR_SHAPE;
    const brq::GemmSplit sp{route == BRQ_GEMM_64x128 ? 64 : route == BRQ_GEMM_128x128 ? 128 : 0, slices};
    if (slices > 1) {
        if (!brq::gemm_split_supported(g, sp)) return BRQ_ERR_SHAPE;
        const int64_t need = brq::split_gemm_workspace(g, sp);
        if (!workspace) return BRQ_ERR_NULL;
        if (need > workspace_bytes) return BRQ_ERR_SHAPE;
    }
    int cus = 0;
    if (brq::device_cus(&cus) != hipSuccess) return BRQ_ERR_LAUNCH;
    const brq::Epilogue e = epilogue(bias, (brq_activation)act, residual, rdt, ldr, ydt);
    if (slices > 1) return launched(brq::launch_gemm_split(sp, a, w, g, y, workspace, e, static_cast<hipStream_t>(stream)));
    return launched(brq::launch_gemm_route(route, a, w, g, y, static_cast<hipStream_t>(stream), &e));
}

}  // extern "C"
