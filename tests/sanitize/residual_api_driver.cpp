// Drives the host side of the residual calls (include/brq_residual.h) at the ends of their arguments' ranges, with launches that do
// nothing: what is refused, what reaches a launch, and that no check overflows on its way (the sanitizers' part).
#include <cstdio>
#include <cstdlib>

#include "../../include/brq_residual.h"
#include "../../paper_2511_04214_amd/csrc/brq_launch.h"
#include "../../paper_2511_04214_amd/csrc/brq_residual.h"

static int launches;
// What a launch may count on: whole rows, and offsets in bytes that 64 bits hold.
static void rows_hold(const brq::RowSet& r, int64_t M, int64_t K) {
    int64_t end;
    if (r.p == nullptr) return;
    if (r.pitch < K * (r.bf16 ? 2 : 4) || r.pitch % 16 != 0 || __builtin_mul_overflow(r.pitch, M, &end)) std::abort();
}
namespace brq {
hipError_t device_cus(int* cus) { *cus = 256; return hipSuccess; }
brq_status check_gemm(const uint8_t*, const uint8_t*, brq_layout, const uint8_t*, const uint8_t*, brq_layout, int64_t M, int64_t N, int64_t K, const void*, brq_dtype,
                      int64_t ldy) {      // (its own ranges are driven with the library's)
    const int64_t most = int64_t(1) << 31;
    return M < 0 || N < 0 || K <= 0 || K % 32 != 0 || M >= most || N >= most || K >= most || ldy < N || ldy >= most / 2 ? BRQ_ERR_SHAPE : BRQ_OK;
}
hipError_t launch_add_rms_norm(const NormArgs& a, bool, hipStream_t) {
    rows_hold(a.x, a.M, a.K), rows_hold(a.res, a.M, a.K), rows_hold(a.h, a.M, a.K), rows_hold(a.y, a.M, a.K);
    ++launches;
    return hipSuccess;
}
hipError_t launch_add_rms_norm_backward(const NormBackwardArgs& a, hipStream_t) {
    rows_hold(a.h, a.M, a.K), rows_hold(a.gy, a.M, a.K), rows_hold(a.gh, a.M, a.K), rows_hold(a.dh, a.M, a.K);
    ++launches;
    return hipSuccess;
}
int64_t norm_backward_parts(int64_t M, int64_t) { return M < 512 ? (M + 1) / 2 : 512; }
hipError_t launch_mxfp4_gemm(const Operand&, const Operand&, const GemmShape& g, void*, hipStream_t, const Epilogue* e, void*) {
    int64_t end;
    if (e && (g.M <= 0 || __builtin_mul_overflow(e->res_pitch, g.M, &end))) std::abort();
    ++launches;
    return hipSuccess;
}
GemmSplit gemm_split(const GemmShape&, int) { return {64, 4}; }
int64_t split_gemm_workspace(const GemmShape&, const GemmSplit&) { return 1024; }
bool gemm_split_supported(const GemmShape&, const GemmSplit& s) { return s.slices <= 16; }
bool gemm_route_supported(int route, const GemmShape&) { return route >= 0 && route < 12; }
hipError_t launch_gemm_split(const GemmSplit&, const Operand&, const Operand&, const GemmShape&, void*, void*, const Epilogue&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_gemm_route(int, const Operand&, const Operand&, const GemmShape&, void*, hipStream_t, const Epilogue*) { ++launches; return hipSuccess; }
}  // namespace brq

#define EXPECT(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

int main() {
    const int64_t ends[] = {INT64_MIN, INT64_MIN + 1, -((int64_t)1 << 40), -1, 0, 1, 31, 32, 64, 65, 4096, 32768, 32800, (1 << 30) - 32, (1 << 30) - 8, 1 << 30, INT32_MAX,
                            (int64_t)1 << 31, (int64_t)1 << 34, (int64_t)1 << 62, INT64_MAX - 31, INT64_MAX};
    alignas(16) static float f[64];
    alignas(16) static uint8_t bytes[64];
    static uint8_t* const P[4] = {bytes, bytes + 16, bytes + 32, nullptr};
    int64_t n = -1;
    long calls = 0, taken = 0;
    auto count = [&](brq_status s) { ++calls; taken += s == BRQ_OK; };
    for (int64_t M : ends)
        for (int64_t K : ends) {
            const brq_status s = brq_add_rms_norm_backward_workspace(M, K, &n);
            EXPECT(s != BRQ_OK || n >= 0);
            count(s);
            count(brq_mxfp4_gemm_epilogue_workspace(BRQ_LAYOUT_TILED, BRQ_LAYOUT_ROWMAJOR, M, K, 64, &n));
            for (int64_t a : ends)
                for (int64_t b : ends) {
                    for (int i = 0; i < 4; ++i) {
                        count(brq_add_rms_norm(f, BRQ_BF16, a, P[i], BRQ_F32, b, M, K, f, 1e-6f, i == 3 ? nullptr : f + 16, b, f + 32, BRQ_BF16, a, nullptr));
                        count(brq_add_rms_norm_rotate_quantize_fused(f, BRQ_F32, a, P[i], BRQ_BF16, b, M, K, nullptr, 0.0f, nullptr, b, BRQ_F32, i == 0 ? 1 : 32, nullptr, bytes, bytes,
                                                                     BRQ_LAYOUT_TILED, nullptr));
                        count(brq_add_rms_norm_backward(f, BRQ_F32, a, P[0], BRQ_BF16, b, P[i], a, M, K, f, 0.0f, f + 16, b, f, bytes, INT64_MAX, nullptr));
                    }
                    for (int act : {0, 1, 2, 3, 4, 0x7ffffffe})
                        count(brq_mxfp4_gemm_epilogue(bytes, bytes, BRQ_LAYOUT_TILED, bytes, bytes, BRQ_LAYOUT_ROWMAJOR, M, K, 64, f, (brq_activation)act, P[1], BRQ_F32, a, f, BRQ_BF16, b,
                                                      bytes, 1024, nullptr));
                    count(brq_mxfp4_gemm_epilogue(bytes, bytes, BRQ_LAYOUT_TILED, bytes, bytes, BRQ_LAYOUT_TILED, 1, M, K, nullptr, BRQ_ACT_RELU, P[1], BRQ_BF16, a, f, BRQ_F32, b, bytes,
                                                  b, nullptr));
                }
        }
    for (int64_t B : ends) count(brq_add_rms_norm_rotate_quantize_fused(f, BRQ_F32, 64, nullptr, BRQ_F32, 0, 1, 64, f, 1.0f, nullptr, 0, BRQ_BF16, B, nullptr, bytes, bytes, BRQ_LAYOUT_ROWMAJOR, nullptr));
    EXPECT(taken > 0 && taken < calls && launches > 0);
    std::printf("%ld calls, %ld taken, %d launches\nresidual api sanitizer driver ok\n", calls, taken, launches);
    return 0;
}
