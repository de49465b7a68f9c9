// The one-tile products alone (kernels: mxfp4_gemm_mid.h), and which shapes they take.
#include "mxfp4_gemm_mid.h"

namespace brq {

bool mid_gemm_pairs(int tile, bool both_tiled, int64_t K) { return !both_tiled && (K > 1024 || tile > 2); }

hipError_t setup_gemm_mid() {
    if (hipError_t e = mid_setup<false>(); e != hipSuccess) return e;
    if (hipError_t e = setup_gemm_split(); e != hipSuccess) return e;
    return setup_gemm_mid_with();
}

// Whole superstages, or both operands row-major with K a multiple of 128 and at least one superstage.  A lane's offset
// inside the tile, below 64 max(NA, MB) rows of Kp / 2 bytes, has 32 bits, and the offset along K 31 (32 Kp bytes).
bool mid_gemm_supported(int tile, const GemmShape& g) {
    const mid::Variant<false>& v = mid::singles<false>[tile];
    const int64_t Kp = g.padded_k(), slabs = v.na > v.mb ? v.na : v.mb;
    return g.M > 0 && g.N > 0 && (g.whole_k() || (!g.a_tiled && !g.w_tiled && g.K % 128 == 0 && g.K >= 512)) &&
           Kp < (int64_t(1) << 26) && slabs * 32 * Kp <= (int64_t(1) << 32);
}

hipError_t launch_gemm_any_k(const Operand& a, const Operand& w, int64_t M, int64_t N, int64_t K, void* y, bool out_bf16, int64_t ldy, hipStream_t s,
                             const Epilogue* epi) {
    return epi ? launch_gemm_any_k_with(a, w, M, N, K, y, out_bf16, ldy, s, *epi) : mid_launch_any_k<false>(a, w, M, N, K, y, out_bf16, ldy, s, {});
}

hipError_t launch_gemm_mid(int tile, const Operand& a, const Operand& w, int64_t M, int64_t N, int64_t K, void* y,
                           bool out_bf16, int64_t ldy, hipStream_t s, const Epilogue* epi) {
    return epi ? launch_gemm_mid_with(tile, a, w, M, N, K, y, out_bf16, ldy, s, *epi) : mid_launch<false>(tile, a, w, M, N, K, y, out_bf16, ldy, s, {});
}

}  // namespace brq
