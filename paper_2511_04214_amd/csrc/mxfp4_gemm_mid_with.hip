// The one-tile products with bias, activation and residual behind them (kernels: mxfp4_gemm_mid.h): a unit of its own, since each of the
// two takes minutes to compile.
#include "mxfp4_gemm_mid.h"

namespace brq {

hipError_t setup_gemm_mid_with() { return mid_setup<true>(); }

hipError_t launch_gemm_any_k_with(const Operand& a, const Operand& w, int64_t M, int64_t N, int64_t K, void* y, bool out_bf16, int64_t ldy, hipStream_t s,
                                  const Epilogue& epi) {
    return mid_launch_any_k<true>(a, w, M, N, K, y, out_bf16, ldy, s, EpilogueArg<true>{epi});
}

hipError_t launch_gemm_mid_with(int tile, const Operand& a, const Operand& w, int64_t M, int64_t N, int64_t K, void* y, bool out_bf16, int64_t ldy, hipStream_t s,
                                const Epilogue& epi) {
    return mid_launch<true>(tile, a, w, M, N, K, y, out_bf16, ldy, s, EpilogueArg<true>{epi});
}

}  // namespace brq
