// Products of few tiles and a long K, split along K: the one-tile kernels (mxfp4_gemm_mid.h) write each slice's fp32 sums, and one more launch adds
// the slices in their order and does what follows the product.
#include "mxfp4_gemm_mid.h"

namespace brq {
namespace {

using mid::k_gemm_mid;
using SplitKern = void (*)(const uint8_t*, const uint8_t*, const uint8_t*, const uint8_t*, int, int, int, void*, int64_t, int, int, int, EpilogueArg<false>, mid::SplitArg<true>);
struct SplitVariant { int dw, da; SplitKern kern; };
#define BRQ_SPLIT(MB, DW, DA, PAIR) {DW, DA, k_gemm_mid<false, 2, MB, DW, DA, PAIR, false, true>}
const SplitVariant variants[2][2] = {{BRQ_SPLIT(1, 6, 6, false), BRQ_SPLIT(1, 6, 6, true)},      // [64 or 128 rows][pairs]
                                     {BRQ_SPLIT(2, 4, 4, false), BRQ_SPLIT(2, 6, 6, true)}};
#undef BRQ_SPLIT

// Each thread 4 columns of a row: what there is of their slices is asked for at once, added in the slices' order.
template <int SLICES>
__global__ __launch_bounds__(256) void k_join(const float* __restrict__ part, int slices, int M, int N, int64_t pitch, void* y, int64_t ldy, Epilogue e) {
    const int64_t quads = pitch / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= M * quads) return;
    const int64_t row = i / quads, col = (i - row * quads) * 4;
    const float* const p = part + row * pitch + col;
    v4f t[SLICES];
#pragma unroll
    for (int k = 0; k < SLICES; ++k) t[k] = *reinterpret_cast<const v4f*>(p + (int64_t)min(k, slices - 1) * M * pitch);
    const int n = (int)min((int64_t)4, N - col);
    float b[4] = {}, r[4] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < n) {
            if (e.bias) b[k] = e.bias[col + k];
            if (e.res) r[k] = residual_at(e, row, col + k);
        }
    float v[4] = {t[0].x, t[0].y, t[0].z, t[0].w};
#pragma unroll
    for (int s = 1; s < SLICES; ++s)
        if (s < slices) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += t[s][k];
        }
    if (e.bias) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += b[k];
    }
    activate(v, e.act);
    if (e.res) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += r[k];
    }
    if (e.out_bf16) {
        uint16_t* const o = reinterpret_cast<uint16_t*>(y) + row * ldy + col;
        typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
        if (n == 4) *reinterpret_cast<u2_any*>(o) = u2_any{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else for (int k = 0; k < n; ++k) o[k] = (uint16_t)f32_to_bf16_bits(v[k]);
    } else {
        float* const o = reinterpret_cast<float*>(y) + row * ldy + col;
        typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
        if (n == 4) *reinterpret_cast<f4_any*>(o) = f4_any{v[0], v[1], v[2], v[3]};
        else for (int k = 0; k < n; ++k) o[k] = v[k];
    }
}

int64_t pitch_of(int64_t N) { return (N + 3) / 4 * 4; }

}  // namespace

hipError_t setup_gemm_split() {
    for (int mb = 1; mb <= 2; ++mb)
        for (const SplitVariant& v : variants[mb - 1])
            if (hipError_t e = hipFuncSetAttribute((const void*)v.kern, hipFuncAttributeMaxDynamicSharedMemorySize, mid::lds_bytes(2, mb, v.dw, v.da)); e != hipSuccess) return e;
    return hipSuccess;
}

int64_t split_gemm_workspace(const GemmShape& g, const GemmSplit& s) { return s.slices > 1 ? s.slices * g.M * pitch_of(g.N) * 4 : 0; }

hipError_t launch_gemm_split(const GemmSplit& sp, const Operand& a, const Operand& w, const GemmShape& g, void* y, void* workspace, const Epilogue& epi, hipStream_t s) {
    const int mb = sp.rows / 64;
    const SplitVariant& v = variants[mb - 1][mid_gemm_pairs(mb - 1, a.tiled && w.tiled, g.K)];
    const int64_t T = (g.M + 64 * mb - 1) / (64 * mb) * ((g.N + 127) / 128) * sp.slices, pitch = pitch_of(g.N);
    // (no streaming hint: the slices are read again at once)
    hipLaunchKernelGGL(v.kern, dim3((uint32_t)((T + 7) / 8 * 8)), dim3(256), mid::lds_bytes(2, mb, v.dw, v.da), s, a.codes, a.scales, w.codes, w.scales, (int)g.M, (int)g.N,
                       (int)g.K, workspace, pitch, (int)a.tiled, (int)w.tiled, 0, EpilogueArg<false>{}, mid::SplitArg<true>{sp.slices});
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const dim3 grid((uint32_t)((g.M * (pitch / 4) + 255) / 256));
    const float* const part = static_cast<const float*>(workspace);
    auto join = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, part, sp.slices, (int)g.M, (int)g.N, pitch, y, g.ldy, epi); };
    if (sp.slices <= 2) join(k_join<2>);
    else if (sp.slices <= 4) join(k_join<4>);
    else if (sp.slices <= 8) join(k_join<8>);
    else join(k_join<MAX_SLICES>);
    return hipGetLastError();
}

}  // namespace brq
