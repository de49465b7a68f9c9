// W4A4 product of up to 16 rows with bias, activation and residual behind it: 16 columns a workgroup, its 8 wavefronts each an eighth of K.
//
// The weights cross HBM once and there is next to nothing to multiply, so the time is what the loads wait for.  A wavefront that walks all of K
// for its columns (k_gemm_smallm) has a chain of K / 512 superstages, 0.35 us each with four of them on their way; here the chain is an eighth of that, and
// 16 columns a workgroup are twice as many workgroups.  Superstage s goes to wavefront s % 8: a workgroup's loads stay close together in K.  The
// contraction is v_mfma_scale_f32_16x16x128: lane (r, q) = (lane & 15, lane >> 4) supplies group q of a 128-element stage of row r of either operand,
// 16 bytes of codes straight from global memory and its byte of the row's 16 scales of a superstage.  The activations are few and lie in the L2.
// The eighths meet in LDS and are added in the wavefronts' order; thread t finishes element (t / 16, t % 16), whose bias and residual it asked for
// before everything else.
#include "gemm_epilogue.h"

namespace brq {
namespace {

constexpr int WAVES = 8;

// SETS superstages in registers; TAIL = the wavefront's number of them mod SETS (all wavefronts go through as many: past the end the last one again,
// with scale bytes 0 in both operands, 2^-254 times at most 36 * 32 a group, which vanishes).
template <int SETS, int TAIL>
__global__ void __launch_bounds__(64 * WAVES) k_gemm_few(const uint8_t* __restrict__ aq, const uint8_t* __restrict__ as, int a_tiled, const uint8_t* __restrict__ wq,
                                                         const uint8_t* __restrict__ ws, int w_tiled, int M, int N, int K, void* y, int64_t ldy, Epilogue e) {
    __shared__ float part[WAVES][64][4];
    load_args(aq, as, a_tiled, wq, ws, w_tiled, M, N, K);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, q = lane >> 4, n0 = blockIdx.x * 16;
    const int nss = (K + 511) / 512, count = (nss + WAVES - 1) / WAVES;
    const RowView va(aq, as, a_tiled != 0, min(r, M - 1), K), vw(wq, ws, w_tiled != 0, min(n0 + r, N - 1), K);
    // the element that this thread finishes
    const int row = tid >> 4, col = n0 + (tid & 15);
    const bool mine = row < M && col < N;               // (of the first 256 threads)
    uint32_t res = 0;
    float bias = 0.0f;
    if (mine) {
        if (e.res) res = e.res_bf16 ? (uint32_t)reinterpret_cast<const uint16_t*>(e.res + row * e.res_pitch)[col] : reinterpret_cast<const uint32_t*>(e.res + row * e.res_pitch)[col];
        if (e.bias) bias = e.bias[col];
    }
    v4i cw[SETS][4], ca[SETS][4], sw[SETS], sa[SETS];
    auto load = [&](auto Kc, int i) __attribute__((always_inline)) {
        constexpr int k = decltype(Kc)::value;
        const int ss = min(wave + i * WAVES, nss - 1);
#pragma unroll
        for (int t = 0; t < 4; ++t) cw[k][t] = vw.group(16 * ss + 4 * t + q);
        sw[k] = *reinterpret_cast<const v4i*>(vw.scales + (int64_t)ss * vw.sstep);
#pragma unroll
        for (int t = 0; t < 4; ++t) ca[k][t] = va.group(16 * ss + 4 * t + q);
        sa[k] = *reinterpret_cast<const v4i*>(va.scales + (int64_t)ss * va.sstep);
        __builtin_amdgcn_sched_barrier(0);
    };
    v4f acc = {};
    auto multiply = [&](auto Kc, int i) __attribute__((always_inline)) {
        constexpr int k = decltype(Kc)::value;
        const int keep = wave + i * WAVES < nss ? 0xff : 0;              // uniform
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            v8i a = {}, b = {};
            a[0] = ca[k][t][0]; a[1] = ca[k][t][1]; a[2] = ca[k][t][2]; a[3] = ca[k][t][3];
            b[0] = cw[k][t][0]; b[1] = cw[k][t][1]; b[2] = cw[k][t][2]; b[3] = cw[k][t][3];
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)((uint32_t)sa[k][t] >> (8 * q)) & keep, 0, (int)((uint32_t)sw[k][t] >> (8 * q)) & keep);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    static_for([&](auto Kc) __attribute__((always_inline)) { load(Kc, decltype(Kc)::value); }, IC<SETS>{});
    int i = 0;
    for (; i + 2 * SETS <= count; i += SETS)
        static_for([&](auto Kc) __attribute__((always_inline)) { multiply(Kc, i + decltype(Kc)::value); load(Kc, i + SETS + decltype(Kc)::value); }, IC<SETS>{});
    // SETS + TAIL superstages are left, or fewer than SETS in all
    static_for([&](auto Kc) __attribute__((always_inline)) {
        multiply(Kc, i + decltype(Kc)::value);
        if constexpr (decltype(Kc)::value < TAIL) load(Kc, i + SETS + decltype(Kc)::value);
    }, IC<SETS>{});
    static_for([&](auto Kc) __attribute__((always_inline)) { multiply(Kc, i + SETS + decltype(Kc)::value); }, IC<TAIL>{});
    *reinterpret_cast<v4f*>(part[wave][lane]) = acc;
    __syncthreads();
    if (!mine || tid >= 256) return;
    // element (row, column) of the 16 x 16: register row % 4 of lane (column, row / 4)
    const int l = (row >> 2) * 16 + (tid & 15);
    float v[1] = {part[0][l][row & 3]};
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v[0] += part[w][l][row & 3];
    if (e.bias) v[0] += bias;
    activate(v, e.act);
    if (e.res) v[0] += as_f32(e.res_bf16 ? res << 16 : res);
    if (e.out_bf16) reinterpret_cast<uint16_t*>(y)[row * ldy + col] = (uint16_t)f32_to_bf16_bits(v[0]);
    else reinterpret_cast<float*>(y)[row * ldy + col] = v[0];
}

}  // namespace

hipError_t launch_gemm_few(const Operand& a, const Operand& w, const GemmShape& g, void* y, const Epilogue& epi, hipStream_t s) {
    const int64_t nss = g.padded_k() / 512, count = (nss + WAVES - 1) / WAVES;
    const dim3 grid((uint32_t)((g.N + 15) / 16)), block(64 * WAVES);
    auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, block, 0, s, a.codes, a.scales, (int)a.tiled, w.codes, w.scales, (int)w.tiled, (int)g.M, (int)g.N, (int)g.K, y, g.ldy, epi);
    };
    if (count == 1) launch(k_gemm_few<1, 0>);
    else if (count == 2) launch(k_gemm_few<2, 0>);
    else if (count == 3) launch(k_gemm_few<3, 0>);
    else if (count % 4 == 0) launch(k_gemm_few<4, 0>);
    else if (count % 4 == 1) launch(k_gemm_few<4, 1>);
    else if (count % 4 == 2) launch(k_gemm_few<4, 2>);
    else launch(k_gemm_few<4, 3>);
    return hipGetLastError();
}

}  // namespace brq
