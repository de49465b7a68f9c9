// W4A4 product of up to 64 rows with bias, activation and residual behind it: 16, 32 or 48 columns a workgroup, its 8 wavefronts each an eighth of K.
//
// The weights cross HBM once and there is little to multiply, so the time is what the loads wait for.  A wavefront that walks all of K
// for its columns (k_gemm_smallm) has a chain of K / 512 superstages, 0.35 us each with four of them on their way; here the chain is an eighth of that, and
// 16 columns a workgroup are twice as many workgroups.  Superstage s goes to wavefront s % 8: a workgroup's loads stay close together in K.  The
// contraction is v_mfma_scale_f32_16x16x128: lane (r, q) = (lane & 15, lane >> 4) supplies group q of a 128-element stage of row r of either operand,
// 16 bytes of codes straight from global memory and its byte of the row's 16 scales of a superstage.  The activations are few and lie in the L2, where
// every workgroup reads all of them: that, and what is in registers at once, ends the gain with many rows, a long K or many columns.
// The eighths meet in LDS and are added in the wavefronts' order, 16 columns at a time; thread t finishes elements (t / 16, t % 16) and 32 rows below, whose bias and
// residual it asked for before everything else.
// us, weights in no cache, tiled, with a bias: 1 x 4096 x 14336 8.2 (HBM: 6), 48 x 4096 x 4096 5.8, 48 x 4096 x 11264 11.0, 48 x 11008 x 4096 9.9 (24 MB).
#include "gemm_epilogue.h"

namespace brq {
namespace {

constexpr int WAVES = 8;

// TILES, COLS: tiles of 16 rows, of 16 columns.  SETS superstages in registers; TAIL = the wavefront's number of them mod SETS (all wavefronts go through as many: past the end
// the last one again, with scale bytes 0 in both operands, 2^-254 times at most 36 * 32 a group, which vanishes).
template <int TILES, int COLS, int SETS, int TAIL, bool LOOP>
__global__ void __launch_bounds__(64 * WAVES) k_gemm_few(const uint8_t* __restrict__ aq, const uint8_t* __restrict__ as, int a_tiled, const uint8_t* __restrict__ wq,
                                                         const uint8_t* __restrict__ ws, int w_tiled, int M, int N, int K, void* y, int64_t ldy, Epilogue e) {
    __shared__ float part[WAVES][TILES][64][4];
    load_args(aq, as, a_tiled, wq, ws, w_tiled, M, N, K);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, q = lane >> 4, n0 = blockIdx.x * (16 * COLS);
    const int nss = (K + 511) / 512, count = (nss + WAVES - 1) / WAVES;
    // where the rows' codes and scales begin, and their steps
    const uint8_t *ac[TILES], *asc[TILES], *wc[COLS], *wsc[COLS];
    uint32_t cstep = 0, sstep = 0, wcstep = 0, wsstep = 0;
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
        const RowView vw(wq, ws, w_tiled != 0, min(n0 + 16 * x + r, N - 1), K);
        wc[x] = vw.codes; wsc[x] = vw.scales; wcstep = vw.cstep; wsstep = vw.sstep;
    }
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
        const RowView va(aq, as, a_tiled != 0, min(16 * x + r, M - 1), K);
        ac[x] = va.codes; asc[x] = va.scales; cstep = va.cstep; sstep = va.sstep;
    }
    // the elements that this thread finishes: rows tid / 16 and, with more than 2 tiles, 32 below it
    constexpr int EACH = (TILES + 1) / 2;
    const int row = tid >> 4, col = n0 + (tid & 15);
    uint32_t res[COLS][EACH] = {};
    float bias[COLS] = {};
#pragma unroll
    for (int z = 0; z < COLS; ++z) {
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (row + 32 * j < M && col + 16 * z < N && e.res) {
                const uint8_t* const p = e.res + (row + 32 * j) * e.res_pitch;
                res[z][j] = e.res_bf16 ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[col + 16 * z] : reinterpret_cast<const uint32_t*>(p)[col + 16 * z];
            }
        if (col + 16 * z < N && e.bias) bias[z] = e.bias[col + 16 * z];
    }
    v4i cw[SETS][COLS][4], ca[SETS][TILES][4], sw[SETS][COLS], sa[SETS][TILES];
    auto load = [&](auto Kc, int i) __attribute__((always_inline)) {
        constexpr int k = decltype(Kc)::value;
        const int ss = min(wave + i * WAVES, nss - 1);
#pragma unroll
        for (int x = 0; x < COLS; ++x) {
#pragma unroll
            for (int t = 0; t < 4; ++t) cw[k][x][t] = *reinterpret_cast<const v4i*>(wc[x] + (int64_t)(4 * ss + t) * wcstep + q * 16);
            sw[k][x] = *reinterpret_cast<const v4i*>(wsc[x] + (int64_t)ss * wsstep);
        }
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
#pragma unroll
            for (int t = 0; t < 4; ++t) ca[k][x][t] = *reinterpret_cast<const v4i*>(ac[x] + (int64_t)(4 * ss + t) * cstep + q * 16);
            sa[k][x] = *reinterpret_cast<const v4i*>(asc[x] + (int64_t)ss * sstep);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    v4f acc[TILES][COLS] = {};
    auto multiply = [&](auto Kc, int i) __attribute__((always_inline)) {
        constexpr int k = decltype(Kc)::value;
        const int keep = wave + i * WAVES < nss ? 0xff : 0;              // uniform
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int z = 0; z < COLS; ++z) {
#pragma unroll
                for (int x = 0; x < TILES; ++x) {
                    v8i a = {}, b = {};
                    a[0] = ca[k][x][t][0]; a[1] = ca[k][x][t][1]; a[2] = ca[k][x][t][2]; a[3] = ca[k][x][t][3];
                    b[0] = cw[k][z][t][0]; b[1] = cw[k][z][t][1]; b[2] = cw[k][z][t][2]; b[3] = cw[k][z][t][3];
                    acc[x][z] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[x][z], 4, 4, 0, (int)((uint32_t)sa[k][x][t] >> (8 * q)) & keep, 0,
                                                                                  (int)((uint32_t)sw[k][z][t] >> (8 * q)) & keep);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    static_for([&](auto Kc) __attribute__((always_inline)) { load(Kc, decltype(Kc)::value); }, IC<SETS>{});
    int i = 0;
    if constexpr (LOOP) {
#pragma unroll 1
        for (; i + 2 * SETS <= count; i += SETS)
            static_for([&](auto Kc) __attribute__((always_inline)) { multiply(Kc, i + decltype(Kc)::value); load(Kc, i + SETS + decltype(Kc)::value); }, IC<SETS>{});
    }
    // SETS + TAIL superstages are left
    static_for([&](auto Kc) __attribute__((always_inline)) {
        multiply(Kc, i + decltype(Kc)::value);
        if constexpr (decltype(Kc)::value < TAIL) load(Kc, i + SETS + decltype(Kc)::value);
    }, IC<SETS>{});
    static_for([&](auto Kc) __attribute__((always_inline)) { multiply(Kc, i + SETS + decltype(Kc)::value); }, IC<TAIL>{});
#pragma unroll
    for (int z = 0; z < COLS; ++z) {                    // 16 columns at a time
        if (z > 0) __syncthreads();
#pragma unroll
        for (int x = 0; x < TILES; ++x) *reinterpret_cast<v4f*>(part[wave][x][lane]) = acc[x][z];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int m = row + 32 * j, n = col + 16 * z;
            if (m < M && n < N) {
                // element (row, column) of a 16 x 16: register row % 4 of lane (column, row / 4)
                const int x = m >> 4, l = ((m & 15) >> 2) * 16 + (tid & 15);
                float v[1] = {part[0][x][l][m & 3]};
#pragma unroll
                for (int w = 1; w < WAVES; ++w) v[0] += part[w][x][l][m & 3];
                if (e.bias) v[0] += bias[z];
                activate(v, e.act);
                if (e.res) v[0] += as_f32(e.res_bf16 ? res[z][j] << 16 : res[z][j]);
                if (e.out_bf16) reinterpret_cast<uint16_t*>(y)[m * ldy + n] = (uint16_t)f32_to_bf16_bits(v[0]);
                else reinterpret_cast<float*>(y)[m * ldy + n] = v[0];
            }
        }
    }
}

using FewKern = void (*)(const uint8_t*, const uint8_t*, int, const uint8_t*, const uint8_t*, int, int, int, int, void*, int64_t, Epilogue);
// Superstages in registers: as many as 200 of those hold, at most 4.
constexpr int sets_of(int tiles, int cols) { return 10 / (tiles + cols) > 4 ? 4 : 10 / (tiles + cols); }
// Superstages a wavefront that there are kernels for, up to two rounds of the registers: one tile takes any number, in a loop.
constexpr int most_of(int tiles, int cols) { return tiles == 1 ? 2 * sets_of(1, 1) : tiles == 4 || tiles + cols == 6 ? 2 : tiles + cols == 5 ? 3 : tiles == 3 ? 3 : 4; }
template <int TILES, int COLS, int N = 1>
FewKern few_kern(int64_t count) {
    constexpr int SETS = sets_of(TILES, COLS);
    if (count == N) return k_gemm_few<TILES, COLS, N <= SETS ? N : SETS, N <= SETS ? 0 : N - SETS, false>;
    if constexpr (TILES == 1 && N > SETS)
        if (count > 2 * SETS && count % SETS == N % SETS) return k_gemm_few<TILES, COLS, SETS, N % SETS, true>;
    if constexpr (N < most_of(TILES, COLS)) return few_kern<TILES, COLS, N + 1>(count);
    else return nullptr;
}
template <int COLS>
FewKern few_kern_of(int tiles, int64_t count) { return tiles == 2 ? few_kern<2, COLS>(count) : tiles == 3 ? few_kern<3, COLS>(count) : few_kern<4, COLS>(count); }

int64_t superstages(const GemmShape& g) { return (g.padded_k() / 512 + WAVES - 1) / WAVES; }

// Tiles of columns: as many as a round of the chip needs, at most 3, and of two tiles of rows one where K is one superstage a wavefront and a CU so holds more than one
// workgroup (32 x 8192 x 4096 7.6 with two -> 6.6 us, 32 x 6144 x 4096 6.8 -> 6.5).
struct FewChoice { FewKern kern; int cols; };      // kern null: there is none
FewChoice few_choice(const GemmShape& g, int cus) {
    const int64_t count = superstages(g);
    const int tiles = (int)((g.M + 15) / 16);
    int cols = tiles == 1 || g.N <= 16 * (int64_t)cus ? 1 : g.N <= 32 * (int64_t)cus ? 2 : 3;
    if (tiles == 2 && cols == 2 && count == 1 && g.K > 2048) cols = 1;
    while (cols > 1 && count > most_of(tiles, cols)) --cols;
    return {tiles == 1 ? few_kern<1, 1>(count) : cols == 1 ? few_kern_of<1>(tiles, count) : cols == 2 ? few_kern_of<2>(tiles, count) : few_kern_of<3>(tiles, count), cols};
}

}  // namespace

bool few_gemm_supported(const GemmShape& g) {
    if (g.M < 1 || g.M > 64 || !g.whole_k() || g.padded_k() >= (int64_t(1) << 26)) return false;
    return g.M <= 16 || superstages(g) <= most_of((int)((g.M + 15) / 16), 1);
}

bool few_gemm_has_kernel(const GemmShape& g, int cus) { return few_choice(g, cus).kern != nullptr; }

hipError_t launch_gemm_few(const Operand& a, const Operand& w, const GemmShape& g, void* y, const Epilogue& epi, hipStream_t s) {
    int cus = 0;
    if (hipError_t e = device_cus(&cus); e != hipSuccess) return e;
    const FewChoice c = few_choice(g, cus);
    const FewKern kern = c.kern;
    const int cols = c.cols;
    if (!kern) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, dim3((uint32_t)((g.N + 16 * cols - 1) / (16 * cols))), dim3(64 * WAVES), 0, s, a.codes, a.scales, (int)a.tiled, w.codes, w.scales, (int)w.tiled,
                       (int)g.M, (int)g.N, (int)g.K, y, g.ldy, epi);
    return hipGetLastError();
}

}  // namespace brq
