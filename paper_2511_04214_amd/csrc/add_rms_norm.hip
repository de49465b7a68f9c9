// The residual's addition and the RMS norm of the sum, alone and in front of the online step, and the gradients.
//
// A row is held in registers from its load to its last store: W wavefronts of 64 lanes, each lane C chunks of 8 elements, chunk
// number (c * W + wavefront) * 64 + chunk_of_lane(lane).  So everything crosses HBM once, and a wavefront's pass c is 512 consecutive
// elements, in the order that the rotations and the quantizer want (brq_device.h).  Lanes behind the row's end load its last chunk
// again, in bounds, and count for nothing.  The sum of squares is taken in fp32: in a lane 8 C products in the order of the elements, then
// pairs of lanes by chunk number, then the wavefronts in turn.  W and C depend on K alone, so the norm alone and the fused
// call have the same bits.
#include "mfma_fp4.h"
#include "brq_launch.h"
#include "brq_residual.h"

namespace brq {
namespace {

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xF, 0xF, true));
}

// Sum over a wavefront, every lane receiving it: chunks xor 1, 2, 4, 8 (the mirror images, in chunk_of_lane's order), 16, 32.
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}

// fl(1/sqrt(2^l2)) as in the row-wise kernels: a power of two, or sqrt(2)/2 times one.
__device__ constexpr uint32_t unit_bits(int l2) {
    return (l2 & 1) ? (0x3F3504F3u - ((uint32_t)((l2 - 1) / 2) << 23)) : (0x3F800000u - ((uint32_t)(l2 / 2) << 23));
}
// H_B / sqrt(B) on each B elements of a wavefront's 512, B = 2^l2b (uniform).
__device__ __forceinline__ void rotate(float (&v)[8], int l2b, uint32_t chunk) {
    float s = 1.0f;
    switch (l2b) {
#define BRQ_CASE(L) case L: wht_inwave<L>(v, chunk); s = wht_sign<L>(chunk) * as_f32(unit_bits(L)); break;
        BRQ_CASE(3) BRQ_CASE(4) BRQ_CASE(5) BRQ_CASE(6) BRQ_CASE(7) BRQ_CASE(8) BRQ_CASE(9)
#undef BRQ_CASE
        default: return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
}

// C chunks of a row as they come from memory: 16 bytes each of bf16, 32 of fp32.
template <int C>
struct Raw {
    v4i lo[C], hi[C];
    __device__ __forceinline__ void load(const uint8_t* row, bool bf16, const uint32_t (&kc)[C]) {
        const int shift = bf16 ? 4 : 5;
        // (no branch with a load at the end of both its sides: the compiler makes one of the two, to a place it has to keep in memory)
        static_for([&](auto c_) __attribute__((always_inline)) { constexpr int c = decltype(c_)::value; lo[c] = *reinterpret_cast<const v4i*>(row + (kc[c] << shift)); }, IC<C>{});
        if (!bf16)          // uniform
            static_for([&](auto c_) __attribute__((always_inline)) { constexpr int c = decltype(c_)::value; hi[c] = *reinterpret_cast<const v4i*>(row + (kc[c] << shift) + 16); }, IC<C>{});
    }
    __device__ __forceinline__ void widen(bool bf16, float (&v)[C][8]) const {
        if (bf16) {
            static_for([&](auto c_) __attribute__((always_inline)) {
                constexpr int c = decltype(c_)::value;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[c][2 * i] = bf16_lo((uint32_t)lo[c][i]);
                    v[c][2 * i + 1] = bf16_hi((uint32_t)lo[c][i]);
                }
            }, IC<C>{});
        } else {
            static_for([&](auto c_) __attribute__((always_inline)) {
                constexpr int c = decltype(c_)::value;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[c][i] = as_f32((uint32_t)lo[c][i]);
                    v[c][4 + i] = as_f32((uint32_t)hi[c][i]);
                }
            }, IC<C>{});
        }
    }
};

// The same without a stop on the way: one chunk, and a row of them.  (The fences keep the compiler from asking for everything at once: it has no
// registers for that.)
__device__ __forceinline__ void load_one(const uint8_t* row, bool bf16, uint32_t kc, float (&v)[8]) {
    Raw<1> t;
    float w[1][8];
    const uint32_t at[1] = {kc};
    t.load(row, bf16, at);
    t.widen(bf16, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = w[0][i];
}
// What is computed from the chunks' numbers is computed again for every row, not kept in registers: there are none for it.
template <int C>
__device__ __forceinline__ void renew(uint32_t (&kc)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        uint32_t k = kc[c];
        asm volatile("" : "+v"(k));
        kc[c] = k;
    }
}
template <int C>
__device__ __forceinline__ void load_row(const RowSet& x, int64_t row, const uint32_t (&kc)[C], float (&v)[C][8]) {
    const uint8_t* const from = x.p + row * x.pitch;
    static_for([&](auto c_) __attribute__((always_inline)) {
        constexpr int c = decltype(c_)::value;
        load_one(from, x.bf16, kc[c], v[c]);
        if constexpr (c % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    }, IC<C>{});
}

__device__ __forceinline__ void store_values(uint8_t* row, bool bf16, uint32_t kc, const float (&v)[8]) {
    if (bf16) {             // uniform
        *reinterpret_cast<v4i*>(row + kc * 16u) =
            v4i{(int)pack_bf16x2(v[0], v[1]), (int)pack_bf16x2(v[2], v[3]), (int)pack_bf16x2(v[4], v[5]), (int)pack_bf16x2(v[6], v[7])};
    } else {
        *reinterpret_cast<v4f*>(row + kc * 32u) = v4f{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<v4f*>(row + kc * 32u + 16) = v4f{v[4], v[5], v[6], v[7]};
    }
}

__device__ __forceinline__ void through_bf16(float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const uint32_t p = pack_bf16x2(v[i], v[i + 1]);
        v[i] = bf16_lo(p);
        v[i + 1] = bf16_hi(p);
    }
}

__device__ __forceinline__ void load_chunk_weight(const float* w, uint32_t kc, float (&v)[8]) {
    const v4f a = *reinterpret_cast<const v4f*>(w + kc * 8u), b = *reinterpret_cast<const v4f*>(w + kc * 8u + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
template <int C>
__device__ __forceinline__ void load_weight(const float* w, const uint32_t (&kc)[C], float (&v)[C][8]) {
#pragma unroll
    for (int c = 0; c < C; ++c) load_chunk_weight(w, kc[c], v[c]);
}

// Rows of a workgroup: 4 / W of W < 4 wavefronts, else one.
template <int W>
constexpr int rows_of = W < 4 ? 4 / W : 1;
template <int W>
constexpr int threads_of = W < 4 ? 256 : 64 * W;

// N sums over a row's wavefronts, every lane receiving them.  `part`: [wavefronts of the workgroup][N]; every thread of the workgroup calls.
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*part)[N], int wave) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63u) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) part[wave][n] = v[n];
        }
        __syncthreads();
        const int first = wave / W * W;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float s = part[first][n];
#pragma unroll
            for (int i = 1; i < W; ++i) s += part[first + i][n];
            v[n] = s;
        }
    }
}

// A workgroup for every row (or 4 / W of them), everything asked for at once, and registers for nothing beyond it: 31 to 63 with up to two chunks a lane, so that a
// CU holds 2048 threads of them.  (In a loop over rows the compiler keeps so much from turn to turn that it has 80 to 128.)
// Many rows are bound by HBM, few by the launch and the chain load, sum, barrier, store.  us, bf16 in and out with the sum, inputs in no cache, a loop over rows -> now, alone / fused with
// B = 32: 1 x 4096 2.8 -> 2.7 / 3.3 -> 3.0, 4096 x 2048 14.6 -> 14.8 / 15.0 -> 14.0, 4096 x 4096 26.1 -> 25.9 (5.2 TB/s) / 26.8 -> 25.2, 4096 x 6144 40.3 -> 40.4 / 46.9 -> 36.2, 4096 x 8192
// 50.4 -> 51.0 / 53.4 -> 46.5, 4096 x 16384 102 -> 100 / 100 -> 90, in the caches 1024 x 32768 66 -> 47 / 55 -> 43.  A residual in fp32: 8192 x 4096 76 (5.3 TB/s), 8192 x 8192 146 -> 149.
template <int W, int C, bool QUANT>
__global__ __launch_bounds__(threads_of<W>, C <= 2 ? 8 : 1) void k_add_rms_norm(const NormArgs a, const KPad pad, int64_t row0) {
    __shared__ float part[threads_of<W> / 64][1];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), sub = wave % W;
    const uint32_t lane = threadIdx.x & 63u, chunk = chunk_of_lane(lane), n = (uint32_t)(a.K / 8);
    uint32_t kc[C];
    bool in[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        kc[c] = (uint32_t)(c * W + sub) * 64u + chunk;
        in[c] = kc[c] < n;
        kc[c] = min(kc[c], n - 1);
    }
    const int64_t mine = row0 + (int64_t)blockIdx.x * rows_of<W> + wave / W, row = min(mine, a.M - 1);
    float v[C][8], w[C][8];
    {
        Raw<C> x, r;
        x.load(a.x.p + row * a.x.pitch, a.x.bf16, kc);
        if (a.res.p) r.load(a.res.p + row * a.res.pitch, a.res.bf16, kc);           // uniform
        if (C <= 2 && a.w) load_weight(a.w, kc, w);
        x.widen(a.x.bf16, v);
        if (a.res.p) {
            float t[C][8];
            r.widen(a.res.bf16, t);
            static_for([&](auto c_) __attribute__((always_inline)) {
                constexpr int c = decltype(c_)::value;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += t[c][i];
                if (a.res.bf16) through_bf16(v[c]);
            }, IC<C>{});
        }
    }
    // (all that was asked for is here before the sum is stored: else the compiler waits for that store too, in front of the squares)
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // vmcnt(0)
    if (a.h.p) {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (in[c] && mine < a.M) store_values(a.h.p + row * a.h.pitch, a.h.bf16, kc[c], v[c]);
    }
    float sum[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v[c][i], v[c][i], s);
        sum[0] += in[c] ? s : 0.0f;
    }
    row_sums<W, 1>(sum, part, wave);
    const float r = 1.0f / sqrtf(sum[0] / (float)a.K + a.eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const bool live = in[c] && mine < a.M;
        if constexpr (C > 2) {                          // (no registers to have it earlier)
            __builtin_amdgcn_sched_barrier(0);
            if (a.w) load_chunk_weight(a.w, kc[c], w[c]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[c][i] *= r;
            if (a.w) v[c][i] *= w[c][i];
        }
        if constexpr (!QUANT) {
            if (live) store_values(a.y.p + row * a.y.pitch, a.y.bf16, kc[c], v[c]);
        } else {
            // (whole quads, and whole blocks, are behind the row's end together: what they hold reaches no one else)
            if (a.y.bf16) through_bf16(v[c]);
            if (a.signs) apply_signs(v[c], a.signs + (size_t)kc[c] * 8);
            rotate(v[c], a.l2b, chunk);
            const uint32_t sb = e8m0_from_amax(quad_max(absmax8(v[c]))), codes = encode8_e2m1(v[c], sb);
            if (live) {
                const uint64_t at = a.tiled ? tiled_code_offset((uint32_t)row, kc[c], pad.stages) : ((uint64_t)row * n + kc[c]) * 4u;
                const uint64_t sat = a.tiled ? tiled_scale_offset((uint32_t)row, kc[c], pad.sstages) : ((uint64_t)row * n + kc[c]) >> 2;
                *reinterpret_cast<uint32_t*>(a.codes + at) = codes;
                if ((lane & 3u) == 0) a.scales[sat] = (uint8_t)sb;
            }
        }
    }
    if constexpr (QUANT) pad.zero(blockIdx.x * threads_of<W> + threadIdx.x, gridDim.x * threads_of<W>);
}

// Wavefronts to a row and chunks to a lane.
struct Split { int w, c; };
Split split_of(int64_t K) {
    const int64_t waves = (K + 511) / 512;              // of one chunk a lane
    Split s{1, 1};
    while (s.w * s.c < waves) s.w < 16 ? s.w *= 2 : s.c *= 2;
    return s;
}

}  // namespace

hipError_t launch_add_rms_norm(const NormArgs& a, bool quantize, hipStream_t stream) {
    int cus = 0;
    if (hipError_t e = device_cus(&cus); e != hipSuccess) return e;
    // Rows of 4097 to 8192: four workgroups of 8 wavefronts on a CU get further than two of 16 that meet at barriers, us, inputs in no cache: 4096 x 6144 fused 44.2 -> 36.2, alone
    // 42.1 -> 40.4, 4096 x 8192 51.3 -> 46.5, 52.8 -> 51.0, with a residual in fp32 75.9 -> 76.2.  (Fewer wavefronts for shorter rows: 1 x 4096 3.0 -> 3.5.)
    Split sp = split_of(a.K);
    if (sp.w == 16 && sp.c == 1) sp = {8, 2};
    constexpr int64_t most = int64_t(1) << 21;          // workgroups of a launch, which has less than 2^32 threads
    const KPad pad = KPad::of(quantize && a.tiled, a.codes, a.scales, a.M, a.K);
    switch (sp.w * 16 + sp.c) {
#define BRQ_NORM(W, C)                                                                                                                             \
    case W * 16 + C:                                                                                                                               \
        for (int64_t row = 0; row < a.M; row += most * rows_of<W>) {                                                                               \
            const int64_t rows = (a.M - row + rows_of<W> - 1) / rows_of<W>;                                                                       \
            const dim3 grid((uint32_t)(rows < most ? rows : most)), block(threads_of<W>);                                                          \
            if (quantize) hipLaunchKernelGGL((k_add_rms_norm<W, C, true>), grid, block, 0, stream, a, pad, row);                                   \
            else hipLaunchKernelGGL((k_add_rms_norm<W, C, false>), grid, block, 0, stream, a, pad, row);                                           \
        }                                                                                                                                          \
        break;
        BRQ_NORM(1, 1) BRQ_NORM(2, 1) BRQ_NORM(4, 1) BRQ_NORM(8, 1) BRQ_NORM(8, 2) BRQ_NORM(16, 2) BRQ_NORM(16, 4)
#undef BRQ_NORM
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

namespace {

// Backward.  With u = h r: dh = r (g - u mean(g u)) + gh, dw = sum over rows of gy u.  A workgroup goes through rows with a stride, the next row's three
// inputs on their way while this one's sums are waited for; it adds up dw of its rows, a lane its own channels, and writes one row of partial sums.
template <int W, int C>
constexpr bool dw_in_lds = C > 1;
template <int W, int C>
constexpr int dw_lds_bytes = dw_in_lds<W, C> ? W * C * 2048 : 0;

template <int W, int C>
__global__ __launch_bounds__(threads_of<W>) void k_add_rms_norm_backward(const NormBackwardArgs a) {
    constexpr bool LDS = dw_in_lds<W, C>;
    __shared__ float part[2][threads_of<W> / 64][2];
    extern __shared__ float shared[];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), sub = wave % W;
    const uint32_t chunk = chunk_of_lane(threadIdx.x & 63u), n = (uint32_t)(a.K / 8);
    uint32_t kc[C];
    bool in[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        kc[c] = (uint32_t)(c * W + sub) * 64u + chunk;
        in[c] = kc[c] < n;
        kc[c] = min(kc[c], n - 1);
    }
    // registers: one chunk a lane leaves room for the weight and all of the next row, more for neither, four not for gy either: asked for again, from the L2 (2048 x 20000
    // 413 -> 143 us, 333 x 32768 92 -> 45; h from there too 149, 47).  Four still do not fit the 128 registers that 1024 threads leave a lane: 42 are spilled to scratch
    // memory, 76 bytes a lane, and 2048 x 20000 takes 143 to 147 us for 57 that its 328 MB do (fp32 201 for 113).
    constexpr bool AHEAD = C == 1, KEEP = C <= 2;          // gy stays
    Raw<C> rh, rg, rd;
    auto fetch = [&](int64_t first) __attribute__((always_inline)) {
        const int64_t row = min(first + wave / W, a.M - 1);
        rh.load(a.h.p + row * a.h.pitch, a.h.bf16, kc);
        rg.load(a.gy.p + row * a.gy.pitch, a.gy.bf16, kc);
        if (a.gh.p) rd.load(a.gh.p + row * a.gh.pitch, a.gh.bf16, kc);
    };
    if constexpr (AHEAD) fetch((int64_t)blockIdx.x * rows_of<W>);
    float w[KEEP ? C : 1][8], dw[LDS ? 1 : C][8] = {};
    if constexpr (AHEAD)
        if (a.w) load_weight(a.w, kc, w);
    // LDS: where nothing else is left for them, this lane's sums lie there: 16 bytes of a lane next to its neighbours', halves apart
    float* const mine_lds = shared + threadIdx.x * 4;
    if constexpr (LDS) {
#pragma unroll
        for (int c = 0; c < 2 * C; ++c) *reinterpret_cast<v4f*>(mine_lds + c * (threads_of<W> * 4)) = v4f{0, 0, 0, 0};
    }
    const float inv = 1.0f / (float)a.K;
    int turn = 0;
    // (uniform over the workgroup: every thread meets every barrier of row_sums)
    for (int64_t first = (int64_t)blockIdx.x * rows_of<W>; first < a.M; first += (int64_t)gridDim.x * rows_of<W>) {
        const int64_t mine = first + wave / W, row = mine < a.M ? mine : a.M - 1;
        float h[C][8], g[KEEP ? C : 1][8], sums[2] = {0.0f, 0.0f};
        if constexpr (AHEAD) {
            rh.widen(a.h.bf16, h);
            rg.widen(a.gy.bf16, g);
        } else {
            renew(kc);
            load_row(a.h, row, kc, h);
            if constexpr (KEEP) load_row(a.gy, row, kc, g);
        }
        [[maybe_unused]] const Raw<C> other = rd;
        const int64_t next = first + (int64_t)gridDim.x * rows_of<W>;
        if (AHEAD && next < a.M) fetch(next);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float s = 0.0f, d = 0.0f;
            if constexpr (!AHEAD) __builtin_amdgcn_sched_barrier(0);
            if constexpr (!KEEP) load_one(a.gy.p + row * a.gy.pitch, a.gy.bf16, kc[c], g[0]);
            if (!AHEAD && a.w) load_chunk_weight(a.w, kc[c], w[KEEP ? c : 0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s = __builtin_fmaf(h[c][i], h[c][i], s);
                d = __builtin_fmaf(a.w ? g[KEEP ? c : 0][i] * w[KEEP ? c : 0][i] : g[KEEP ? c : 0][i], h[c][i], d);
            }
            sums[0] += in[c] ? s : 0.0f;
            sums[1] += in[c] ? d : 0.0f;
        }
        // (the sums' places alternate: the next row's are written while others still read these)
        row_sums<W, 2>(sums, part[turn], wave);
        turn ^= 1;
        if constexpr (!AHEAD) renew(kc);
        const float r = 1.0f / sqrtf(sums[0] * inv + a.eps), mean = sums[1] * r * inv;
        float d[C][8];
        if (AHEAD && a.gh.p) other.widen(a.gh.bf16, d);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (!AHEAD) __builtin_amdgcn_sched_barrier(0);
            if (!AHEAD && a.gh.p) load_one(a.gh.p + row * a.gh.pitch, a.gh.bf16, kc[c], d[c]);
            const bool live = in[c] && mine < a.M;
            float o[8], t[8];
            if (!AHEAD && a.w) {            // once more, from the L2, instead of a register each meanwhile
                asm volatile("" ::: "memory");
                load_chunk_weight(a.w, kc[c], w[KEEP ? c : 0]);
            }
            if constexpr (!KEEP) {
                asm volatile("" ::: "memory");
                load_one(a.gy.p + row * a.gy.pitch, a.gy.bf16, kc[c], g[0]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = h[c][i] * r, gi = g[KEEP ? c : 0][i];
                t[i] = live ? gi * u : 0.0f;
                o[i] = r * ((a.w ? gi * w[KEEP ? c : 0][i] : gi) - u * mean);
                if (a.gh.p) o[i] += d[c][i];
            }
            if (live) store_values(a.dh.p + row * a.dh.pitch, a.dh.bf16, kc[c], o);
            if (a.partial) {
                if constexpr (LDS) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        v4f* const at = reinterpret_cast<v4f*>(mine_lds + (2 * c + j) * (threads_of<W> * 4));
                        *at += v4f{t[4 * j], t[4 * j + 1], t[4 * j + 2], t[4 * j + 3]};
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) dw[c][i] += t[i];
                }
            }
        }
    }
    if (!a.partial) return;
    if constexpr (rows_of<W> == 1) {
        uint8_t* const to = reinterpret_cast<uint8_t*>(a.partial + (int64_t)blockIdx.x * a.K);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = LDS ? mine_lds[(2 * c + i / 4) * (threads_of<W> * 4) + i % 4] : dw[LDS ? 0 : c][i];
            if (in[c]) store_values(to, false, kc[c], t);
        }
    } else {
        __shared__ float sum[rows_of<W>][W * C * 512];
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (in[c]) store_values(reinterpret_cast<uint8_t*>(sum[wave / W]), false, kc[c], dw[c]);
        __syncthreads();
        for (int k = (int)threadIdx.x; k < (int)a.K; k += threads_of<W>) {
            float s = sum[0][k];
#pragma unroll
            for (int i = 1; i < rows_of<W>; ++i) s += sum[i][k];
            a.partial[(int64_t)blockIdx.x * a.K + k] = s;
        }
    }
}

// dw: the sums of the partial sums' columns, 16 columns a workgroup, 64 threads each.
__global__ __launch_bounds__(1024) void k_add_rms_norm_dw(const float* partial, int parts, int64_t K, float* dw) {
    __shared__ float sum[64][17];
    const int64_t k = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15u);
    const int p0 = (int)(threadIdx.x >> 4);
    float v = 0.0f;
#pragma unroll 4
    for (int p = p0; p < parts; p += 64) v += partial[(int64_t)p * K + k];
    sum[p0][threadIdx.x & 15u] = v;
    __syncthreads();
    if (threadIdx.x < 16) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) s += sum[i][threadIdx.x];
        dw[k] = s;
    }
}

}  // namespace

hipError_t setup_add_rms_norm() {
#define BRQ_SETUP(W, C)                                                                                                                     \
    if (dw_lds_bytes<W, C> > 0)                                                                                                             \
        if (hipError_t e = hipFuncSetAttribute((const void*)k_add_rms_norm_backward<W, C>, hipFuncAttributeMaxDynamicSharedMemorySize, dw_lds_bytes<W, C>); e != hipSuccess) return e
    BRQ_SETUP(16, 2);
    BRQ_SETUP(16, 4);
#undef BRQ_SETUP
    return hipSuccess;
}

// Workgroups of the backward pass, each of which writes a row of partial sums that is read again: 8 or 16 wavefronts a CU are enough for its loads, and a few
// hundred rows had better make half as many partial ones.  us, a workgroup a row up to twice as many -> now: 512 x 4096 12.9 -> 10.8, 1024 x 4096 16.0 -> 13.5,
// 2048 x 2048 16.3 -> 13.7, 4096 x 4096 33.6 -> 31.5; the same where fewer than 128 would be left (64 x 4096 6.2, with half of them 7.0).
int64_t norm_backward_parts(int64_t M, int64_t K) {
    const Split sp = split_of(K);
    const int64_t rows = sp.w < 4 ? 4 / sp.w : 1, n = (M + rows - 1) / rows, half = (n + 1) / 2, few = n < 128 ? n : 128, most = sp.w >= 8 ? 256 : 512;
    return half > most ? most : half > few ? half : few;
}

hipError_t launch_add_rms_norm_backward(const NormBackwardArgs& a, hipStream_t stream) {
    int cus = 0;
    if (hipError_t e = device_cus(&cus); e != hipSuccess) return e;      // (also the per-device kernel set-up)
    const int parts = (int)norm_backward_parts(a.M, a.K);
    if (a.M > 0) {
        const Split sp = split_of(a.K);
        switch (sp.w * 16 + sp.c) {
#define BRQ_BACK(W, C)                                                                                                                                     \
    case W * 16 + C:                                                                                                                                       \
        hipLaunchKernelGGL((k_add_rms_norm_backward<W, C>), dim3(parts), dim3(threads_of<W>), (dw_lds_bytes<W, C>), stream, a);                             \
        break;
            BRQ_BACK(1, 1) BRQ_BACK(2, 1) BRQ_BACK(4, 1) BRQ_BACK(8, 1) BRQ_BACK(16, 1) BRQ_BACK(16, 2) BRQ_BACK(16, 4)
#undef BRQ_BACK
            default: return hipErrorInvalidValue;
        }
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (!a.dw) return hipSuccess;
    hipLaunchKernelGGL(k_add_rms_norm_dw, dim3((uint32_t)(a.K / 16)), dim3(1024), 0, stream, a.partial, parts, a.K, a.dw);
    return hipGetLastError();
}

}  // namespace brq
