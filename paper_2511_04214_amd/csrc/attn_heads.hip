// Passes over query, key and value heads: RMS norm, rotation by position and block rotation in one pass, its backward
// pass, the same in front of the MXFP4 quantizer that writes the cache, and the cache's values read back.
//
// A head of D channels is held by L = D/8 lanes, 8 channels each; a wavefront holds 64/L heads.  The lanes hold the
// chunks in the order of chunk_of_lane (brq_device.h), in which both the block rotation's wide stages and the
// partner of a rotation by position over the whole head are DPP reads of the mirror image.
#include "brq_attn.h"
#include "brq_device.h"
#include "brq_launch.h"
#include "mfma_fp4.h"

namespace brq {
namespace {

// Lane of a head's lanes that holds chunk c: the inverse of chunk_of_lane.
__device__ __forceinline__ uint32_t lane_of_chunk(uint32_t c) {
    const uint32_t b2 = ((c >> 2) ^ (c >> 3)) & 1u;
    return (c & 24u) | (b2 << 2) | ((c & 3u) ^ (b2 ? 3u : 0u));
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror16 = 0x140, kMirror8 = 0x141;

// Sum over the L lanes of a head, every lane receiving it.
template <int L>
__device__ __forceinline__ float head_sum(float v) {
    v += dpp<kXor1>(v);
    v += dpp<kXor2>(v);
    v += dpp<kMirror8>(v);
    if constexpr (L >= 16) v += dpp<kMirror16>(v);
    if constexpr (L >= 32) v += __shfl_xor(v, 16);
    return v;
}

// H_B / sqrt(B) on each B channels of the head; 2^l2b <= 8 L.
template <int L>
__device__ __forceinline__ void rotate_block(float (&v)[8], int l2b, uint32_t chunk) {
    float s = 1.0f;
    switch (l2b) {
        case 0: return;
        case 3: wht_inwave<3>(v, chunk); s = wht_sign<3>(chunk) * 0.35355339059327373f; break;
        case 4: wht_inwave<4>(v, chunk); s = wht_sign<4>(chunk) * 0.25f; break;
        case 5: wht_inwave<5>(v, chunk); s = wht_sign<5>(chunk) * 0.17677669529663687f; break;
        case 6: wht_inwave<6>(v, chunk); s = wht_sign<6>(chunk) * 0.125f; break;
        case 7: if constexpr (L >= 16) { wht_inwave<7>(v, chunk); s = wht_sign<7>(chunk) * 0.08838834764831843f; } break;
        case 8: if constexpr (L >= 32) { wht_inwave<8>(v, chunk); s = wht_sign<8>(chunk) * 0.0625f; } break;
        default: break;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
}

// The rotation of one token as a lane needs it: y = c v + s partner.
struct Turn {
    float c[8], s[8];
    __device__ __forceinline__ void load(const Rope& r, int64_t row, uint32_t chunk, bool back) {
        const int half = r.rot >> 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
        if ((int)chunk * 8 >= r.rot) return;
        if (r.interleaved) {
            const v4f cc = *reinterpret_cast<const v4f*>(r.cos + row * half + chunk * 4);
            const v4f ss = *reinterpret_cast<const v4f*>(r.sin + row * half + chunk * 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = cc[i >> 1];
                s[i] = ((i & 1) != 0) != back ? ss[i >> 1] : -ss[i >> 1];
            }
        } else {
            const bool second = (int)chunk * 8 >= half;
            const int64_t at = row * half + (second ? (int)chunk * 8 - half : (int)chunk * 8);
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                const v4f cc = *reinterpret_cast<const v4f*>(r.cos + at + j), ss = *reinterpret_cast<const v4f*>(r.sin + at + j);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    c[j + i] = cc[i];
                    s[j + i] = second != back ? ss[i] : -ss[i];
                }
            }
        }
    }
    template <int L>
    __device__ __forceinline__ void apply(float (&v)[8], const Rope& r, uint32_t lane, uint32_t chunk) const {
        float p[8];
        if (r.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = v[i ^ 1];
        } else if (L <= 16 && r.rot == L * 8) {      // the whole head: the partner is the mirror image
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = L == 16 ? dpp<kMirror16>(v[i]) : dpp<kMirror8>(v[i]);
        } else {
            const int n = r.rot >> 4;                // chunks of a half
            const int other = (int)chunk < n ? (int)chunk + n : (int)chunk < 2 * n ? (int)chunk - n : (int)chunk;
            const int src = (int)((lane & ~(uint32_t)(L - 1)) | lane_of_chunk((uint32_t)other));
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = __shfl(v[i], src);
        }
        if (r.rot < L * 8) {                         // channels behind the rotated ones stay as they are: 0 times an infinity is not 0
            const bool turned = (int)chunk * 8 < r.rot;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = turned ? __builtin_fmaf(p[i], s[i], v[i] * c[i]) : v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(p[i], s[i], v[i] * c[i]);
        }
    }
};

// STREAM: past the caches.  For the outputs of the forward and backward pass (8192 tokens, 168 MB of them: 97.2 -> 91.2 us one call after
// the other, 101 -> 104 alone), not for queries on their way to attention (a step of 16 sequences 17.25 -> 17.45).
template <bool STREAM, class T>
__device__ __forceinline__ void store16(uint8_t* p, T x) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<T*>(p));
    else *reinterpret_cast<T*>(p) = x;
}
template <bool BF16, bool STREAM>
__device__ __forceinline__ void store_chunk(uint8_t* p, const float (&v)[8]) {
    if constexpr (BF16) {
        store16<STREAM>(p, v4i{(int)pack_bf16x2(v[0], v[1]), (int)pack_bf16x2(v[2], v[3]), (int)pack_bf16x2(v[4], v[5]), (int)pack_bf16x2(v[6], v[7])});
    } else {
        store16<STREAM>(p, v4f{v[0], v[1], v[2], v[3]});
        store16<STREAM>(p + 16, v4f{v[4], v[5], v[6], v[7]});
    }
}

__device__ __forceinline__ void load_weight(const float* w, uint32_t chunk, float (&v)[8]) {
    typedef float quad __attribute__((ext_vector_type(4), aligned(4)));          // (weights are aligned to 4 bytes, no more)
    if (w) {
        const quad a = *reinterpret_cast<const quad*>(w + chunk * 8), b = *reinterpret_cast<const quad*>(w + chunk * 8 + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    }
}

__device__ __forceinline__ float sum_squares(const float (&v)[8]) {
    float a = v[0] * v[0], b = v[1] * v[1];
#pragma unroll
    for (int i = 2; i < 8; i += 2) {
        a = __builtin_fmaf(v[i], v[i], a);
        b = __builtin_fmaf(v[i + 1], v[i + 1], b);
    }
    return a + b;
}

// A lane's place in a wavefront's 64/L heads, and its walk over groups of that many heads of one token.
template <int L>
struct Walk {
    const uint8_t* p;
    int64_t step;
    int h, n;                            // the lane's head, the number of heads
    __device__ __forceinline__ Walk(const Heads& x, int64_t t, int group, uint32_t lane, uint32_t byte)
        : p(x.p + t * x.ts + group * (64 / L) * x.hs + (int64_t)(lane / L) * x.hs + byte), step(x.hs * (64 / L)), h(group * (64 / L) + (int)(lane / L)), n(x.n) {}
    __device__ __forceinline__ bool there() const { return h < n; }
    // where to read: the last groups' lanes without a head read the first lane's, which there is
    __device__ __forceinline__ const uint8_t* read(int64_t hs, uint32_t lane) const { return there() ? p : p - (int64_t)(lane / L) * hs; }
    __device__ __forceinline__ void next() {
        p += step;
        h += 64 / L;
    }
};
enum Kind { kQuery, kKey, kValue };

// One wavefront: token t, `each` groups of 64/L heads from part * each on; groups are queries first, then keys, then values.
// Everything but the lane's place is uniform and stays in scalar registers; the next group's load is under way while one is
// worked on.
template <int L, bool IN_BF16, bool OUT_BF16, bool APPEND>
__global__ __launch_bounds__(256) void k_heads(const HeadsArgs a, int splits, int each) {
    constexpr int D = L * 8, HPW = 64 / L, ES = IN_BF16 ? 2 : 4, OS = OUT_BF16 ? 2 : 4;
    const uint32_t lane = threadIdx.x & 63u, l = lane & (L - 1), chunk = chunk_of_lane(l);
    const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t = wave / splits;
    const int part = (int)(wave - t * splits);
    if (t >= a.T) return;
    const int nq = (a.q.n + HPW - 1) / HPW, nk = (a.k.n + HPW - 1) / HPW, nv = APPEND ? (a.v.n + HPW - 1) / HPW : 0;
    const int begin = part * each, end = min(begin + each, nq + nk + nv);
    bool placed = true;
    Turn turn;
    if (a.rope.rot && begin < nq + nk) {
        const int64_t row = a.rope.pos[t];
        placed = row >= 0 && row < a.rope.rows;
        turn.load(a.rope, placed ? row : 0, chunk, false);
    }
    int64_t slot = -1;
    if constexpr (APPEND) {
        slot = a.slots[t];
        if (a.rope.rot && begin >= nq + nk) placed = a.rope.pos[t] >= 0 && a.rope.pos[t] < a.rope.rows;
    }
    const bool write = placed && slot >= 0 && slot < a.num_slots;
    const int in_page = (int)(slot & (kKv4Page - 1));

    auto segment = [&](auto kind, const Heads& src, const Heads& dst, const float* weight, int l2b, int g0, int g1) {
        constexpr int K = decltype(kind)::value;
        if (g0 >= g1) return;
        constexpr bool STORE = !APPEND || K == kQuery;
        Walk<L> in(src, t, g0, lane, chunk * 8 * ES), out(STORE ? dst : Heads{a.pool, 0, kv4_head_bytes(D), src.n}, STORE ? t : 0, g0, lane, STORE ? chunk * 8 * OS : 0);
        if constexpr (!STORE) out.p += write ? slot / kKv4Page * a.Hk * kv4_head_bytes(D) : 0;
        float w[8];
        if (K != kValue && weight) load_weight(weight, chunk, w);
        RawChunk<IN_BF16> raw = load_raw<IN_BF16>(in.read(src.hs, lane));
        for (int it = g0; it < g1; ++it) {
            float v[8];
            widen<IN_BF16>(raw, v);
            in.next();
            if (it + 1 < g1) raw = load_raw<IN_BF16>(in.read(src.hs, lane));
            if constexpr (K != kValue) {
                // (the hardware's reciprocal root, a bit of 24 off at most: outputs of 32 bits are 1 to 1.3 times as far off as a plain form's)
                if (weight) {
                    const float r = __builtin_amdgcn_rsqf(head_sum<L>(sum_squares(v)) * (1.0f / D) + a.eps);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = v[i] * r * w[i];
                }
                if (a.rope.rot) turn.apply<L>(v, a.rope, lane, chunk);
            }
            rotate_block<L>(v, l2b, chunk);
            uint8_t* to = const_cast<uint8_t*>(out.p);
            if constexpr (STORE) {
                if (!placed) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = as_f32(0x7fc00000u);
                }
                if (out.there()) store_chunk<OUT_BF16, !APPEND>(to, v);
            } else {
                uint32_t sb = e8m0_from_amax(quad_max(absmax8(v)));
                // 6 * 2^(252 - 127) is a number in 32 bits and in bf16; under 253, the scale of an infinity, 6 would become one, and 0 times
                // it NaN in the rows that do not see the token
                if constexpr (K == kValue) sb = min(sb, 252u);
                const uint32_t codes = encode8_e2m1(v, sb);
                if (write && out.there()) {
                    if constexpr (K == kKey) {
                        *reinterpret_cast<uint32_t*>(to + kv4_key_code(D, in_page) + chunk * 4) = codes;
                        if ((l & 3u) == 0) to[kv4_key_scale(D, in_page, (int)(chunk >> 2))] = (uint8_t)sb;
                    } else {
                        if constexpr (D == 128) {
                            *reinterpret_cast<uint32_t*>(to + kv4_value_code(D, in_page, (int)chunk)) = codes;
                        } else {
                            *reinterpret_cast<uint16_t*>(to + kv4_value_code(D, in_page, (int)chunk * 2)) = (uint16_t)codes;
                            *reinterpret_cast<uint16_t*>(to + kv4_value_code(D, in_page, (int)chunk * 2 + 1)) = (uint16_t)(codes >> 16);
                        }
                        if ((l & 3u) == 0) to[kv4_value_scale(D, in_page, (int)(chunk >> 2))] = (uint8_t)sb;
                    }
                }
            }
            out.next();
        }
    };
    segment(IC<kQuery>{}, a.q, a.qo, a.wq, a.l2b, begin, min(end, nq));
    segment(IC<kKey>{}, a.k, a.ko, a.wk, a.l2b, max(begin - nq, 0), min(end - nq, nk));
    if constexpr (APPEND) segment(IC<kValue>{}, a.v, a.ko, nullptr, a.l2bv, max(begin - nq - nk, 0), end - nq - nk);
}

// Wavefronts of a launch: as many to a token as make about 8 for every SIMD together, at most one for each group of heads.
int token_splits(int64_t T, int groups) {
    const int64_t want = (8192 + T - 1) / T;
    return (int)(want < groups ? want : groups);
}

}  // namespace

hipError_t launch_heads(int D, bool in_bf16, bool out_bf16, bool append, const HeadsArgs& a, hipStream_t stream) {
    const int hpw = 512 / D;
    const int groups = (a.q.n + hpw - 1) / hpw + (a.k.n + hpw - 1) / hpw + (append ? (a.v.n + hpw - 1) / hpw : 0);
    const int each = (groups + token_splits(a.T, groups) - 1) / token_splits(a.T, groups), splits = (groups + each - 1) / each;
    const dim3 grid((uint32_t)((a.T * splits + 3) / 4)), block(256);
#define BRQ_HEADS(L_, IN, OUT, APP) hipLaunchKernelGGL((k_heads<L_, IN, OUT, APP>), grid, block, 0, stream, a, splits, each)
#define BRQ_HEADS_T(L_)                                                        \
    do {                                                                       \
        if (in_bf16 && out_bf16) BRQ_HEADS(L_, true, true, false);             \
        else if (in_bf16) BRQ_HEADS(L_, true, false, false);                   \
        else if (out_bf16) BRQ_HEADS(L_, false, true, false);                  \
        else BRQ_HEADS(L_, false, false, false);                               \
    } while (0)
    if (append) {
        if (D == 64) { if (in_bf16) BRQ_HEADS(8, true, true, true); else BRQ_HEADS(8, false, false, true); }
        else { if (in_bf16) BRQ_HEADS(16, true, true, true); else BRQ_HEADS(16, false, false, true); }
    } else if (D == 64) BRQ_HEADS_T(8);
    else if (D == 128) BRQ_HEADS_T(16);
    else BRQ_HEADS_T(32);
#undef BRQ_HEADS_T
#undef BRQ_HEADS
    return hipGetLastError();
}

namespace {

// Backward.  A wavefront goes through (token, part) items with a stride and keeps both weights' gradients for its
// lanes' channels in registers; a workgroup adds its wavefronts' up in LDS and writes one row of partial sums.
template <int L, bool X_BF16, bool G_BF16>
__global__ __launch_bounds__(256, 3) void k_heads_backward(const HeadsArgs a, int splits, int each) {
    constexpr int D = L * 8, HPW = 64 / L, ES = X_BF16 ? 2 : 4, GS = G_BF16 ? 2 : 4;
    const uint32_t lane = threadIdx.x & 63u, l = lane & (L - 1), chunk = chunk_of_lane(l);
    const int nq = (a.q.n + HPW - 1) / HPW, nk = (a.k.n + HPW - 1) / HPW;
    float dw[2][8] = {};
    const int64_t items = a.T * splits;
    for (int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); item < items; item += (int64_t)gridDim.x * 4) {
        const int64_t t = item / splits;
        const int part = (int)(item - t * splits);
        Turn turn;
        bool placed = true;
        if (a.rope.rot) {
            const int64_t row = a.rope.pos[t];
            placed = row >= 0 && row < a.rope.rows;
            turn.load(a.rope, placed ? row : 0, chunk, true);
        }
        const int begin = part * each, end = min(begin + each, nq + nk);
        auto segment = [&](auto kind, const Heads& src, const Heads& grad, const Heads& dst, const float* weight, int g0, int g1) {
            constexpr int K = decltype(kind)::value;
            if (g0 >= g1) return;
            Walk<L> in(src, t, g0, lane, chunk * 8 * ES), gr(grad, t, g0, lane, chunk * 8 * GS), out(dst, t, g0, lane, chunk * 8 * ES);
            float w[8];
            if (weight) load_weight(weight, chunk, w);
            RawChunk<G_BF16> rg = load_raw<G_BF16>(gr.read(grad.hs, lane));
            RawChunk<X_BF16> rx = {};
            if (weight) rx = load_raw<X_BF16>(in.read(src.hs, lane));
            for (int it = g0; it < g1; ++it) {
                float g[8], x[8];
                widen<G_BF16>(rg, g);
                widen<X_BF16>(rx, x);
                in.next();
                gr.next();
                if (it + 1 < g1) {
                    rg = load_raw<G_BF16>(gr.read(grad.hs, lane));
                    if (weight) rx = load_raw<X_BF16>(in.read(src.hs, lane));
                }
                rotate_block<L>(g, a.l2b, chunk);
                if (a.rope.rot) turn.apply<L>(g, a.rope, lane, chunk);
                if (!placed) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = as_f32(0x7fc00000u);
                }
                if (weight) {
                    float y[8];
                    const float r = __builtin_amdgcn_rsqf(head_sum<L>(sum_squares(x)) * (1.0f / D) + a.eps);
                    float dot = 0.0f;
                    const bool mine = out.there();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] *= r;                                            // u = x / rms
                        y[i] = g[i] * w[i];
                        dot = __builtin_fmaf(y[i], x[i], dot);
                        dw[K][i] += mine ? g[i] * x[i] : 0.0f;
                    }
                    const float mean = head_sum<L>(dot) * (1.0f / D);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = r * (y[i] - x[i] * mean);
                }
                if (out.there()) store_chunk<X_BF16, true>(const_cast<uint8_t*>(out.p), g);
                out.next();
            }
        };
        segment(IC<kQuery>{}, a.q, a.gq, a.qo, a.wq, begin, min(end, nq));
        segment(IC<kKey>{}, a.k, a.gk, a.ko, a.wk, max(begin - nq, 0), end - nq);
    }
    if (!a.partial) return;
    __shared__ float sum[4][2][D];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = dw[n][i];
#pragma unroll
            for (int m = L; m < 64; m *= 2) v += __shfl_xor(v, m);
            if (lane < (uint32_t)L) sum[threadIdx.x >> 6][n][chunk * 8 + i] = v;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * D; c += 256) {
        const float* s = &sum[0][0][0] + c;
        a.partial[(int64_t)blockIdx.x * (2 * D) + c] = (s[0] + s[2 * D]) + (s[4 * D] + s[6 * D]);
    }
}

// Sums of the partial sums' columns: 16 columns a workgroup, 64 threads each.
__global__ __launch_bounds__(1024) void k_heads_weight_grads(const float* partial, int rows, int D, float* dwq, float* dwk) {
    __shared__ float sum[64][17];
    const int c = (int)blockIdx.x * 16 + (int)(threadIdx.x & 15u), r0 = (int)(threadIdx.x >> 4);
    float v = 0.0f;
#pragma unroll 4
    for (int r = r0; r < rows; r += 64) v += partial[(int64_t)r * (2 * D) + c];
    sum[r0][threadIdx.x & 15u] = v;
    __syncthreads();
    if (threadIdx.x < 16) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) s += sum[i][threadIdx.x];
        float* out = c < D ? dwq : dwk;
        if (out) out[c < D ? c : c - D] = s;
    }
}

}  // namespace

int64_t heads_backward_workgroups(int64_t T, int Hq, int Hk, int D) {
    const int hpw = 512 / D, groups = (Hq + hpw - 1) / hpw + (Hk + hpw - 1) / hpw;
    const int64_t n = (T * token_splits(T, groups) + 3) / 4;
    return n < 768 ? n : 768;                        // three to a CU, as many as its registers hold
}

hipError_t launch_heads_backward(int D, bool x_bf16, bool g_bf16, const HeadsArgs& a, hipStream_t stream) {
    const int hpw = 512 / D, groups = (a.q.n + hpw - 1) / hpw + (a.k.n + hpw - 1) / hpw;
    const int each = (groups + token_splits(a.T, groups) - 1) / token_splits(a.T, groups), splits = (groups + each - 1) / each;
    const int wgs = (int)heads_backward_workgroups(a.T, a.q.n, a.k.n, D);
#define BRQ_BACK(L_, X, G) hipLaunchKernelGGL((k_heads_backward<L_, X, G>), dim3(wgs), dim3(256), 0, stream, a, splits, each)
#define BRQ_BACK_T(L_)                                          \
    do {                                                        \
        if (x_bf16 && g_bf16) BRQ_BACK(L_, true, true);         \
        else if (x_bf16) BRQ_BACK(L_, true, false);             \
        else if (g_bf16) BRQ_BACK(L_, false, true);             \
        else BRQ_BACK(L_, false, false);                        \
    } while (0)
    if (D == 64) BRQ_BACK_T(8);
    else if (D == 128) BRQ_BACK_T(16);
    else BRQ_BACK_T(32);
#undef BRQ_BACK_T
#undef BRQ_BACK
    if (hipError_t e = hipGetLastError(); e != hipSuccess || !a.partial) return e;
    return launch_heads_weight_grads(a.partial, wgs, D, a.dwq, a.dwk, stream);
}

hipError_t launch_heads_weight_grads(const float* partial, int rows, int D, float* dwq, float* dwk, hipStream_t stream) {
    hipLaunchKernelGGL(k_heads_weight_grads, dim3(2 * D / 16), dim3(1024), 0, stream, partial, rows, D, dwq, dwk);
    return hipGetLastError();
}

namespace {

// A thread reads back 8 channels of keys and of values of one token and head.
template <int D, bool OUT_BF16>
__global__ __launch_bounds__(256) void k_kv4_read(const uint8_t* pool, int64_t num_slots, int Hk, int64_t T, const int64_t* slots, Heads k, Heads v) {
    constexpr int L = D / 8, OS = OUT_BF16 ? 2 : 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, th = i / L, t = th / Hk;
    const int chunk = (int)(i % L), h = (int)(th - t * Hk);
    if (t >= T) return;
    const int64_t slot = slots[t];
    float x[2][8];
    if (slot >= 0 && slot < num_slots) {
        const int p = (int)(slot & (kKv4Page - 1));
        const uint8_t* head = pool + ((slot / kKv4Page) * Hk + h) * kv4_head_bytes(D);
        uint32_t c[2], s[2];
        c[0] = *reinterpret_cast<const uint32_t*>(head + kv4_key_code(D, p) + chunk * 4);
        s[0] = head[kv4_key_scale(D, p, chunk >> 2)];
        if constexpr (D == 128) {
            c[1] = *reinterpret_cast<const uint32_t*>(head + kv4_value_code(D, p, chunk));
        } else {
            c[1] = *reinterpret_cast<const uint16_t*>(head + kv4_value_code(D, p, chunk * 2)) |
                   (uint32_t)*reinterpret_cast<const uint16_t*>(head + kv4_value_code(D, p, chunk * 2 + 1)) << 16;
        }
        s[1] = head[kv4_value_scale(D, p, chunk >> 2)];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const float scale = as_f32(s[n] << 23);
            typedef float f2 __attribute__((ext_vector_type(2)));
            const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[n], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[n], scale, 1);
            const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[n], scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[n], scale, 3);
            x[n][0] = a.x; x[n][1] = a.y; x[n][2] = b.x; x[n][3] = b.y;
            x[n][4] = d.x; x[n][5] = d.y; x[n][6] = e.x; x[n][7] = e.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j >> 3][j & 7] = as_f32(0x7fc00000u);
    }
    store_chunk<OUT_BF16, false>(k.p + t * k.ts + h * k.hs + chunk * 8 * OS, x[0]);
    store_chunk<OUT_BF16, false>(v.p + t * v.ts + h * v.hs + chunk * 8 * OS, x[1]);
}

}  // namespace

hipError_t launch_kv4_read(int D, const uint8_t* pool, int64_t num_slots, int Hk, int64_t T, const int64_t* slots, const Heads& k,
                           const Heads& v, bool out_bf16, hipStream_t stream) {
    const dim3 grid((uint32_t)((T * Hk * (D / 8) + 255) / 256)), block(256);
#define BRQ_READ(D_, OUT) hipLaunchKernelGGL((k_kv4_read<D_, OUT>), grid, block, 0, stream, pool, num_slots, Hk, T, slots, k, v)
    if (D == 64) { if (out_bf16) BRQ_READ(64, true); else BRQ_READ(64, false); }
    else { if (out_bf16) BRQ_READ(128, true); else BRQ_READ(128, false); }
#undef BRQ_READ
    return hipGetLastError();
}

}  // namespace brq
