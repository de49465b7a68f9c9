// Attention over the MXFP4 cache (include/brq_attn.h).
//
// Scores on the block-scaled matrix instruction: a key is its 4-bit codes and E8M0 bytes as they stand in the cache, no
// instruction spent on unpacking; a bf16 query is the sum of two e4m3 terms of 4 significant bits each under one power of
// two (the second 2^-4 below the first), which costs what one bf16 product would (two 8-bit products at twice the rate)
// and is exact but for channels 2^-14 below the row's largest.  Values have a scale per token, which
// is the sum's axis, so they are unpacked to bf16 (exact) and multiplied by the softmax weights rounded to bf16.
// The products are made transposed, S^T = K Q^T and O^T = V^T P^T: a lane then holds one query row's scores for the very
// tokens that it has to supply to the second product, and one row's output, so that weights go from the first product's
// accumulators to the second's operand without leaving the lane and a row's rescaling is one factor a lane.
#include "brq_attn.h"
#include "brq_device.h"
#include "brq_launch.h"
#include "mfma_fp4.h"

namespace brq {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int v2i __attribute__((ext_vector_type(2)));

// Two 4-bit values, byte B of w, as bf16 under the exponent in bits 30:23 of `scale`.
template <int B>
__device__ __forceinline__ uint32_t two_values(uint32_t w, uint32_t scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, as_f32(scale), B));
}

// Range of query rows [q0, q1) of a sequence; empty where the offsets are none.
__device__ __forceinline__ void query_rows(const AttnArgs& a, int s, int64_t* q0, int* n) {
    int64_t b = s, e = (int64_t)s + 1;
    if (a.cu_q) {
        b = a.cu_q[s];
        e = a.cu_q[s + 1];
    }
    *q0 = b;
    *n = b < 0 || e > a.T || e <= b ? 0 : (int)min(e - b, (int64_t)a.max_q);
}

// The two e4m3 terms of 16 query channels, and what scales them.  `sign`: 0x8000 to negate.
struct Terms { v4i hi, lo; };
__device__ __forceinline__ Terms two_terms(const v4i (&w)[2], uint32_t byte, uint32_t sign) {
    const float s1 = as_f32(byte << 23), s2 = as_f32((byte - 4u) << 23);
    Terms t;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        typedef short v2s __attribute__((ext_vector_type(2)));
        v2s hi = {0, 0}, lo = {0, 0};
        const uint32_t a = (uint32_t)w[i >> 1][(i & 1) * 2] ^ (sign * 0x10001u), b = (uint32_t)w[i >> 1][(i & 1) * 2 + 1] ^ (sign * 0x10001u);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, bf16_lo(a), bf16_hi(a), s1, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, bf16_lo(b), bf16_hi(b), s1, true);
        const uint32_t h = __builtin_bit_cast(uint32_t, hi);
        const f32x2 ra = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, s1, false), rb = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, s1, true);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, bf16_lo(a) - ra.x, bf16_hi(a) - ra.y, s2, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, bf16_lo(b) - rb.x, bf16_hi(b) - rb.y, s2, true);
        t.hi[i] = (int)h;
        t.lo[i] = __builtin_bit_cast(int, lo);
    }
    return t;
}
// E8M0 byte under which a row whose largest channel is `top` lies in [128, 256): at least 4, so that the second term's exists.
__device__ __forceinline__ uint32_t terms_byte(float top) {
    const uint32_t e = (as_u32(top) >> 23) & 0xffu;
    return e < 11u ? 4u : e - 7u;
}
__device__ __forceinline__ float absmax_bf16(const v4i& w) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(bf16_lo((uint32_t)w[i])), fabsf(bf16_hi((uint32_t)w[i]))));
    return m;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---- up to 16 query rows (tokens x heads of a group) against a range of pages: decoding

// A page of one head as a lane takes it: 4 subtiles of 16 tokens.
template <int D>
struct PageRegs {
    v4i k[4];
    uint32_t ks;
    uint32_t v[4][D / 32];       // 4 tokens of the lane's column
    v4i vs;                      // byte i of element u: scale of token 16 u + 4 g + i
};

// Workgroup: sequence, cache head, split.  Wavefront w goes through pages first + w, first + w + 4, ...
template <int D>
__global__ __launch_bounds__(256, 2) void k_attention_few(const AttnArgs a, int splits, int pages_a_split, float* part_o, float* part_ml) {
    constexpr int MT = D / 16, HB = kv4_head_bytes(D);
    const int lane = (int)threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int split = (int)blockIdx.x % splits, sh = (int)blockIdx.x / splits, s = sh / a.Hk, kvh = sh - s * a.Hk;
    int64_t q0;
    int nq;
    query_rows(a, s, &q0, &nq);
    if (nq == 0) return;
    const int rows = nq * a.G, len = a.kv_lens[s], all = min(len, min(a.max_kv, a.table_cols * kKv4Page));
    // the tokens of this lane's row, and of any row
    const int tok = n < rows ? n / a.G : 0, head = kvh * a.G + (n < rows ? n - tok * a.G : 0), p = len - (a.cu_q ? (int)(a.cu_q[s + 1] - a.cu_q[s]) : 1) + tok;
    int end = all, begin = 0, end_any = all, begin_any = 0, end_all = all, begin_all = 0;
    if (a.causal) {
        const int p0 = p - tok, p1 = p0 + nq - 1;
        end = min(all, p + 1);
        end_any = min(all, p1 + 1);
        end_all = min(all, p0 + 1);
        if (a.window) {
            begin = max(0, p - a.window + 1);
            begin_any = max(0, p0 - a.window + 1);
            begin_all = max(0, p1 - a.window + 1);
        }
    }
    end_any = __builtin_amdgcn_readfirstlane(end_any);
    begin_any = __builtin_amdgcn_readfirstlane(begin_any);
    end_all = __builtin_amdgcn_readfirstlane(end_all);
    begin_all = __builtin_amdgcn_readfirstlane(begin_all);
    const int page0 = max(begin_any / kKv4Page, split * pages_a_split);
    const int page1 = min((max(end_any, 0) + kKv4Page - 1) / kKv4Page, (split + 1) * pages_a_split);

    // queries
    v8i qh, ql;
    uint32_t qs_hi, qs_lo;
    {
        const uint8_t* qp = a.q.p + (q0 + tok) * a.q.ts + head * a.q.hs;
        const uint32_t sign = a.scale < 0.0f ? 0x8000u : 0u;
        const v4i zero = {0, 0, 0, 0};
        v4i x[D / 64][2];
        float top = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 64; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v4i l = *reinterpret_cast<const v4i*>(qp + (k * 64 + g * 16 + i * 8) * 2);
                x[k][i] = n < rows ? l : zero;
                top = fmaxf(top, absmax_bf16(x[k][i]));
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const uint32_t byte = terms_byte(top);
        const Terms t0 = two_terms(x[0], byte, sign);
        if constexpr (D == 128) {
            const Terms t1 = two_terms(x[1], byte, sign);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qh[i] = t0.hi[i]; qh[i + 4] = t1.hi[i];
                ql[i] = t0.lo[i]; ql[i + 4] = t1.lo[i];
            }
            qs_hi = byte;
            qs_lo = byte - 4u;
        } else {                 // both terms are one operand: the second as channels 64 ... 127, against the same keys again
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qh[i] = t0.hi[i];
                qh[i + 4] = t0.lo[i];
            }
            qs_hi = g < 2 ? byte : byte - 4u;
        }
    }
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 1e-30f);

    v4f o[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) o[j] = v4f{0, 0, 0, 0};
    float l = 0.0f, ref = 0.0f, top_ref = -INFINITY;      // ref: what is subtracted; top_ref: the same, -inf before any token

    const int32_t* row = a.table + (int64_t)s * a.table_cols;
    auto load = [&](PageRegs<D>& r, int number) {
        const uint8_t* h = uniform_ptr(a.pool + ((int64_t)number * a.Hk + kvh) * HB);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            r.k[u] = *reinterpret_cast<const v4i*>(h + u * 8 * D + n * (D / 2) + (D == 128 ? g : g & 1) * 16);
        r.ks = *reinterpret_cast<const uint32_t*>(h + 32 * D + ((D == 128 ? g : g & 1) * 16 + n) * 4);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint8_t* vp = h + 34 * D + (u * 64 + lane) * (D / 8);
            if constexpr (D == 128) {
                const v4i x = *reinterpret_cast<const v4i*>(vp);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.v[u][i] = (uint32_t)x[i];
            } else {
                const v2i x = *reinterpret_cast<const v2i*>(vp);
                r.v[u][0] = (uint32_t)x[0];
                r.v[u][1] = (uint32_t)x[1];
            }
        }
        r.vs = *reinterpret_cast<const v4i*>(h + 66 * D + (g * (D / 32) + n * D / 512) * 16);
    };
    auto use = [&](PageRegs<D>& r, int page) {
        const int t0 = page * kKv4Page;
        v4f x[4];
        static_for([&](auto iu) {
            constexpr int u = decltype(iu)::value;
            v8i kk = {r.k[u].x, r.k[u].y, r.k[u].z, r.k[u].w, 0, 0, 0, 0};
            x[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kk, qh, v4f{0, 0, 0, 0}, 4, 0, u, (int)r.ks, 0, (int)qs_hi);
            if constexpr (D == 128) x[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kk, ql, x[u], 4, 0, u, (int)r.ks, 0, (int)qs_lo);
        }, IC<4>{});
        if (t0 < begin_all || t0 + kKv4Page > end_all) {               // some row does not see some token
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = t0 + u * 16 + g * 4 + i;
                    x[u][i] = t >= begin && t < end ? x[u][i] : -INFINITY;
                }
            if (t0 + kKv4Page > all) {                                 // tokens that are none: whatever their scales say, 0 times them is to be 0
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int left = all - (t0 + u * 16 + g * 4);
                    r.vs[u] = left <= 0 ? 0 : left >= 4 ? r.vs[u] : r.vs[u] & ((1 << (8 * left)) - 1);
                }
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 4; ++u) top = fmaxf(fmaxf(fmaxf(top, x[u][0]), fmaxf(x[u][1], x[u][2])), x[u][3]);
        top *= c;
        if (__any(top > top_ref + 8.0f)) {       // weights stay below 2^8 without a new reference
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(top, top_ref), f = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top_ref - now);
            top_ref = now;
            ref = now == -INFINITY ? 0.0f : now;
            l *= f;
#pragma unroll
            for (int j = 0; j < MT; ++j) o[j] *= f;
        }
        bf16x8 pw[2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][i], c, -ref));
            l += (e[0] + e[1]) + (e[2] + e[3]);
            const uint32_t w0 = pack_bf16x2(e[0], e[1]), w1 = pack_bf16x2(e[2], e[3]);
            v4i& d = reinterpret_cast<v4i&>(pw[u >> 1]);
            d[(u & 1) * 2] = (int)w0;
            d[(u & 1) * 2 + 1] = (int)w1;
        }
        static_for([&](auto ih) {                // tokens 32 h ... 32 h + 31: subtiles 2 h and 2 h + 1
            constexpr int h = decltype(ih)::value;
            uint32_t sc[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t b = (uint32_t)r.vs[2 * h + u];
                sc[u][0] = b << 23;
                sc[u][1] = b << 15;
                sc[u][2] = b << 7;
                sc[u][3] = b >> 1;
            }
            static_for([&](auto ib) {            // channels 2 b and 2 b + 1 of the lane's column
                constexpr int b = decltype(ib)::value;
                uint32_t y[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if constexpr (D == 128) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[u][i] = two_values<b>(r.v[2 * h + u][i], sc[u][i] & 0x7fffffffu);
                    } else {
                        y[u][0] = two_values<b>(r.v[2 * h + u][0], sc[u][0] & 0x7fffffffu);
                        y[u][1] = two_values<b + 2>(r.v[2 * h + u][0], sc[u][1] & 0x7fffffffu);
                        y[u][2] = two_values<b>(r.v[2 * h + u][1], sc[u][2] & 0x7fffffffu);
                        y[u][3] = two_values<b + 2>(r.v[2 * h + u][1], sc[u][3] & 0x7fffffffu);
                    }
                }
                v4i even, odd;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        even[u * 2 + i] = (int)__builtin_amdgcn_perm(y[u][2 * i + 1], y[u][2 * i], 0x05040100u);
                        odd[u * 2 + i] = (int)__builtin_amdgcn_perm(y[u][2 * i + 1], y[u][2 * i], 0x07060302u);
                    }
                o[2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pw[h], o[2 * b], 0, 0, 0);
                o[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pw[h], o[2 * b + 1], 0, 0, 0);
            }, IC<D / 32>{});
        }, IC<2>{});
    };

    // 64 page numbers at a time, one a lane; the next page's loads are under way while one is used
    for (int chunk = page0 + w; chunk < page1; chunk += 64 * 4) {
        const int mine = chunk + lane * 4, entry = mine < page1 ? row[mine] : -1;
        uint64_t left = __ballot(entry >= 0 && entry < a.num_pages);
        auto next = [&](int* page) {             // the next page that is one, or -1
            if (left == 0) return -1;
            const int i = __builtin_ctzll(left);
            left &= left - 1;
            *page = chunk + i * 4;
            return __builtin_amdgcn_readlane(entry, i);
        };
        PageRegs<D> ra, rb;
        int pa = 0, pb = 0, na = next(&pa), nb;
        if (na >= 0) load(ra, na);
        while (na >= 0) {
            nb = next(&pb);
            if (nb >= 0) load(rb, nb);
            use(ra, pa);
            if (nb < 0) break;
            na = next(&pa);
            if (na >= 0) load(ra, na);
            use(rb, pb);
        }
    }

    // the four wavefronts' sums, brought to one reference, added up
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __shared__ float so[4][16][D + 4], sm[4][16], sl[4][16];
    if (g == 0) {
        sm[w][n] = top_ref;
        sl[w][n] = l;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, sm[i][n]);
    const float f = top_ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top_ref - top);
    if (n < rows) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) so[w][n][(g * 4 + i) * MT + j] = o[j][i] * f;
    }
    __syncthreads();
    for (int e = (int)threadIdx.x; e < rows * (D / 4); e += 256) {
        const int r = e / (D / 4), d = (e - r * (D / 4)) * 4;
        v4f y = *reinterpret_cast<const v4f*>(&so[0][r][d]);
#pragma unroll
        for (int i = 1; i < 4; ++i) y += *reinterpret_cast<const v4f*>(&so[i][r][d]);
        float m = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, sm[i][r]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += sm[i][r] == -INFINITY ? 0.0f : sl[i][r] * __builtin_amdgcn_exp2f(sm[i][r] - m);
        const int tk = r / a.G;
        const int64_t t = q0 + tk, hq = kvh * a.G + (r - tk * a.G), at = t * (a.Hk * a.G) + hq;
        if (part_o) {
            *reinterpret_cast<v4f*>(part_o + (at * splits + split) * D + d) = y;
            if (d == 0) *reinterpret_cast<f32x2*>(part_ml + (at * splits + split) * 2) = f32x2{m, sum};
        } else {
            const float k = sum > 0.0f ? 1.0f / sum : 0.0f;
            *reinterpret_cast<v2i*>(a.o.p + t * a.o.ts + hq * a.o.hs + d * 2) = v2i{(int)pack_bf16x2(y.x * k, y.y * k), (int)pack_bf16x2(y.z * k, y.w * k)};
            if (a.lse && d == 0) a.lse[at] = sum > 0.0f ? (m + __log2f(sum)) * kLn2 : -INFINITY;
        }
    }
}

// Joins the splits of one row and head: groups of D/4 threads take every so many splits, then their sums are joined.
template <int D, int THREADS>
__global__ __launch_bounds__(THREADS) void k_attention_join(const AttnArgs a, int splits, const float* part_o, const float* part_ml) {
    constexpr int TH = D / 4, GROUPS = THREADS / TH;
    const int Hq = a.Hk * a.G, group = (int)threadIdx.x / TH, d = (int)(threadIdx.x % TH) * 4;
    const int64_t id = blockIdx.x, si = id / Hq;                            // (sequence, row, head)
    const int h = (int)(id - si * Hq), s = (int)(si / a.max_q), i = (int)(si - (int64_t)s * a.max_q);
    int64_t q0;
    int nq;
    query_rows(a, s, &q0, &nq);
    if (i >= nq) return;
    const int64_t t = q0 + i, at = t * Hq + h;
    const float *po = part_o + at * splits * D + d, *pm = part_ml + at * splits * 2;
    float m = -INFINITY, sum = 0.0f;
    v4f y = {0, 0, 0, 0};
#pragma unroll 4
    for (int k = group; k < splits; k += GROUPS) {
        const f32x2 ml = *reinterpret_cast<const f32x2*>(pm + k * 2);
        const v4f x = *reinterpret_cast<const v4f*>(po + (int64_t)k * D);
        const float now = fmaxf(m, ml.x), r = now == -INFINITY ? 0.0f : now;
        const float f0 = __builtin_amdgcn_exp2f(m - r), f1 = __builtin_amdgcn_exp2f(ml.x - r);
        y = y * f0 + x * f1;
        sum = sum * f0 + ml.y * f1;
        m = now;
    }
    __shared__ float so[GROUPS][D], sm[GROUPS], sl[GROUPS];
    *reinterpret_cast<v4f*>(&so[group][d]) = y;
    if (d == 0) {
        sm[group] = m;
        sl[group] = sum;
    }
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) m = fmaxf(m, sm[k]);
    const float r = m == -INFINITY ? 0.0f : m;
    y = v4f{0, 0, 0, 0};
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
        const float f = __builtin_amdgcn_exp2f(sm[k] - r);
        y += *reinterpret_cast<const v4f*>(&so[k][d]) * f;
        sum += sl[k] * f;
    }
    const float k = sum > 0.0f ? 1.0f / sum : 0.0f;
    *reinterpret_cast<v2i*>(a.o.p + t * a.o.ts + h * a.o.hs + d * 2) = v2i{(int)pack_bf16x2(y.x * k, y.y * k), (int)pack_bf16x2(y.z * k, y.w * k)};
    if (a.lse && d == 0) a.lse[at] = sum > 0.0f ? (m + __log2f(sum)) * kLn2 : -INFINITY;
}

// One wavefront: one query row and head.  A lane owns a token of the page for the scores, D/64 channels for the sum.
template <int D>
__global__ __launch_bounds__(64) void k_attention_rows(const AttnArgs a) {
    const int lane = (int)threadIdx.x, Hq = a.Hk * a.G;
    const int64_t id = blockIdx.x, si = id / Hq;
    const int h = (int)(id - si * Hq), s = (int)(si / a.max_q), i = (int)(si - (int64_t)s * a.max_q);
    int64_t q0 = s, q1 = s + 1;
    if (a.cu_q) {
        q0 = a.cu_q[s];
        q1 = a.cu_q[s + 1];
    }
    if (q0 < 0 || q1 > a.T || i >= q1 - q0) return;
    const int64_t t = q0 + i;
    const int len = a.kv_lens[s], p = len - (int)(q1 - q0) + i;
    int end = min(len, min(a.max_kv, a.table_cols * kKv4Page)), begin = 0;
    if (a.causal) {
        end = min(end, p + 1);
        if (a.window) begin = max(0, p - a.window + 1);
    }
    __shared__ float qs[D], ps[64];
    for (int d = lane; d < D; d += 64)
        qs[d] = bf16_lo(*reinterpret_cast<const uint16_t*>(a.q.p + t * a.q.ts + h * a.q.hs + d * 2));
    __syncthreads();
    constexpr int N = D / 64;
    float m = -INFINITY, l = 0.0f, o[N] = {};
    for (int page = begin / kKv4Page; page * kKv4Page < end; ++page) {
        const int number = a.table[(int64_t)s * a.table_cols + page];
        if (number < 0 || number >= a.num_pages) continue;
        const uint8_t* head = a.pool + ((int64_t)number * a.Hk + h / a.G) * kv4_head_bytes(D);
        const int j = page * kKv4Page + lane;
        float x = 0.0f;
        for (int c = 0; c < D / 8; ++c) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(head + kv4_key_code(D, lane) + c * 4);
            const float scale = as_f32((uint32_t)head[kv4_key_scale(D, lane, c >> 2)] << 23);
            const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
            const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
            const float* q = qs + c * 8;
            x += q[0] * v0.x + q[1] * v0.y + q[2] * v1.x + q[3] * v1.y + q[4] * v2.x + q[5] * v2.y + q[6] * v3.x + q[7] * v3.y;
        }
        x = j >= begin && j < end ? x * a.scale : -INFINITY;
        float mx = x;
        for (int k = 1; k < 64; k *= 2) mx = fmaxf(mx, __shfl_xor(mx, k));
        const float m2 = fmaxf(m, mx), f = expf(m - m2), e = expf(x - m2);       // (a page that is gone through has a token that is seen)
        float sum = e;
        for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
        l = l * f + sum;
        m = m2;
        ps[lane] = e;
        __syncthreads();
        for (int n = 0; n < N; ++n) o[n] *= f;
        const int channel = lane * N;                                           // N = 1: half of a byte
        for (int tok = 0; tok < kKv4Page; ++tok) {
            const int at = page * kKv4Page + tok;
            if (at < begin || at >= end) continue;
            const int byte = channel / 2;
            const uint32_t w = head[kv4_value_code(D, tok, byte / (D / 32)) + byte % (D / 32)];
            const float scale = as_f32((uint32_t)head[kv4_value_scale(D, tok, channel / 32)] << 23);
            const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
            if constexpr (N == 1) {
                o[0] += ps[tok] * ((channel & 1) ? v.y : v.x);
            } else {
                o[0] += ps[tok] * v.x;
                o[1] += ps[tok] * v.y;
            }
        }
        __syncthreads();
    }
    const float r = l > 0.0f ? 1.0f / l : 0.0f;
    for (int n = 0; n < N; ++n)
        *reinterpret_cast<uint16_t*>(a.o.p + t * a.o.ts + h * a.o.hs + (lane * N + n) * 2) = (uint16_t)f32_to_bf16_bits(o[n] * r);
    if (a.lse && lane == 0) a.lse[t * Hq + h] = l > 0.0f ? m + logf(l) : -INFINITY;
}

// How the pages are split: enough workgroups that each CU has several, none with less than two pages a wavefront.
#ifndef BRQ_WGS
#define BRQ_WGS 2
#endif
struct Splits { int n, pages; };
Splits splits_of(int64_t S, int Hk, int64_t max_kv, int cus) {
    const int64_t pages = (max_kv + kKv4Page - 1) / kKv4Page, groups = S * Hk;
    int64_t n = (cus * BRQ_WGS + groups - 1) / groups;
    n = n < (pages + 7) / 8 ? n : (pages + 7) / 8;
    n = n < 1 ? 1 : n > 256 ? 256 : n;
    const int64_t each = (pages + n - 1) / n;
    return {(int)(each ? (pages + each - 1) / each : 1), (int)(each ? each : 1)};
}
bool few_rows(int64_t max_q, int G) { return max_q * G <= 16; }

}  // namespace

int64_t kv4_attention_workspace(int64_t T, int64_t S, int Hq, int Hk, int D, int64_t max_q, int64_t max_kv, int cus) {
    if (!few_rows(max_q, Hq / Hk)) return 0;
    const Splits sp = splits_of(S, Hk, max_kv, cus);
    return sp.n == 1 ? 0 : T * Hq * sp.n * (D + 2) * 4;
}

template <int D>
static hipError_t launch_attention(const AttnArgs& a, int cus, hipStream_t stream) {
    const int Hq = a.Hk * a.G;
    if (few_rows(a.max_q, a.G)) {
        const Splits sp = splits_of(a.S, a.Hk, a.max_kv, cus);
        float *po = sp.n == 1 ? nullptr : static_cast<float*>(a.workspace), *pm = po ? po + a.T * Hq * sp.n * D : nullptr;
        hipLaunchKernelGGL((k_attention_few<D>), dim3((uint32_t)(a.S * a.Hk * sp.n)), dim3(256), 0, stream, a, sp.n, sp.pages, po, pm);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || !po) return e;
        const int64_t rows = (int64_t)a.S * a.max_q * Hq;
        if (sp.n <= 8) hipLaunchKernelGGL((k_attention_join<D, 64>), dim3((uint32_t)rows), dim3(64), 0, stream, a, sp.n, po, pm);
        else hipLaunchKernelGGL((k_attention_join<D, 256>), dim3((uint32_t)rows), dim3(256), 0, stream, a, sp.n, po, pm);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_attention_rows<D>), dim3((uint32_t)((int64_t)a.S * a.max_q * Hq)), dim3(64), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_kv4_attention(int D, const AttnArgs& a, hipStream_t stream) {
    int cus = 0;
    if (hipError_t e = device_cus(&cus); e != hipSuccess) return e;
    return D == 64 ? launch_attention<64>(a, cus, stream) : launch_attention<128>(a, cus, stream);
}

}  // namespace brq
