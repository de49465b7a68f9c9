// Attention over the MXFP4 cache (include/brq_attn.h).
#include "brq_attn.h"
#include "brq_device.h"
#include "brq_launch.h"

namespace brq {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

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

}  // namespace

int64_t kv4_attention_workspace(int64_t, int64_t, int, int, int, int64_t, int64_t, int) { return 0; }

hipError_t launch_kv4_attention(int D, const AttnArgs& a, hipStream_t stream) {
    const dim3 grid((uint32_t)((int64_t)a.S * a.max_q * a.Hk * a.G)), block(64);
    if (D == 64) hipLaunchKernelGGL((k_attention_rows<64>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((k_attention_rows<128>), grid, block, 0, stream, a);
    return hipGetLastError();
}

}  // namespace brq
