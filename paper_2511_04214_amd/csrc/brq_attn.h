// What the attention side's translation units share: views of heads, the cache's layout, launch entry points.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace brq {

// x[t][h][d] at p + t * ts + h * hs bytes; D contiguous.
struct Heads {
    uint8_t* p;
    int64_t ts, hs;
    int n;
};

// Rotation by position; rot = 0: none.
struct Rope {
    const float *cos, *sin;
    const int64_t* pos;
    int64_t rows;
    int rot, interleaved;
};

// Everything of the passes over heads.
struct HeadsArgs {
    Heads q, k, v;              // n = 0: not there
    Heads qo, ko;               // outputs of q and k (forward), of their gradients (backward)
    Heads gq, gk;               // backward: gradients of the outputs
    const float *wq, *wk;       // [D] or null
    float eps;
    Rope rope;
    int64_t T;
    int l2b, l2bv;              // log2 of the rotation blocks, 0: none
    // append
    const int64_t* slots;
    uint8_t* pool;
    int64_t num_slots;
    int Hk;
    // backward
    float* partial;             // [workgroups][2][D] or null
    float *dwq, *dwk;           // [D] or null
};

// ---- a page of the cache (include/brq_attn.h): bytes from a head's start
constexpr int kKv4Page = 64;
__host__ __device__ constexpr int kv4_head_bytes(int D) { return 68 * D; }
__device__ __forceinline__ int kv4_key_code(int D, int t) { return t * (D / 2); }
__device__ __forceinline__ int kv4_key_scale(int D, int t, int n) { return 32 * D + (n * 16 + (t & 15)) * 4 + (t >> 4); }
// of 16 columns of D/32 code bytes (D/16 channels)
__device__ __forceinline__ int kv4_value_code(int D, int t, int column) { return 34 * D + (((t >> 2) * 16 + column) * 4 + (t & 3)) * (D / 32); }
__device__ __forceinline__ int kv4_value_scale(int D, int t, int n) { return 66 * D + (((t >> 2 & 3) * (D / 32) + n) * 4 + (t >> 4)) * 4 + (t & 3); }

hipError_t launch_heads(int D, bool in_bf16, bool out_bf16, bool append, const HeadsArgs& a, hipStream_t stream);
hipError_t launch_heads_backward(int D, bool x_bf16, bool g_bf16, const HeadsArgs& a, hipStream_t stream);
hipError_t launch_heads_weight_grads(const float* partial, int rows, int D, float* dwq, float* dwk, hipStream_t stream);
int64_t heads_backward_workgroups(int64_t T, int Hq, int Hk, int D);
hipError_t launch_kv4_read(int D, const uint8_t* pool, int64_t num_slots, int Hk, int64_t T, const int64_t* slots, const Heads& k,
                           const Heads& v, bool out_bf16, hipStream_t stream);

struct AttnArgs {
    Heads q, o;
    int64_t T;
    const uint8_t* pool;
    int64_t num_pages;
    int Hk, G;                  // heads in the cache, query heads to each
    const int32_t *table, *kv_lens, *cu_q;
    int table_cols, S;
    float scale;
    int causal, window, max_q, max_kv;
    float* lse;                 // [T][Hk * G] or null
    void* workspace;
};
hipError_t launch_kv4_attention(int D, const AttnArgs& a, hipStream_t stream);
int64_t kv4_attention_workspace(int64_t T, int64_t S, int Hq, int Hk, int D, int64_t max_q, int64_t max_kv, int cus);

struct PagesArgs {
    uint8_t* pool;
    int64_t page_bytes;
    int num_pages;
    int32_t* table;
    int S, cols;
    int32_t *lens, *refs;
    const int32_t *a, *b;       // the call's lists
    int n;
    int32_t* result;            // failed / live
    int32_t* workspace;
};
hipError_t launch_pages_copy(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream);

}  // namespace brq
