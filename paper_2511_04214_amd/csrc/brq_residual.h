// What the residual side's translation units share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace brq {

// Rows of a matrix at p, `pitch` bytes apart.
struct RowSet {
    uint8_t* p;
    int64_t pitch;
    bool bf16;
};

// The norm with the residual's addition in front of it, alone or in front of the online step.
struct NormArgs {
    RowSet x, res, h, y;        // p null: not there (res, h; y in front of the online step, whose y.bf16 then rounds it on its way)
    const float* w;             // [K] or null
    float eps;
    int64_t M, K;
    // the online step
    uint8_t *codes, *scales;
    bool tiled;
    int l2b;                    // log2 of the rotation block, 0: none
    const int8_t* signs;        // [K] or null
};
constexpr int64_t NORM_MAX_K = 32768;
hipError_t launch_add_rms_norm(const NormArgs& a, bool quantize, hipStream_t s);

struct NormBackwardArgs {
    RowSet h, gy, gh, dh;       // gh.p null: no other gradient
    const float* w;             // [K] or null
    float eps;
    int64_t M, K;
    float* partial;             // [norm_backward_parts][K] or null
    float* dw;                  // [K] or null
};
int64_t norm_backward_parts(int64_t M, int64_t K);
hipError_t launch_add_rms_norm_backward(const NormBackwardArgs& a, hipStream_t s);

}  // namespace brq
