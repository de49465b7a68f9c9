// Drives the host side of the attention calls (include/brq_attn.h) at the ends of their arguments' ranges, with launches that do
// nothing: what is refused, what reaches a launch, and that no check overflows on its way (the sanitizers' part).
#include <cstdio>
#include <cstdlib>

#include "../../include/brq_attn.h"
#include "../../paper_2511_04214_amd/csrc/brq_attn.h"
#include "../../paper_2511_04214_amd/csrc/brq_launch.h"

static int launches;
namespace brq {
hipError_t device_cus(int* cus) { *cus = 256; return hipSuccess; }
hipError_t launch_heads(int, bool, bool, bool, const HeadsArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_heads_backward(int, bool, bool, const HeadsArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_heads_weight_grads(const float*, int, int, float*, float*, hipStream_t) { ++launches; return hipSuccess; }
int64_t heads_backward_workgroups(int64_t, int, int, int) { return 1; }
hipError_t launch_kv4_read(int, const uint8_t*, int64_t, int, int64_t, const int64_t*, const Heads&, const Heads&, bool, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_kv4_attention(int, const AttnArgs&, hipStream_t) { ++launches; return hipSuccess; }
int64_t kv4_attention_workspace(int64_t, int64_t, int, int, int, int64_t, int64_t, int) { return 0; }
hipError_t launch_pages_copy(const PagesArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_pages_fork(const PagesArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_pages_free(const PagesArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_pages_reserve(const PagesArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_pages_compact(const PagesArgs&, hipStream_t) { ++launches; return hipSuccess; }
}  // namespace brq

#define EXPECT(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

int main() {
    const int64_t ends[] = {INT64_MIN, INT64_MIN + 1, -((int64_t)1 << 40), -((int64_t)1 << 31), -1, 0, 1, 2, 64, 65535, 65536, (1 << 25) - 1, 1 << 25, (int64_t)INT32_MAX - 64,
                            INT32_MAX, (int64_t)1 << 31, (int64_t)1 << 34, ((int64_t)1 << 35) - 16, (int64_t)1 << 35, (int64_t)1 << 40, (int64_t)1 << 62, INT64_MAX - 1, INT64_MAX};
    const int64_t sizes[] = {INT64_MIN, -1, 0, 1, 7, 64, 128, 65535, (1 << 25) - 1, 1 << 25, INT32_MAX, (int64_t)1 << 31, INT64_MAX};
    alignas(16) static float f[64];
    alignas(16) static int64_t pos[16];
    alignas(16) static int32_t i32[64];
    alignas(16) static uint8_t bytes[64];
    int64_t n;
    long calls = 0, taken = 0;
    auto count = [&](brq_status s) { ++calls; taken += s == BRQ_OK; };
    // heads: every pair of ends of strides and counts
    for (int64_t T : sizes)
        for (int64_t H : sizes)
            for (int64_t ts : ends)
                for (int64_t hs : ends) {
                    const brq_heads x{f, H, ts, hs};
                    const brq_rope r{f, f, pos, 1, 64, 0};
                    count(brq_qk_norm_rope(&x, nullptr, BRQ_BF16, T, 64, f, nullptr, 1e-6f, &r, 32, &x, nullptr, BRQ_F32, nullptr));
                    count(brq_qk_norm_rope_backward(&x, nullptr, BRQ_F32, T, 128, f, nullptr, 1e-6f, nullptr, 1, &x, nullptr, BRQ_BF16, &x, nullptr, f, nullptr, f, 1 << 20, nullptr));
                    count(brq_kv4_append(nullptr, &x, &x, BRQ_BF16, T, 64, nullptr, nullptr, 0.0f, nullptr, 64, 8, pos, bytes, 1, nullptr, nullptr));
                    count(brq_kv4_read(bytes, 1, T, 128, pos, &x, &x, BRQ_F32, nullptr));
                    count(brq_kv4_attention(&x, T, 64, bytes, 1, 1, i32, 1, i32, i32, 1, 0.1f, 1, 0, 1, 64, &x, f, nullptr, 0, nullptr));
                }
    EXPECT(taken > 0 && taken < calls && launches > 0);
    // attention and pages: every triple of ends of what sizes the grid, the table and the workspace
    for (int64_t a : ends)
        for (int64_t b : ends)
            for (int64_t c : ends) {
                count(brq_kv4_attention_workspace(a, b, c, 1, 64, 1, 64, &n));
                count(brq_kv4_attention_workspace(1, a, 65535, 1, 128, b, c, &n));
                count(brq_kv4_attention_workspace(1, a, b, c, 128, 16, 64, &n));
                count(brq_qk_norm_rope_backward_workspace(a, b, c, 256, &n));
                count(brq_kv4_pages_workspace(a, b, &n));
                count(brq_kv4_page_bytes(a, b, &n));
                const brq_heads x{f, 4, 256, 64};
                count(brq_kv4_attention(&x, 2, 64, bytes, a, 4, i32, b, i32, i32, 1, -0.1f, 1, c, 2, 64, &x, nullptr, nullptr, 0, nullptr));
                count(brq_kv4_pages_copy(bytes, a, b, i32, i32, c, nullptr));
                count(brq_kv4_pages_fork(bytes, 64, a, i32, b, c, i32, i32, i32, i32, 3, i32, bytes, nullptr));
                count(brq_kv4_pages_free(i32, a, b, i32, i32, c, i32, 3, nullptr));
                count(brq_kv4_pages_reserve(i32, a, b, i32, c, i32, i32, 3, i32, bytes, nullptr));
                count(brq_kv4_pages_compact(bytes, 64, a, i32, b, c, i32, i32, bytes, nullptr));
            }
    // the largest grids: sequences of more rows than an int holds are refused however the factors are spread
    EXPECT(brq_kv4_attention_workspace(1, INT32_MAX, 65535, 1, 64, (1 << 25) - 1, 64, &n) == BRQ_ERR_SHAPE);
    EXPECT(brq_kv4_attention_workspace(1, (1 << 22) - 1, 1, 1, 64, 16, 64, &n) == BRQ_OK);
    EXPECT(brq_kv4_attention_workspace(1, 1 << 22, 1, 1, 64, 16, 64, &n) == BRQ_ERR_SHAPE);
    std::printf("attention api sanitizer driver ok: %ld calls, %ld taken\n", calls, taken);
    return 0;
}
