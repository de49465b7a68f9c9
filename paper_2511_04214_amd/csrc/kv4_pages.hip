// Pages of the MXFP4 cache: copied, shared, given up, reserved and made dense, on the device (include/brq_attn.h).
//
// What moves pages is bound by HBM; what finds them (counts of free and live pages in page order, so that results do not
// depend on the schedule) is one workgroup that goes through the counts, 16 a thread and step, 16384 a step; of caches of up to 4096 pages 4 a
// thread, in one step (a compaction of 96 sequences' pages 36.2 -> 34.0 us).
#include <type_traits>

#include "brq_attn.h"
#include "brq_device.h"
#include "brq_launch.h"

namespace brq {
namespace {

constexpr int kScan = 1024;       // threads of the workgroup that counts
constexpr int kSmall = kScan * 4; // pages of a cache whose counts are taken 4 a thread, 16 otherwise

// Sum of v over the workgroup's threads in front of this one; *total: over all.  T: an integer, or two counts in one.
template <class T>
__device__ __forceinline__ T scan_before(T v, T* lds, T* total) {
    const int lane = (int)(threadIdx.x & 63u), w = (int)(threadIdx.x >> 6);
    T x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const T y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) lds[w] = x;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kScan / 64; ++i) {
        const T n = lds[i];
        before += i < w ? n : 0;
        all += n;
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

// The counts of a thread's pages: -1 past the end.
template <int PER>
__device__ __forceinline__ void load_refs(const int32_t* refs, int n, int at, int (&r)[PER]) {
    if (at + PER <= n && (reinterpret_cast<uintptr_t>(refs) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const v4i v = *reinterpret_cast<const v4i*>(refs + at + i);
            r[i] = v.x; r[i + 1] = v.y; r[i + 2] = v.z; r[i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) r[i] = at + i < n ? refs[at + i] : -1;
    }
}

__device__ __forceinline__ bool in_range(int x, int n) { return x >= 0 && x < n; }

// Bytes of page `from` to page `to`, by all threads of the workgroups `part` of `parts`.
__device__ __forceinline__ void move_page(uint8_t* pool, int64_t page_bytes, int from, int to, int part, int parts) {
    const v4i* s = reinterpret_cast<const v4i*>(pool + (int64_t)from * page_bytes);
    v4i* d = reinterpret_cast<v4i*>(pool + (int64_t)to * page_bytes);
    const int n = (int)(page_bytes / 16), step = parts * (int)blockDim.x;
    int i = part * (int)blockDim.x + (int)threadIdx.x;
    for (; i + 3 * step < n; i += 4 * step) {
        const v4i a = s[i], b = s[i + step], c = s[i + 2 * step], e = s[i + 3 * step];
        d[i] = a; d[i + step] = b; d[i + 2 * step] = c; d[i + 3 * step] = e;
    }
    for (; i < n; i += step) d[i] = s[i];
}

// ---- workspace of fork and reserve: [0] free pages found (no more than wanted), first[n] (a call's pages in front of item i), pages[...]
struct Found {
    int32_t *count, *first, *pages;
    __host__ __device__ Found(int32_t* w, int n) : count(w), first(w + 4), pages(w + 4 + n) {}
};

// Pages that item i wants: FORK: one where its parent's last page is not full; reserve: its row's columns below the wanted
// length that have no page, none where the table has too few columns.
template <bool FORK>
__device__ __forceinline__ int wanted(const PagesArgs& a, int i) {
    if constexpr (FORK) {
        const int p = a.a[i], c = a.b[i];
        if (!in_range(p, a.S) || !in_range(c, a.S)) return 0;
        const int len = a.lens[p];
        if (len <= 0 || len > a.cols * (int64_t)kKv4Page || len % kKv4Page == 0) return 0;
        return in_range(a.table[(int64_t)p * a.cols + len / kKv4Page], a.num_pages) ? 1 : 0;
    } else {
        const int s = a.a[i], tokens = a.b[i];
        if (!in_range(s, a.S) || tokens <= 0) return 0;
        const int cols = (tokens - 1) / kKv4Page + 1;
        if (cols > a.cols) return 0;
        int n = 0;
        for (int c = 0; c < cols; ++c) n += a.table[(int64_t)s * a.cols + c] < 0;
        return n;
    }
}

// A row of the table that is to get pages, LANES lanes to it.
template <int LANES>
struct Row {
    int32_t* at = nullptr;
    int cols = 0, need = 0;
    bool none = false;           // too few columns
    __device__ static uint64_t bits(bool b) {
        return LANES == 64 ? __ballot(b) : __ballot(b) >> (threadIdx.x & (64u - LANES)) & ((1ull << (LANES & 63)) - 1);
    }
    __device__ Row(const PagesArgs& a, int i, int lane) {
        if (i < a.n && in_range(a.a[i], a.S) && a.b[i] > 0) {
            cols = (a.b[i] - 1) / kKv4Page + 1;
            at = a.table + (int64_t)a.a[i] * a.cols;
            none = cols > a.cols;
            if (none) cols = 0;
        }
        for (int c0 = 0; __any(c0 < cols); c0 += LANES) need += __popcll(bits(c0 + lane < cols && at[c0 + lane] < 0));
    }
    // `first`: its first page of those found, `found` of them.
    __device__ void fill(const PagesArgs& a, const int32_t* pages, int first, int found, int lane) {
        if (none || (need > 0 && (int64_t)first + need > found)) {
            if (lane == 0) atomicAdd(a.result, 1);
            cols = 0;
        }
        if (need == 0) cols = 0;
        for (int c0 = 0; __any(c0 < cols); c0 += LANES) {
            const bool empty = c0 + lane < cols && at[c0 + lane] < 0;
            const uint64_t m = bits(empty);
            if (empty) {
                const int page = pages[first + __popcll(m & ((1ull << lane) - 1))];
                at[c0 + lane] = page;
                a.refs[page] = 1;
            }
            first += __popcll(m);
        }
    }
};

// The first `want` free pages, lowest first, by a workgroup; r: the thread's counts, of the first step already there.  Returns how many.
template <int PER>
__device__ __forceinline__ int find_free(const PagesArgs& a, int32_t* pages, int want, int (&r)[PER], int* lds) {
    int found = 0, total;
    for (int at = 0; at < a.num_pages && found < want; at += kScan * PER) {
        int n = 0;
        const int mine = at + (int)threadIdx.x * PER;
        if (at > 0) load_refs(a.refs, a.num_pages, mine, r);
#pragma unroll
        for (int i = 0; i < PER; ++i) n += r[i] == 0;
        int rank = found + scan_before(n, lds, &total);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (r[i] == 0) {
                if (rank < want) pages[rank] = mine + i;
                ++rank;
            }
        found += total;
    }
    return min(found, want);
}

template <bool FORK, int PER>
__global__ __launch_bounds__(kScan) void k_find_free(const PagesArgs a) {
    __shared__ int lds[17];
    // 1024 rows of up to 2^25 columns each, rows named twice among them, want more pages than 32 bits count; forks one each (64 bits: 4.1 us, 3.7)
    typedef typename std::conditional<FORK, int, int64_t>::type Count;
    __shared__ Count lds2[17];
    const Found f(a.workspace, a.n);
    int r[PER];
    Count want = 0, total;
    load_refs(a.refs, a.num_pages, (int)threadIdx.x * PER, r);                   // (on their way while the wants are counted)
    for (int i0 = 0; i0 < a.n; i0 += kScan) {
        const int i = i0 + (int)threadIdx.x;
        const Count before = scan_before<Count>(i < a.n ? wanted<FORK>(a, i) : 0, lds2, &total);
        if (i < a.n) f.first[i] = (int)min<Count>(want + before, a.num_pages);   // (more than there are is as good as any more)
        want = min<Count>(want + total, a.num_pages);
    }
    const int found = find_free(a, f.pages, (int)want, r, lds);
    if (threadIdx.x == 0) {
        f.count[0] = found;
        a.result[0] = 0;
    }
}

// Reservations of up to 64 sequences in one launch, 16 lanes a row: 48 of 1000 tokens each 4.4 us; with a lane a row to count and a
// wavefront a row to fill, a launch apart or not, 8.4 us.
template <int PER>
__global__ __launch_bounds__(kScan) void k_reserve_few(const PagesArgs a) {
    __shared__ int lds[17];
    const Found f(a.workspace, a.n);
    const int lane = (int)threadIdx.x & 15;
    int total, r[PER];
    load_refs(a.refs, a.num_pages, (int)threadIdx.x * PER, r);
    Row<16> row(a, (int)threadIdx.x >> 4, lane);
    if (threadIdx.x == 0) a.result[0] = 0;
    const int first = __shfl(scan_before(lane == 0 ? row.need : 0, lds, &total), (int)threadIdx.x & 48);
    const int found = find_free(a, f.pages, min(total, a.num_pages), r, lds);
    __syncthreads();
    row.fill(a, f.pages, first, found, lane);
}

// Pairs (parent, child): `parts` workgroups copy the last page's bytes, the first of them also writes the child's row.
__global__ __launch_bounds__(256) void k_fork(const PagesArgs a, int parts) {
    const int i = (int)(blockIdx.x / parts), part = (int)(blockIdx.x % parts);
    const Found f(a.workspace, a.n);
    const int p = a.a[i], c = a.b[i];
    if (!in_range(p, a.S) || !in_range(c, a.S)) return;
    const int want = wanted<true>(a, i), len = a.lens[p], full = len > 0 ? min(len / kKv4Page, a.cols) : 0;
    int32_t *from = a.table + (int64_t)p * a.cols, *to = a.table + (int64_t)c * a.cols;
    const bool failed = want > 0 && f.first[i] >= f.count[0];
    const int page = want > 0 && !failed ? f.pages[f.first[i]] : -1;
    if (page >= 0 && full < a.cols) {                     // (always, unless another pair is just writing the parent's length)
        const int last = from[full];
        if (in_range(last, a.num_pages)) move_page(a.pool, a.page_bytes, last, page, part, parts);
    }
    if (part != 0) return;
    for (int k = (int)threadIdx.x; k < a.cols; k += 256) {
        int32_t e = -1;
        if (!failed) {
            if (k < full) {
                e = from[k];
                if (in_range(e, a.num_pages)) atomicAdd(a.refs + e, 1);
                else e = -1;
            } else if (k == full) {
                e = page;
            }
        }
        to[k] = e;
    }
    if (threadIdx.x == 0) {
        a.lens[c] = failed ? 0 : len;
        if (page >= 0) a.refs[page] = 1;
        if (failed) atomicAdd(a.result, 1);
    }
}

__global__ __launch_bounds__(64) void k_reserve(const PagesArgs a) {
    const Found f(a.workspace, a.n);
    const int i = (int)blockIdx.x, lane = (int)threadIdx.x;
    Row<64>(a, i, lane).fill(a, f.pages, f.first[i], f.count[0], lane);
}

// The entry is taken out by an exchange: a sequence named twice is given up once.
__global__ __launch_bounds__(256) void k_free(const PagesArgs a) {
    const int s = a.a[blockIdx.x];
    if (!in_range(s, a.S)) return;
    int32_t* row = a.table + (int64_t)s * a.cols;
    for (int k = (int)threadIdx.x; k < a.cols; k += 256) {
        const int e = atomicExch(row + k, -1);
        if (in_range(e, a.num_pages)) atomicSub(a.refs + e, 1);
    }
    if (threadIdx.x == 0) a.lens[s] = 0;
}

__global__ __launch_bounds__(256) void k_copy(const PagesArgs a, int parts) {
    const int i = (int)(blockIdx.x / parts), part = (int)(blockIdx.x % parts);
    const int s = a.a[i], d = a.b[i];
    if (in_range(s, a.num_pages) && in_range(d, a.num_pages) && s != d) move_page(a.pool, a.page_bytes, s, d, part, parts);
}

// ---- compaction.  Workspace: [0] moves, [1] live pages, from[N/2 + 1], to[N/2 + 1], then rank[N]: of the live pages above, which move theirs is.
struct Moves {
    int32_t *count, *from, *to, *rank;
    __host__ __device__ Moves(int32_t* w, int n) : count(w), from(w + 4), to(w + 4 + n / 2 + 1), rank(w + 4 + 2 * (n / 2 + 1)) {}
};

template <int PER>
__global__ __launch_bounds__(kScan) void k_plan_moves(const PagesArgs a) {
    __shared__ int lds[17];
    __shared__ uint64_t lds2[17];
    const Moves v(a.workspace, a.num_pages);
    constexpr int kStep = kScan * PER;
    int live = 0, total, r[PER];
    for (int at = 0; at < a.num_pages; at += kStep) {
        int n = 0;
        load_refs(a.refs, a.num_pages, at + (int)threadIdx.x * PER, r);
#pragma unroll
        for (int i = 0; i < PER; ++i) n += r[i] > 0;
        scan_before(n, lds, &total);
        live += total;
    }
    // free pages below `live` and live pages at or above it: as many of one as of the other
    int holes = 0, high = 0;
    for (int at = 0; at < a.num_pages; at += kStep) {
        uint32_t nh = 0, ns = 0;
        const int mine = at + (int)threadIdx.x * PER;
        if (a.num_pages > kStep) load_refs(a.refs, a.num_pages, mine, r);         // (otherwise they are still there)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            nh += r[i] <= 0 && mine + i < live;
            ns += r[i] > 0 && mine + i >= live;
        }
        uint64_t both;
        const uint64_t before = scan_before((uint64_t)ns << 32 | nh, lds2, &both);
        int hole = holes + (int)(uint32_t)before, src = high + (int)(before >> 32);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (mine + i < live) {
                if (r[i] <= 0) v.to[hole++] = mine + i;
            } else if (mine + i < a.num_pages) {
                v.rank[mine + i] = r[i] > 0 ? src : -1;                           // -1: an entry that names a free page
                if (r[i] > 0) v.from[src++] = mine + i;
            }
        }
        holes += (int)(uint32_t)both;
        high += (int)(both >> 32);
    }
    if (threadIdx.x == 0) {
        v.count[0] = high;
        v.count[1] = live;
        a.result[0] = live;
    }
}

__global__ __launch_bounds__(256) void k_move(const PagesArgs a, int parts) {
    const Moves v(a.workspace, a.num_pages);
    const int moves = v.count[0], live = v.count[1];
    for (int64_t k = blockIdx.x; k < (int64_t)moves * parts; k += gridDim.x) {
        const int i = (int)(k / parts), part = (int)(k % parts), from = v.from[i], to = v.to[i];
        move_page(a.pool, a.page_bytes, from, to, part, parts);
        if (part == 0 && threadIdx.x == 0) {
            a.refs[to] = a.refs[from];
            a.refs[from] = 0;
        }
    }
    const int64_t entries = (int64_t)a.S * a.cols;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < entries; k += (int64_t)gridDim.x * 256) {
        const int e = a.table[k];
        if (e >= live && e < a.num_pages) {
            const int m = v.rank[e];
            a.table[k] = m < 0 ? -1 : v.to[m];
        }
    }
}

// Workgroups to each of n pages: 16 KB a piece, and no more than a grid can have.
int parts_of(int64_t page_bytes, int64_t n) {
    const int64_t parts = (page_bytes + 16383) / 16384, most = (int64_t(1) << 23) / n;
    return (int)(parts < most ? parts : most > 1 ? most : 1);
}

}  // namespace

hipError_t launch_pages_copy(const PagesArgs& a, hipStream_t stream) {
    const int parts = parts_of(a.page_bytes, a.n);
    hipLaunchKernelGGL(k_copy, dim3((uint32_t)a.n * parts), dim3(256), 0, stream, a, parts);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream) {
    if (a.num_pages <= kSmall) hipLaunchKernelGGL((k_find_free<true, 4>), dim3(1), dim3(kScan), 0, stream, a);
    else hipLaunchKernelGGL((k_find_free<true, 16>), dim3(1), dim3(kScan), 0, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (a.n == 0) return hipSuccess;
    const int parts = parts_of(a.page_bytes, a.n);
    hipLaunchKernelGGL(k_fork, dim3((uint32_t)a.n * parts), dim3(256), 0, stream, a, parts);
    return hipGetLastError();
}

hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(k_free, dim3((uint32_t)a.n), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t stream) {
    if (a.n <= 64) {
        if (a.num_pages <= kSmall) hipLaunchKernelGGL((k_reserve_few<4>), dim3(1), dim3(kScan), 0, stream, a);
        else hipLaunchKernelGGL((k_reserve_few<16>), dim3(1), dim3(kScan), 0, stream, a);
        return hipGetLastError();
    }
    if (a.num_pages <= kSmall) hipLaunchKernelGGL((k_find_free<false, 4>), dim3(1), dim3(kScan), 0, stream, a);
    else hipLaunchKernelGGL((k_find_free<false, 16>), dim3(1), dim3(kScan), 0, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(k_reserve, dim3((uint32_t)a.n), dim3(64), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream) {
    if (a.num_pages <= kSmall) hipLaunchKernelGGL((k_plan_moves<4>), dim3(1), dim3(kScan), 0, stream, a);
    else hipLaunchKernelGGL((k_plan_moves<16>), dim3(1), dim3(kScan), 0, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(k_move, dim3(2048), dim3(256), 0, stream, a, parts_of(a.page_bytes, 1));
    return hipGetLastError();
}

}  // namespace brq
