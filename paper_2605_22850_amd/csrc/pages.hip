// Pages of a pool as they are shared, copied, freed and moved together.  The
// state is one count per page, the number of tables that hold it; a page whose
// count is not positive is free.  Everything happens on the device and in
// stream order: no call waits for the host.
//
// Two kinds of kernel.  A plan (which pages are free, which move where) is one
// workgroup's scan over the counts, one page or 16 to a thread: 4 bytes a page.  The copies
// are 16-byte pieces with remapped pages, bound by memory.
//
// Measured, in a pool of 512 pages of 32 layers (2 MB a page): 160 pages move in 138 us
// (671 MB, 4.9 TB/s; a copy of 1 GiB moves 5.1) after a plan of 4.3; sixteen copies of
// one page take 10 us (33.6 MB written, 3.4 TB/s: the start and the end of a launch are
// as long as what lies between) after a take of 2.8.
#include <algorithm>

#include "common.hpp"

namespace oc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kCopyThreads = 256;
constexpr int kSegment = kCopyThreads * 8 * 16;       // bytes of one workgroup's piece of a page
constexpr int kPlanThreads = 1024;

// Copy `bytes` (a multiple of 16, at most kSegment) with one workgroup: eight
// loads of a thread in flight.  What is written is not read again soon, so it
// bypasses the caches; and so does what is read, unless several copies read it.
template <bool REREAD>
__device__ inline void copy_segment(const unsigned char *src, unsigned char *dst, int bytes) {
    u32x4 x[8];
    const int t = (int)threadIdx.x * 16;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (t + i * kCopyThreads * 16 < bytes) {
            const u32x4 *from = reinterpret_cast<const u32x4 *>(src + t + i * kCopyThreads * 16);
            x[i] = REREAD ? *from : __builtin_nontemporal_load(from);
        }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (t + i * kCopyThreads * 16 < bytes)
            __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4 *>(dst + t + i * kCopyThreads * 16));
}

// Segment `item` of the copies of n pairs of pages: every region of a pair in
// turn.  Pairs with an id outside the pool are left out.
template <bool REREAD>
__device__ inline void copy_item(const PagesArgs &a, int64_t item, int32_t src, int32_t dst) {
    const int segments = (int)((a.page_bytes + kSegment - 1) / kSegment);
    const int64_t in_pair = item % ((int64_t)a.regions * segments);
    const int region = (int)(in_pair / segments), seg = (int)(in_pair - (int64_t)region * segments);
    if ((uint32_t)src >= (uint32_t)a.num_pages || (uint32_t)dst >= (uint32_t)a.num_pages) return;
    unsigned char *const base = a.pool + (int64_t)region * a.num_pages * a.page_bytes + (int64_t)seg * kSegment;
    const int64_t left = a.page_bytes - (int64_t)seg * kSegment;
    copy_segment<REREAD>(base + src * a.page_bytes, base + dst * a.page_bytes, (int)(left < kSegment ? left : kSegment));
}
static int64_t copy_items(const PagesArgs &a, int64_t n) {
    return n * a.regions * ((a.page_bytes + kSegment - 1) / kSegment);
}
__device__ inline int64_t items_per_pair(const PagesArgs &a) {
    return (int64_t)a.regions * ((a.page_bytes + kSegment - 1) / kSegment);
}

__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(PagesArgs a, const int32_t *src, const int32_t *dst,
                                                                  int64_t items) {
    const int64_t per = items_per_pair(a);
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) copy_item<false>(a, i, src[i / per], dst[i / per]);
}

// Exclusive sum of x over the workgroup's threads; the total in every thread.
__device__ inline uint32_t block_scan(uint32_t x, uint32_t *total, uint32_t *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();                                  // the last call's sums have been read
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        before += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    *total = all;
    return before + s - x;
}

// Which of this thread's N pages from `first` on are held (one bit each).  N is 1 where
// that covers the pool, so that no thread goes through several pages one after the
// other (512 pages: a take 3.5 -> 2.8 us, a plan 6.8 -> 4.3), else 16, four loads at once.
template <int N>
__device__ inline uint32_t held_pages(const int32_t *counts, int64_t first, int32_t num_pages) {
    typedef int32_t i32x4 __attribute__((ext_vector_type(4), aligned(4)));
    uint32_t held = 0;
    if constexpr (N % 4 == 0) {
        if (first + N <= num_pages) {
            i32x4 c[N / 4];
#pragma unroll
            for (int i = 0; i < N / 4; ++i) c[i] = *reinterpret_cast<const i32x4 *>(counts + first + i * 4);
#pragma unroll
            for (int i = 0; i < N; ++i) held |= (uint32_t)(c[i / 4][i % 4] > 0) << i;
            return held;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (first + i < num_pages) held |= (uint32_t)(counts[first + i] > 0) << i;
    return held;
}
template <int N>
__device__ inline uint32_t pages_below(int64_t first, int64_t limit) {
    const int64_t n = limit - first;
    return n <= 0 ? 0u : n >= N ? (1u << N) - 1 : (1u << n) - 1;
}

// The n lowest free pages, in order, to out[i * stride], with a count of 1;
// *status 0.  With fewer than n free: -1 to all of them, *status OC_ENOMEM, the
// counts as they were.
template <int N>
__global__ __launch_bounds__(kPlanThreads) void pages_take_kernel(PagesArgs a, int32_t n, int32_t *out, int64_t stride) {
    __shared__ uint32_t sums[kPlanThreads / 64];
    constexpr int64_t STEP = (int64_t)kPlanThreads * N;
    int64_t found = 0;
    for (int64_t p0 = 0; p0 < a.num_pages && found < n; p0 += STEP) {
        const int64_t first = p0 + (int64_t)threadIdx.x * N;
        uint32_t free = ~held_pages<N>(a.counts, first, a.num_pages) & pages_below<N>(first, a.num_pages), total;
        int64_t at = found + block_scan((uint32_t)__popc(free), &total, sums);
        for (; free && at < n; free &= free - 1, ++at) out[at * stride] = (int32_t)(first + __ffs(free) - 1);
        found += total;
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i < n; i += kPlanThreads) {
        if (found >= n) a.counts[out[i * stride]] = 1;
        else out[i * stride] = -1;
    }
    if (threadIdx.x == 0) *a.status = found >= n ? OC_OK : OC_ENOMEM;
}

// The first `table_wgs` workgroups write the children's tables and the counts of the
// shared pages; the others copy the parent's last, partial page to the children's
// own, which are in their tables already (-1, and so no copy, where they did not get
// one).
__global__ __launch_bounds__(kCopyThreads) void pages_fork_kernel(PagesArgs a, const int32_t *parent, int32_t full,
                                                                  int32_t part, int32_t n, int32_t *children,
                                                                  int64_t stride, int64_t items, int32_t table_wgs) {
    if ((int)blockIdx.x >= table_wgs) {
        const int64_t per = items_per_pair(a), wgs = (int64_t)gridDim.x - table_wgs;
        for (int64_t i = (int64_t)blockIdx.x - table_wgs; i < items; i += wgs)
            copy_item<true>(a, i, parent[full], children[i / per * stride + full]);
        return;
    }
    if (!part) {
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = OC_OK;
    } else if (*a.status != OC_OK) {
        return;
    }
    const int64_t entries = (int64_t)n * full;
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += (int64_t)table_wgs * kCopyThreads) {
        const int64_t c = i / full, e = i - c * full;
        const int32_t p = parent[e];
        children[c * stride + e] = p;
        if (c == 0 && (uint32_t)p < (uint32_t)a.num_pages) atomicAdd(a.counts + p, n);
    }
}

__global__ __launch_bounds__(kCopyThreads) void pages_release_kernel(PagesArgs a, const int32_t *pages, int32_t n) {
    const int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x;
    if (i >= n) return;
    const int32_t p = pages[i];
    if ((uint32_t)p < (uint32_t)a.num_pages) atomicSub(a.counts + p, 1);
}

// Workspace of a compaction, in 32-bit words: [0] moves; from 16 on the
// sources, the targets, and every page's new id.
__device__ __host__ inline int64_t ws_src(int64_t) { return 16; }
__device__ __host__ inline int64_t ws_dst(int64_t P) { return 16 + (P / 2 + 1); }
__device__ __host__ inline int64_t ws_map(int64_t P) { return 16 + 2 * (P / 2 + 1); }

// With `live` pages held, those at or behind `live` move, in order, to the free
// ones before it, in order: as many of each, and no page is read and written.  With
// b(p) held pages before page p, a free page p in front is the (p - b(p))-th target
// and a held one behind the (b(p) - b(live))-th source, so one scan gives both.
template <int N>
__global__ __launch_bounds__(kPlanThreads) void pages_plan_kernel(PagesArgs a, int32_t *ws, int32_t *num_live) {
    constexpr int NEAR = 2048;                        // moves whose ids stay in LDS too
    __shared__ uint32_t sums[kPlanThreads / 64];
    __shared__ int32_t near_src[NEAR], near_dst[NEAR];
    __shared__ int64_t before_live;
    constexpr int64_t STEP = (int64_t)kPlanThreads * N;
    const int64_t P = a.num_pages;
    int32_t *const src = ws + ws_src(P), *const dst = ws + ws_dst(P), *const map = ws + ws_map(P);
    uint32_t held = 0, below = 0, total = 0;          // this thread's pages, those held before them, and in the step
    int64_t live = 0;
    for (int64_t p0 = 0; p0 < P; p0 += STEP) {
        held = held_pages<N>(a.counts, p0 + (int64_t)threadIdx.x * N, a.num_pages);
        below = block_scan((uint32_t)__popc(held), &total, sums);
        live += total;
    }
    int64_t run = 0;
    for (int64_t p0 = 0; p0 < P; p0 += STEP) {
        const int64_t first = p0 + (int64_t)threadIdx.x * N;
        if (P > STEP) {                               // else the pass above has them
            held = held_pages<N>(a.counts, first, a.num_pages);
            below = block_scan((uint32_t)__popc(held), &total, sums);
        }
        const int64_t b = run + below;
        if (live >= p0 && live < p0 + STEP) {         // the step that has page `live`: no source came before it
            if (live >= first && live < first + N)
                before_live = b + __popc(held & ((1u << (live - first)) - 1));
            __syncthreads();
        }
        const uint32_t low = pages_below<N>(first, live), here = pages_below<N>(first, P);
        // (the bounds hold unless another stream changes the counts meanwhile)
        for (uint32_t f = ~held & low; f; f &= f - 1) {
            const int i = __ffs(f) - 1;
            const int64_t k = first + i - b - __popc(held & ((1u << i) - 1));
            if (k < 0 || k > P / 2) break;
            dst[k] = (int32_t)(first + i);
            if (k < NEAR) near_dst[k] = (int32_t)(first + i);
        }
        if (p0 + STEP > live) {
            for (uint32_t f = held & here & ~low; f; f &= f - 1) {
                const int i = __ffs(f) - 1;
                const int64_t m = b + __popc(held & ((1u << i) - 1)) - before_live;
                if (m < 0 || m > P / 2) break;
                src[m] = (int32_t)(first + i);
                if (m < NEAR) near_src[m] = (int32_t)(first + i);
            }
        }
        for (int i = 0; i < N && first + i < P; ++i) map[first + i] = (int32_t)(first + i);
        run += total;
    }
    __syncthreads();
    int64_t moves = live < P ? live - before_live : 0;
    if (moves > P / 2) moves = P / 2;
    for (int64_t i = threadIdx.x; i < moves; i += kPlanThreads) {
        const int32_t s = i < NEAR ? near_src[i] : src[i], d = i < NEAR ? near_dst[i] : dst[i];
        map[s] = d;
        a.counts[d] = a.counts[s];
        a.counts[s] = 0;
    }
    if (threadIdx.x == 0) {
        ws[0] = (int32_t)moves;
        *num_live = (int32_t)live;
    }
}

// The first `table_wgs` workgroups rewrite the tables, the others copy the pages.
__global__ __launch_bounds__(kCopyThreads) void pages_move_kernel(PagesArgs a, int32_t *tables, int32_t entries,
                                                                  int64_t stride, int64_t n_entries, const int32_t *ws,
                                                                  int32_t table_wgs) {
    const int32_t *const src = ws + ws_src(a.num_pages), *const dst = ws + ws_dst(a.num_pages), *const map = ws + ws_map(a.num_pages);
    if ((int)blockIdx.x >= table_wgs) {
        const int64_t per = items_per_pair(a), items = (int64_t)ws[0] * per, wgs = (int64_t)gridDim.x - table_wgs;
        for (int64_t i = (int64_t)blockIdx.x - table_wgs; i < items; i += wgs) copy_item<false>(a, i, src[i / per], dst[i / per]);
        return;
    }
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < n_entries; i += (int64_t)table_wgs * kCopyThreads) {
        int32_t *const e = tables + i / entries * stride + i % entries;
        const int32_t p = *e;
        if ((uint32_t)p < (uint32_t)a.num_pages) *e = map[p];
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// workgroups of a copy: eight to a CU, each taking its next segment when one is done
static unsigned copy_grid(int64_t items) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(items, 2048)); }

hipError_t launch_pages_take(const PagesArgs &a, int32_t n, int32_t *out, int64_t stride, hipStream_t s) {
    if (a.num_pages <= kPlanThreads)
        hipLaunchKernelGGL(pages_take_kernel<1>, dim3(1), dim3(kPlanThreads), 0, s, a, n, out, stride);
    else
        hipLaunchKernelGGL(pages_take_kernel<16>, dim3(1), dim3(kPlanThreads), 0, s, a, n, out, stride);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesArgs &a, const int32_t *src, const int32_t *dst, int32_t n, hipStream_t s) {
    const int64_t items = copy_items(a, n);
    hipLaunchKernelGGL(pages_copy_kernel, dim3(copy_grid(items)), dim3(kCopyThreads), 0, s, a, src, dst, items);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs &a, const int32_t *parent, int32_t full, bool part, int32_t n,
                             int32_t *children, int64_t stride, hipStream_t s) {
    if (part) {
        const hipError_t e = launch_pages_take(a, n, children + full, stride, s);
        if (e != hipSuccess) return e;
    }
    const int64_t items = part ? copy_items(a, n) : 0;
    const unsigned tables = copy_grid(((int64_t)n * full + kCopyThreads - 1) / kCopyThreads);
    hipLaunchKernelGGL(pages_fork_kernel, dim3(tables + copy_grid(items)), dim3(kCopyThreads), 0, s, a, parent, full, (int32_t)part,
                       n, children, stride, items, (int32_t)tables);
    return hipGetLastError();
}

hipError_t launch_pages_release(const PagesArgs &a, const int32_t *pages, int32_t n, hipStream_t s) {
    hipLaunchKernelGGL(pages_release_kernel, dim3((unsigned)(((int64_t)n + kCopyThreads - 1) / kCopyThreads)),
                       dim3(kCopyThreads), 0, s, a, pages, n);
    return hipGetLastError();
}

size_t pages_workspace_bytes(int64_t num_pages) { return (size_t)(ws_map(num_pages) + num_pages) * 4; }

hipError_t launch_pages_compact(const PagesArgs &a, int32_t *tables, int32_t n_tables, int32_t entries, int64_t stride,
                                int32_t *num_live, int32_t *ws, hipStream_t s) {
    if (a.num_pages <= kPlanThreads)
        hipLaunchKernelGGL(pages_plan_kernel<1>, dim3(1), dim3(kPlanThreads), 0, s, a, ws, num_live);
    else
        hipLaunchKernelGGL(pages_plan_kernel<16>, dim3(1), dim3(kPlanThreads), 0, s, a, ws, num_live);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // the moves are counted on the device: enough workgroups for as many as there can be
    const int64_t n_entries = (int64_t)n_tables * entries;
    const unsigned table_wgs = copy_grid((n_entries + kCopyThreads - 1) / kCopyThreads);
    hipLaunchKernelGGL(pages_move_kernel, dim3(table_wgs + copy_grid(copy_items(a, a.num_pages / 2))), dim3(kCopyThreads), 0, s, a,
                       tables, std::max(entries, 1), stride, n_entries, ws, (int32_t)table_wgs);
    return hipGetLastError();
}

}  // namespace oc
