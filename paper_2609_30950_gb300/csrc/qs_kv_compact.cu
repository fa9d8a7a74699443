// qs_kv_compact.cu -- pages that requests hold move to the pool's low end, in front of a limit.
//
// With used(x) where a table holds page x: the sources are the used x >= limit, the places the unused x < limit, both in
// ascending order; the i-th source moves to the i-th place for i < k = min(sources, places, moves that the caller has
// room for).  The free list becomes the places that are left, the lowest on top.
// Four steps, each of which needs all of the one before: a bit for each page that a table holds; sources and places of each
// span of 32768 pages, counted; their ranks (a sum over the spans before, a prefix sum over the span's words), moves and
// list; the tables.  Memory is read once (tables twice) and little of it: a chain of four launches' latencies.
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kWordsPer = kCompactSpan / 32 / kThreads;
static_assert(kWordsPer * 32 * kThreads == kCompactSpan, "a thread's words of a span");

__device__ __forceinline__ int held_pages(const KvCompactParams& p, int r, bool report) {
    const int n = __ldcg(p.pages.lens + r);
    const long long most = static_cast<long long>(p.max_pages) << p.page_shift;
    if (n >= 0 && n <= most) return static_cast<int>((static_cast<unsigned>(n) + (1u << p.page_shift) - 1) >> p.page_shift);
    if (report) raise_status(p.status, QS_DEV_PAGES);
    return n < 0 ? 0 : p.max_pages;
}

// A warp takes one of `parts` parts of a request's columns.
template <class F>
__device__ __forceinline__ void each_entry(const KvCompactParams& p, bool report, F f) {
    const int lane = threadIdx.x & 31, workers = gridDim.x * kWarps, items = p.R * p.parts;
    for (int item = blockIdx.x * kWarps + (threadIdx.x >> 5); item < items; item += workers) {
        const int r = item / p.parts, c0 = (item - r * p.parts) * p.chunk, c1 = min(c0 + p.chunk, held_pages(p, r, report && c0 == 0));
#pragma unroll 4
        for (int c = c0 + lane; c < c1; c += 32) f(static_cast<size_t>(r) * p.max_pages + c);
    }
}

__global__ void __launch_bounds__(kThreads) kv_compact_mark_kernel(const KvCompactParams p) {
    chain_wait();
    each_entry(p, true, [&](size_t at) {
        const int x = __ldcg(p.pages.table + at);
        if (x < 0 || x >= p.n_pages) {
            raise_status(p.status, QS_DEV_PAGES);
            return;
        }
        const uint32_t bit = 1u << (x & 31);
        if (!(__ldcg(p.used + (x >> 5)) & bit)) atomicOr(p.used + (x >> 5), bit);   // pages held together come many times
    });
}

// Pages of word w that are sources, and those that are places.
__device__ __forceinline__ uint32_t in_pool(const KvCompactParams& p, int w) {
    const long long n = p.n_pages - 32LL * w;
    return n >= 32 ? kFull : n <= 0 ? 0u : (1u << n) - 1;
}
__device__ __forceinline__ uint32_t below_limit(const KvCompactParams& p, int w) {
    const long long n = p.limit - 32LL * w;
    return n >= 32 ? kFull : n <= 0 ? 0u : (1u << n) - 1;
}

__device__ __forceinline__ int2 warp_add(int2 x) {
    return make_int2(__reduce_add_sync(kFull, x.x), __reduce_add_sync(kFull, x.y));
}

__global__ void __launch_bounds__(kThreads) kv_compact_count_kernel(const KvCompactParams p) {
    __shared__ int2 sums[kWarps];
    chain_wait();
    int2 n = make_int2(0, 0);
#pragma unroll
    for (int k = 0; k < kWordsPer; ++k) {
        const int w = (blockIdx.x * kWordsPer + k) * kThreads + threadIdx.x;
        const uint32_t all = in_pool(p, w), low = below_limit(p, w);
        const uint32_t used = all ? __ldcg(p.used + w) : 0u;
        n.x += __popc(used & all & ~low);
        n.y += __popc(~used & all & low);
    }
    n = warp_add(n);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        int2 t = make_int2(0, 0);
        for (int w = 0; w < kWarps; ++w) t.x += sums[w].x, t.y += sums[w].y;
        p.spans[blockIdx.x] = t;
    }
}

__global__ void __launch_bounds__(kThreads) kv_compact_move_kernel(const KvCompactParams p, const int spans) {
    __shared__ int2 sums[2][kWarps];
    chain_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // sources and places of the spans before this one, and of all
    int2 before = make_int2(0, 0), all = make_int2(0, 0);
    for (int s = tid; s < spans; s += kThreads) {
        const int2 n = __ldcg(p.spans + s);
        if (s < static_cast<int>(blockIdx.x)) before.x += n.x, before.y += n.y;
        all.x += n.x;
        all.y += n.y;
    }
    before = warp_add(before);
    all = warp_add(all);
    if (lane == 0) sums[0][warp] = before, sums[1][warp] = all;
    __syncthreads();
    before = all = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        before.x += sums[0][w].x, before.y += sums[0][w].y;
        all.x += sums[1][w].x, all.y += sums[1][w].y;
    }
    __syncthreads();
    const int moved = min(min(all.x, all.y), p.moves.n), left = all.y - moved;
    if (blockIdx.x == 0) {
        if (tid == 0) {
            p.pages.free_out[0] = left;
            if (p.left) p.left[0] = all.x - moved;
            p.head[0] = moved;
        }
        for (int i = moved + tid; i < p.moves.n; i += kThreads) p.moves.src[i] = p.moves.dst[i] = -1;
    }
    // consecutive words a thread, so that a prefix sum over the threads ranks them
    const int w0 = (blockIdx.x * kThreads + tid) * kWordsPer;
    uint32_t source[kWordsPer], place[kWordsPer];
    int2 n = make_int2(0, 0);
#pragma unroll
    for (int k = 0; k < kWordsPer; ++k) {
        const uint32_t in = in_pool(p, w0 + k), low = below_limit(p, w0 + k), used = in ? __ldcg(p.used + w0 + k) : 0u;
        source[k] = used & in & ~low;
        place[k] = ~used & in & low;
        n.x += __popc(source[k]);
        n.y += __popc(place[k]);
        if (in) p.used[w0 + k] = 0;   // as it was found
    }
    int2 end = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(kFull, end.x, o), y = __shfl_up_sync(kFull, end.y, o);
        if (lane >= o) end.x += x, end.y += y;
    }
    if (lane == 31) sums[0][warp] = end;
    __syncthreads();
    int i = before.x + end.x - n.x, j = before.y + end.y - n.y;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
        if (w < warp) i += sums[0][w].x, j += sums[0][w].y;
#pragma unroll
    for (int k = 0; k < kWordsPer; ++k) {
        for (uint32_t bits = source[k]; bits; bits &= bits - 1, ++i) {
            const int x = (w0 + k) * 32 + __ffs(bits) - 1;
            p.rank[x] = i;
            if (i < moved) p.moves.src[i] = x;
        }
        for (uint32_t bits = place[k]; bits; bits &= bits - 1, ++j) {
            const int x = (w0 + k) * 32 + __ffs(bits) - 1;
            if (j < moved)
                p.moves.dst[j] = x;
            else
                p.pages.free_list[left - 1 - (j - moved)] = x;
        }
    }
}

__global__ void __launch_bounds__(kThreads) kv_compact_table_kernel(const KvCompactParams p) {
    chain_wait();
    const int moved = __ldcg(p.head);
    each_entry(p, false, [&](size_t at) {
        int x = __ldcg(p.pages.table + at);
        bool moves = false;
        if (x >= p.limit && x < p.n_pages) {
            const int i = __ldcg(p.rank + x);
            if (i < moved) {
                x = __ldcg(p.moves.dst + i);
                moves = true;
            }
        }
        if (moves || p.table_out != p.pages.table) p.table_out[at] = x;
    });
    if (p.others)
        for (int i = blockIdx.x * kThreads + threadIdx.x; i < moved; i += gridDim.x * kThreads) {
            const int src = __ldcg(p.moves.src + i), dst = __ldcg(p.moves.dst + i);
            p.others[dst] = __ldcg(p.others + src);
            p.others[src] = 0;
        }
}

}  // namespace

cudaError_t launch_kv_compact(const KvCompactParams& p, cudaStream_t stream) {
    const int spans = static_cast<int>((static_cast<long long>(p.n_pages) + kCompactSpan - 1) / kCompactSpan);
    const long long warps = static_cast<long long>(p.R) * p.parts, most = 8LL * device_sm_count();
    long long grid = (warps + kWarps - 1) / kWarps;
    grid = grid < 1 ? 1 : grid < most ? grid : most;
    cudaError_t e = launch_chained(kv_compact_mark_kernel, static_cast<int>(grid), kThreads, 0, stream, true, p);
    if (e == cudaSuccess) e = launch_chained(kv_compact_count_kernel, spans, kThreads, 0, stream, true, p);
    if (e == cudaSuccess) e = launch_chained(kv_compact_move_kernel, spans, kThreads, 0, stream, true, p, spans);
    if (e == cudaSuccess) e = launch_chained(kv_compact_table_kernel, static_cast<int>(grid), kThreads, 0, stream, true, p);
    return e;
}

}  // namespace qs
