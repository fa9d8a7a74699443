// qs_kv_compact.cu -- pages that requests hold move to the pool's low end, in front of a limit.
//
// With used(x) where a table holds page x: the sources are the used x >= limit, the places the unused x < limit, both in
// ascending order; the i-th source moves to the i-th place for i < k = min(sources, places, moves that the caller has
// room for).  The free list becomes the places that are left, the lowest on top.
// Four steps, each of which needs all of the one before: a bit for each page that a table holds; sources and places of each
// span of pages, counted; their ranks (a sum over the spans before, a prefix sum over the span's words), moves and
// list; the tables.  Memory is read once (tables twice) and little of it: a chain of latencies.  One cluster whose CTAs meet at its
// barrier where tables are short and the pool has at most a span for each of its CTAs, a launch a step else.  Host
// included, the cluster against the launches, requests x columns: 27 x 51 9.2 and 13.1 us, 60 x 82 9.9 and 13.9, 120 x 144 13.1 and
// 13.2, 180 x 144 15.2 and 13.9.
// A span is 8192 pages, a word of bits a thread (more where the pool would have over 2048 spans, whose sums every CTA reads):
// 132000 pages 17.3 us in a graph (21 when this was chosen, and 46 by spans of 32768, a thread's pages one after another).
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kBatch = 8, kCluster = 8, kClusterEntries = 1 << 14;
static_assert(32 * kThreads == kCompactSpan, "a word a thread");

__device__ __forceinline__ int held_pages(const KvCompactParams& p, int r, bool report) {
    const int n = __ldcg(p.pages.lens + r);
    const long long most = static_cast<long long>(p.max_pages) << p.page_shift;
    if (n >= 0 && n <= most) return static_cast<int>((static_cast<unsigned>(n) + (1u << p.page_shift) - 1) >> p.page_shift);
    if (report) raise_status(p.status, QS_DEV_PAGES);
    return n < 0 ? 0 : p.max_pages;
}

// A warp takes one of `parts` parts of a request's columns.  f gets the entry's place and kBatch entries, 32 apart, of which those
// in front of n count.  They are read together: 720 rows of up to 687, 20.7 -> 17.3 us against one after another, each behind
// the store of the one before.
template <class F>
__device__ __forceinline__ void each_entry(const KvCompactParams& p, bool report, F f) {
    const int lane = threadIdx.x & 31, workers = gridDim.x * kWarps, items = p.R * p.parts;
    for (int item = blockIdx.x * kWarps + (threadIdx.x >> 5); item < items; item += workers) {
        const int r = item / p.parts, c0 = (item - r * p.parts) * p.chunk;
        const int c1 = min(kv_part_end(c0, p.chunk), held_pages(p, r, report && c0 == 0));
        const size_t row = static_cast<size_t>(r) * p.max_pages;
        for (int c = c0 + lane; c < c1; c += 32 * kBatch) {
            int x[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) x[k] = c + k * 32 < c1 ? __ldcg(p.pages.table + row + c + k * 32) : 0;
            f(row + c, x, c1 - c);
        }
    }
}

__device__ void compact_mark(const KvCompactParams& p) {
    each_entry(p, true, [&](size_t, const int(&x)[kBatch], int n) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (k * 32 >= n) continue;
            if (x[k] < 0 || x[k] >= p.n_pages)
                raise_status(p.status, QS_DEV_PAGES);
            else
                atomicOr(p.used + (x[k] >> 5), 1u << (x[k] & 31));   // nothing waits for it
        }
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

__device__ void compact_count(const KvCompactParams& p, int2* sums) {
    int2 n = make_int2(0, 0);
    for (int k = 0; k < p.words; ++k) {
        const int w = (blockIdx.x * p.words + k) * kThreads + threadIdx.x;
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

__device__ void compact_move(const KvCompactParams& p, int spans, int2 (*sums)[kWarps]) {
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
    const int moved = min(min(all.x, all.y), p.moves.n), left = all.y - moved;
    if (blockIdx.x == 0 && tid == 0) {
        p.pages.free_out[0] = left;
        if (p.left) p.left[0] = all.x - moved;
        p.head[0] = moved;
    }
    // unsigned: the step behind the last entry may be above 2^31
    for (unsigned i = moved + blockIdx.x * kThreads + tid; i < static_cast<unsigned>(p.moves.n); i += spans * kThreads)
        p.moves.src[i] = p.moves.dst[i] = -1;
    int i0 = before.x, j0 = before.y;   // ranks of the next words' first source and place
    for (int k = 0; k < p.words; ++k) {
        __syncthreads();   // the sums are read
        const int w = (blockIdx.x * p.words + k) * kThreads + tid;
        const uint32_t in = in_pool(p, w), low = below_limit(p, w), used = in ? __ldcg(p.used + w) : 0u;
        const uint32_t source = used & in & ~low, place = ~used & in & low;
        if (in) p.used[w] = 0;   // as it was found
        const int2 n = make_int2(__popc(source), __popc(place));
        int2 end = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(kFull, end.x, o), y = __shfl_up_sync(kFull, end.y, o);
            if (lane >= o) end.x += x, end.y += y;
        }
        if (lane == 31) sums[0][warp] = end;
        __syncthreads();
        int i = i0 + end.x - n.x, j = j0 + end.y - n.y;
#pragma unroll
        for (int v = 0; v < kWarps; ++v) {
            if (v < warp) i += sums[0][v].x, j += sums[0][v].y;
            i0 += sums[0][v].x;
            j0 += sums[0][v].y;
        }
        // a word's pages by the warp's lanes, word after word
        const unsigned below = (1u << lane) - 1;
#pragma unroll 4
        for (int v = 0; v < 32; ++v) {
            const uint32_t from = __shfl_sync(kFull, source, v), to = __shfl_sync(kFull, place, v);
            const int iv = __shfl_sync(kFull, i, v) + __popc(from & below), jv = __shfl_sync(kFull, j, v) + __popc(to & below);
            const int x = (w - lane + v) * 32 + lane;
            if ((from >> lane) & 1) {
                p.rank[x] = iv;
                if (iv < moved) p.moves.src[iv] = x;
            }
            if ((to >> lane) & 1) {
                if (jv < moved)
                    p.moves.dst[jv] = x;
                else
                    p.pages.free_list[left - 1 - (jv - moved)] = x;
            }
        }
    }
}

__device__ void compact_table(const KvCompactParams& p) {
    const int moved = __ldcg(p.head);
    each_entry(p, false, [&](size_t at, const int(&x)[kBatch], int n) {
        int i[kBatch], to[kBatch];   // -1: stays
#pragma unroll
        for (int k = 0; k < kBatch; ++k) i[k] = x[k] >= p.limit && x[k] < p.n_pages ? __ldcg(p.rank + x[k]) : moved;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) to[k] = i[k] < moved ? __ldcg(p.moves.dst + i[k]) : -1;
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (k * 32 < n && (to[k] >= 0 || p.table_out != p.pages.table)) p.table_out[at + k * 32] = to[k] >= 0 ? to[k] : x[k];
    });
    if (p.others)
        for (int i = blockIdx.x * kThreads + threadIdx.x; i < moved; i += gridDim.x * kThreads) {
            const int src = __ldcg(p.moves.src + i), dst = __ldcg(p.moves.dst + i);
            p.others[dst] = __ldcg(p.others + src);
            p.others[src] = 0;
        }
}

// One step.
template <int kStep>
__global__ void __launch_bounds__(kThreads) kv_compact_step_kernel(const KvCompactParams p, const int spans) {
    __shared__ int2 sums[2][kWarps];
    chain_wait();
    if (kStep == 0) compact_mark(p);
    if (kStep == 1) compact_count(p, sums[0]);
    if (kStep == 2) compact_move(p, spans, sums);
    if (kStep == 3) compact_table(p);
}

// All four; CTAs of one cluster, a span each at most.
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads) kv_compact_kernel(const KvCompactParams p, const int spans) {
    __shared__ int2 sums[2][kWarps];
    const bool mine = static_cast<int>(blockIdx.x) < spans;
    chain_wait();
    compact_mark(p);
    cluster_sync();
    if (mine) compact_count(p, sums[0]);
    cluster_sync();
    if (mine) compact_move(p, spans, sums);
    cluster_sync();
    compact_table(p);
}

}  // namespace

cudaError_t launch_kv_compact(KvCompactParams p, cudaStream_t stream) {
    p.words = 1;
    while ((static_cast<long long>(p.n_pages) + static_cast<long long>(kCompactSpan) * p.words - 1) / (static_cast<long long>(kCompactSpan) * p.words) > 2048)
        p.words *= 2;
    const long long span = static_cast<long long>(kCompactSpan) * p.words;
    const int spans = static_cast<int>((p.n_pages + span - 1) / span);
    const long long warps = static_cast<long long>(p.R) * p.parts, most = 8LL * device_sm_count();
    long long grid = (warps + kWarps - 1) / kWarps;
    grid = grid < 1 ? 1 : grid < most ? grid : most;
    if (p.words == 1 && spans <= kCluster && static_cast<long long>(p.R) * p.max_pages <= kClusterEntries)
        return launch_chained(kv_compact_kernel, kCluster, kThreads, 0, stream, true, p, spans);
    cudaError_t e = launch_chained(kv_compact_step_kernel<0>, static_cast<int>(grid), kThreads, 0, stream, true, p, spans);
    if (e == cudaSuccess) e = launch_chained(kv_compact_step_kernel<1>, spans, kThreads, 0, stream, true, p, spans);
    if (e == cudaSuccess) e = launch_chained(kv_compact_step_kernel<2>, spans, kThreads, 0, stream, true, p, spans);
    if (e == cudaSuccess) e = launch_chained(kv_compact_step_kernel<3>, static_cast<int>(grid), kThreads, 0, stream, true, p, spans);
    return e;
}

}  // namespace qs
