// qs_kv_group.cu -- which requests share their first tokens, and the blocks of rows that read those once.
//
// Group g is the requests [start_g, start_g+1) and has c_g tokens in common.  A request takes part if it has them all and sees
// them all (n >= c, and no window or n <= window), the group shares if two take part; its rows are its requests' query
// heads of a key head, in blocks.  Every row of a block sees all c tokens, so that no row has a mask of its own there; a request that
// does not take part reads its tokens by itself.  One CTA: two searches and a prefix sum in shared memory, some
// latencies (256 requests: see the table of the design notes).
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kThreads = 1024;

struct Sums {
    long long units;
    int groups, blocks;
};
__device__ __forceinline__ Sums plus(const Sums& a, const Sums& b) { return {a.units + b.units, a.groups + b.groups, a.blocks + b.blocks}; }
__device__ __forceinline__ Sums shuffled(const Sums& a, int o) {
    return {__shfl_up_sync(kFull, a.units, o), __shfl_up_sync(kFull, a.groups, o), __shfl_up_sync(kFull, a.blocks, o)};
}

__global__ void __launch_bounds__(kThreads) kv_group_kernel(const KvGroupParams p) {
    extern __shared__ int smem[];
    __shared__ Sums s_warp[32];
    chain_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, N = p.N;
    int* const start = smem;            // N + 1
    int* const count = start + N + 1;   // requests that take part; then blocks of a key head, 0 where nothing is shared
    int* const owner = count + N;       // the first of them; then the group's first block
    for (int g = tid; g <= N; g += kThreads) start[g] = __ldcg(p.start + g);
    for (int g = tid; g < N; g += kThreads) count[g] = 0, owner[g] = p.R;
    __syncthreads();
    bool bad = N > 0 && tid == 0 && (start[0] < 0 || start[N] > p.R);
    for (int g = tid; g < N; g += kThreads) bad = bad || start[g] > start[g + 1];
    if (__syncthreads_or(bad)) {   // no group at all
        if (tid == 0) {
            raise_status(p.status, QS_DEV_PAGES);
            *p.out = p.head;
        }
        for (int r = tid; r < p.R; r += kThreads) p.shared[r] = make_int4(0, 0, 0, 0);
        return;
    }
    // the group of request r, or -1
    auto group_of = [&](int r) {
        int lo = 0, n = N + 1;   // first g with start[g] > r
        while (n > 0) {
            const int half = n >> 1;
            if (start[lo + half] <= r) {
                lo += half + 1;
                n -= half + 1;
            } else {
                n = half;
            }
        }
        return lo > 0 && lo <= N ? lo - 1 : -1;
    };
    auto common = [&](int g) {
        const int c = __ldcg(p.common + g);
        if (c < 0 || c > p.most) raise_status(p.status, QS_DEV_PAGES);
        return c < 0 || c > p.most ? 0 : c;
    };
    auto takes_part = [&](int r, int c) {
        const int n = __ldcg(p.lens + r);
        return c > 0 && n >= c && n <= p.most && (p.window == 0 || n <= p.window);
    };
    for (int r = tid; r < p.R; r += kThreads) {
        const int g = group_of(r);
        if (g >= 0 && takes_part(r, common(g))) {
            atomicAdd(count + g, 1);
            atomicMin(owner + g, r);
        }
    }
    __syncthreads();
    const int per = (N + kThreads - 1) / kThreads, g0 = min(N, tid * per), g1 = min(N, g0 + per);
    auto blocks_of = [&](int g) {
        return count[g] < 2 ? 0 : static_cast<int>((static_cast<long long>(start[g + 1] - start[g]) * p.G + p.rows - 1) / p.rows);
    };
    auto sums_of = [&](int g) {
        const int blocks = blocks_of(g);
        if (blocks == 0) return Sums{0, 0, 0};
        return Sums{static_cast<long long>(blocks) * p.Hkv * ((common(g) + p.tile - 1) / p.tile + kSharedRowUnits), 1, blocks * p.Hkv};
    };
    Sums mine{0, 0, 0};
    for (int g = g0; g < g1; ++g) mine = plus(mine, sums_of(g));
    Sums before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums x = shuffled(before, o);
        if (lane >= o) before = plus(before, x);
    }
    if (lane == 31) s_warp[warp] = before;
    const Sums lower = shuffled(before, 1);
    __syncthreads();
    Sums at{0, 0, 0}, all{0, 0, 0};
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) at = plus(at, s_warp[w]);
        all = plus(all, s_warp[w]);
    }
    if (lane) at = plus(at, lower);
    for (int g = g0; g < g1; ++g) {
        const Sums s = sums_of(g);
        const int blocks = blocks_of(g);
        if (blocks) p.groups[at.groups] = {start[g], (start[g + 1] - start[g]) * p.G, owner[g], common(g), blocks, at.blocks, at.units};
        count[g] = blocks;
        owner[g] = at.blocks;
        at = plus(at, s);
    }
    if (tid == 0) {
        KvGroupHead head = p.head;
        head.groups = all.groups;
        head.units = all.units;
        *p.out = head;
    }
    __syncthreads();
    for (int r = tid; r < p.R; r += kThreads) {
        const int g = group_of(r);
        int4 rec = make_int4(0, 0, 0, 0);
        if (g >= 0 && count[g]) {
            const int c = common(g);
            if (takes_part(r, c)) rec = make_int4(c, owner[g], count[g], (r - start[g]) * p.G);
        }
        p.shared[r] = rec;
    }
}

}  // namespace

cudaError_t launch_kv_group(const KvGroupParams& p, cudaStream_t stream) {
    // The limit is the kernel's, not the call's: every call sets the same one.
    constexpr int kMost = (3 * kKvMaxRequests + 1) * sizeof(int);
    const cudaError_t e = cudaFuncSetAttribute(kv_group_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    return launch_chained(kv_group_kernel, 1, kThreads, (3 * static_cast<size_t>(p.N) + 1) * sizeof(int), stream, true, p);
}

}  // namespace qs
