// qs_kv_group.cu -- which requests share their first tokens, and the blocks of rows that read those once.
//
// Group g is the requests [start_g, start_g+1) and has c_g tokens in common.  A request takes part if it has them all and sees
// them all (n >= c, and no window or n <= window), the group shares if two take part; its rows are its requests' query
// heads of a key head, in blocks.  Every row of a block sees all c tokens, so that no row has a mask of its own there; a request that
// does not take part reads its tokens by itself, and so do all of them where sharing would gain nothing (qs_kv.h).  A few numbers a
// request: one CTA, two searches and a prefix sum in shared memory, a chain of latencies (4 to 256 requests 4.2 us).
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kMostThreads = 1024;

struct Sums {
    long long units, gain;   // gain: ns
    int groups, blocks;
};
__device__ __forceinline__ Sums plus(const Sums& a, const Sums& b) { return {a.units + b.units, a.gain + b.gain, a.groups + b.groups, a.blocks + b.blocks}; }
__device__ __forceinline__ Sums shuffled(const Sums& a, int o) {
    return {__shfl_up_sync(kFull, a.units, o), __shfl_up_sync(kFull, a.gain, o), __shfl_up_sync(kFull, a.groups, o), __shfl_up_sync(kFull, a.blocks, o)};
}
// Inclusive prefix sum over a warp's lanes.
__device__ __forceinline__ Sums scanned(Sums a) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums x = shuffled(a, o);
        if ((threadIdx.x & 31) >= o) a = plus(a, x);
    }
    return a;
}

// kPer: requests a thread, kept in registers.
template <int kPer>
__global__ void __launch_bounds__(kMostThreads) kv_group_kernel(const KvGroupParams p) {
    extern __shared__ int smem[];
    __shared__ Sums s_warp[32];
    __shared__ int s_tokens;
    chain_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, N = p.N;
    int* const start = smem;             // N + 1
    int* const common = start + N + 1;   // tokens
    int* const count = common + N;       // requests that take part; then blocks of a key head, 0 where nothing is shared
    int* const owner = count + N;        // the first of them; then the group's first block
    int len[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int r = k * threads + tid;
        len[k] = r < p.R ? __ldcg(p.lens + r) : 0;
    }
    for (int g = tid; g < N; g += threads) {
        const int c = __ldcg(p.common + g);
        if (c < 0 || c > p.most) raise_status(p.status, QS_DEV_PAGES);
        common[g] = c < 0 || c > p.most ? 0 : c;
        count[g] = 0;
        owner[g] = p.R;
    }
    for (int g = tid; g <= N; g += threads) start[g] = __ldcg(p.start + g);
    if (tid == 0) s_tokens = 0;
    __syncthreads();
    bool bad = tid == 0 && (start[0] < 0 || start[N] > p.R);
    for (int g = tid; g < N; g += threads) bad = bad || start[g] > start[g + 1];
    if (__syncthreads_or(bad)) {   // no group at all
        if (tid == 0) {
            raise_status(p.status, QS_DEV_PAGES);
            *p.out = p.head;
        }
        for (int r = tid; r < p.R; r += threads) p.shared[r] = make_int4(0, 0, 0, 0);
        return;
    }
    int group[kPer];   // that a request takes part in, or -1
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int r = k * threads + tid;
        group[k] = -1;
        if (r >= p.R) continue;
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
        if (lo == 0 || lo > N) continue;
        const int g = lo - 1, c = common[g];
        if (c > 0 && len[k] >= c && len[k] <= p.most && (p.window == 0 || len[k] <= p.window)) {
            group[k] = g;
            atomicAdd(count + g, 1);
            atomicMin(owner + g, r);
        }
    }
    __syncthreads();
    // a thread's groups, one after another
    const int per = (N + threads - 1) / threads, g0 = min(N, tid * per), g1 = min(N, g0 + per);
    auto sums_of = [&](int g) {
        if (count[g] < 2) return Sums{0, 0, 0, 0};
        const long long rows = static_cast<long long>(start[g + 1] - start[g]) * p.G;
        const int blocks = static_cast<int>((rows + p.rows - 1) / p.rows), tiles = (common[g] + p.tile - 1) / p.tile;
        const float halves = static_cast<float>((rows + p.half_rows - 1) / p.half_rows);
        const float gain = (static_cast<float>(count[g]) * tiles * p.alone_ns - halves * (tiles + kSharedRowUnits) * p.block_ns) * p.Hkv;
        if (p.least_ns > 0 && gain <= 0.0f) return Sums{0, 0, 0, 0};
        const bool light = rows - static_cast<long long>(blocks - 1) * p.rows <= p.light_rows;
        const long long units = static_cast<long long>(tiles + kSharedRowUnits) * ((blocks - 1) * kSharedWeight + (light ? kSharedHalfWeight : kSharedWeight));
        return Sums{units * p.Hkv, static_cast<long long>(gain), 1, blocks * p.Hkv};
    };
    Sums mine{0, 0, 0, 0};
    for (int g = g0; g < g1; ++g) mine = plus(mine, sums_of(g));
    const Sums end = scanned(mine);
    if (lane == 31) s_warp[warp] = end;
    __syncthreads();
    const Sums warps = scanned(lane < threads / 32 ? s_warp[lane] : Sums{0, 0, 0, 0});
    auto from = [](const Sums& a, int l) {
        return Sums{__shfl_sync(kFull, a.units, l), __shfl_sync(kFull, a.gain, l), __shfl_sync(kFull, a.groups, l), __shfl_sync(kFull, a.blocks, l)};
    };
    Sums all = from(warps, 31);
    const bool worth = p.least_ns <= 0 || all.gain >= p.least_ns;
    if (!worth) all = Sums{0, 0, 0, 0};
    const Sums lower = from(warps, (warp + 31) & 31), before = shuffled(end, 1);
    Sums at = warp ? lower : Sums{0, 0, 0, 0};
    if (lane) at = plus(at, before);
    for (int g = g0; g < g1; ++g) {
        const Sums s = worth ? sums_of(g) : Sums{0, 0, 0, 0};
        const int blocks = s.blocks / p.Hkv;
        if (blocks) {
            p.groups[at.groups] = {start[g], (start[g + 1] - start[g]) * p.G, owner[g], common[g], blocks, at.blocks, at.units};
            atomicMax(&s_tokens, common[g]);
        }
        count[g] = blocks;
        owner[g] = at.blocks;
        at = plus(at, s);
    }
    __syncthreads();
    if (tid == 0) {
        KvGroupHead head = p.head;
        head.groups = all.groups;
        head.tokens = s_tokens;
        head.units = all.units;
        *p.out = head;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int r = k * threads + tid, g = group[k];
        if (r >= p.R) continue;
        p.shared[r] = g >= 0 && count[g] ? make_int4(common[g], owner[g], count[g], (r - start[g]) * p.G) : make_int4(0, 0, 0, 0);
    }
}

template <int kPer>
cudaError_t launch_group(const KvGroupParams& p, int threads, cudaStream_t stream) {
    // The limit is the kernel's, not the call's: every call sets the same one.
    constexpr int kMost = (4 * kKvMaxRequests + 1) * sizeof(int);
    const cudaError_t e = cudaFuncSetAttribute(kv_group_kernel<kPer>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    return launch_chained(kv_group_kernel<kPer>, 1, threads, (4 * static_cast<size_t>(p.N) + 1) * sizeof(int), stream, true, p);
}

}  // namespace

cudaError_t launch_kv_group(const KvGroupParams& p, cudaStream_t stream) {
    if (p.R > kMostThreads) return launch_group<kKvMaxRequests / kMostThreads>(p, kMostThreads, stream);
    return launch_group<1>(p, p.R <= 256 ? 256 : kMostThreads, stream);
}

}  // namespace qs
