// qs_kv_fork.cu -- requests take over the first tokens of others: tables, holders of each page, free list, copies.
//
// Request r takes over the first m_r tokens of request p = parent_r as they stand before the call, m_r = min(n_p, keep_r).
// Of p's pages it holds the first w = floor(m / page) whole; where m ends inside a page (a cut), that one is to be written
// by r alone.  With h(x) = others(x) + 1 holders of a page before the call:
//     longest_p = max of w over the requests that take over from p
//     r may go on with the page it is cut in where w = longest_p and h = 1 (no one else is left with it whole);
//     one does, p itself if it may, else the first; every other cut takes a page from the list's top, in request order:
//     (inclusive prefix sum of cuts)_r <= free, or r is refused
//     h'(x) = h(x) - (requests whose old pages have x) + (requests whose new pages have x)
//     pages with h' = 0 come back, in the order of the last request that held them and of its pages.
// Four steps, each of which needs all of the one before: who gets what (one CTA: R <= 8192, prefix sums and two reductions
// in shared memory); counts of holders and the new rows, to the work space (atomic sums of whole numbers: any order gives the same, and
// a maximum that says who held a page last); pages that come back, counted; their places, and the rows in place.  Every held
// page is looked at, not only those of requests that change, and every page's count: the formula then holds whatever the counts
// were before.
// Memory is read a few times and little of it; a chain of latencies bounds it (64 requests of 82 pages 10.0 us, 975 of up to 656 29.0).
// A page that a request held and takes over again, the prefix of a beam that goes on with its sibling, needs no counting, and
// columns are looked up four at a time, not behind one another: 12.9 -> 10.0 us for the 64.
// One cluster whose CTAs meet at its barrier where tables are short, a launch a step else.  The cluster against the launches,
// host included (in a graph), requests x columns: 64 x 82 10.0 and 13.2 us (9.6 and 11.0), 128 x 82 13.2 and 14.3 (12.8 and
// 12.4), 256 x 82 18.4 and 14.0, 16 x 1019 14.8 and 13.7, 256 x 519 47 and 15.4.
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kForkThreads = 1024, kForkCluster = 8;   // at most; CTAs of the cluster
constexpr int kForkClusterRequests = 256, kForkClusterEntries = 1 << 13, kForkClusterPages = 1 << 14;   // at most; a thread a request
constexpr int kBatch = 4;   // columns of a lane that are read together
constexpr int kNoTail = -1, kBadTail = -2;

// Record of a request: parent, old pages, whole pages (bit 31: the tail is fresh), tail page.
__device__ __forceinline__ int whole_of(const int4& rec) { return rec.z & 0x7fffffff; }
__device__ __forceinline__ bool fresh_of(const int4& rec) { return rec.z < 0; }
// First old column that the request leaves.
__device__ __forceinline__ int leaves_from(const int4& rec, int r) {
    return rec.x == r ? whole_of(rec) + (rec.w >= 0 && !fresh_of(rec) ? 1 : 0) : 0;
}
// Inclusive prefix sum of x over the CTA's threads; all of them in `all`.
__device__ __forceinline__ int block_sum(int x, int& all, int* sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    int w = lane < warps ? sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, w, o);
        if (lane >= o) w += y;
    }
    all = __shfl_sync(kFull, w, 31);
    const int before = __shfl_sync(kFull, w, (warp + 31) & 31);
    __syncthreads();
    return x + (warp ? before : 0);
}

// Who gets what.  kPer: requests a thread.  smem: 2 R ints.
template <int kPer>
__device__ void fork_decide(const KvForkParams& p, int* smem, int* sums) {
    int* const longest = smem;
    unsigned* const best = reinterpret_cast<unsigned*>(smem + p.R);
    const int tid = threadIdx.x, threads = blockDim.x, R = p.R, sh = p.page_shift;
    const long long most = static_cast<long long>(p.max_pages) << sh;
    auto length = [&](int r) {
        const int n = __ldcg(p.pages.lens + r);
        if (n >= 0 && n <= most) return n;
        raise_status(p.status, QS_DEV_PAGES);
        return n < 0 ? 0 : static_cast<int>(most);
    };
    int free_n = __ldcg(p.pages.free_count);
    for (int r = tid; r < R; r += threads) longest[r] = 0, best[r] = 0xffffffffu;
    int par[kPer], n[kPer], m[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int r = k * threads + tid;
        par[k] = -1;
        n[k] = m[k] = 0;
        if (r >= R) continue;
        par[k] = __ldcg(p.parent + r);
        const int keep = p.keep ? __ldcg(p.keep + r) : -1;
        n[k] = length(r);
        if (par[k] >= R) {
            raise_status(p.status, QS_DEV_PAGES);
            par[k] = r;
        }
        if (par[k] < 0) continue;
        m[k] = par[k] == r ? n[k] : length(par[k]);
        if (keep >= 0 && keep < m[k]) m[k] = keep;
    }
    if (free_n < 0 || free_n > p.n_pages) {
        if (tid == 0) raise_status(p.status, QS_DEV_PAGES);
        free_n = min(max(free_n, 0), p.n_pages);
    }
    __syncthreads();
    int tail[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        tail[k] = kNoTail;
        if (par[k] < 0) continue;
        const int whole = m[k] >> sh;
        if (whole) atomicMax(longest + par[k], whole);
        if (m[k] & ((1 << sh) - 1)) tail[k] = __ldcg(p.pages.table + static_cast<size_t>(par[k]) * p.max_pages + whole);
        if (tail[k] >= p.n_pages || tail[k] < kNoTail || (tail[k] == kNoTail && (m[k] & ((1 << sh) - 1)))) {
            raise_status(p.status, QS_DEV_PAGES);
            tail[k] = kBadTail;
        }
    }
    __syncthreads();
    bool could[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int r = k * threads + tid;
        could[k] = tail[k] >= 0 && (m[k] >> sh) == longest[par[k]] && __ldcg(p.others + tail[k]) == 0;
        if (could[k]) atomicMin(best + par[k], r == par[k] ? 0u : static_cast<unsigned>(r) + 1u);
    }
    __syncthreads();
    int asked = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (k * threads >= R) break;
        const int r = k * threads + tid;
        const bool need = tail[k] >= 0 && !(could[k] && best[par[k]] == (r == par[k] ? 0u : static_cast<unsigned>(r) + 1u));
        int all;
        const int end = asked + block_sum(need, all, sums);
        asked += all;
        if (r >= R) continue;
        const bool ok = !need || end <= free_n;
        int src = -1, dst = -1, whole = m[k] >> sh;
        if (need && ok) {
            src = tail[k];
            dst = __ldcg(p.pages.free_list + free_n - end);
            if (dst < 0 || dst >= p.n_pages) {
                raise_status(p.status, QS_DEV_PAGES);
                src = dst = -1;
                tail[k] = kBadTail;
            } else {
                tail[k] = dst;
            }
        }
        if (!ok) {
            m[k] = whole = 0;
            par[k] = -1;
            tail[k] = kNoTail;
        }
        const int pages = static_cast<int>((static_cast<unsigned>(n[k]) + (1u << sh) - 1) >> sh);
        p.rec[r] = make_int4(par[k], pages, whole | (dst >= 0 ? static_cast<int>(0x80000000u) : 0), tail[k]);
        p.pages.lens_out[r] = m[k];
        p.ok[r] = ok;
        p.moves.src[r] = src;
        p.moves.dst[r] = dst;
    }
    // unsigned: the step behind the last entry may be above 2^31
    for (unsigned r = R + tid; r < static_cast<unsigned>(p.moves.n); r += threads) p.moves.src[r] = p.moves.dst[r] = -1;
    if (tid == 0) p.head[0] = free_n - min(asked, free_n);
}

// Columns that the request takes from another's row, [0, this).
__device__ __forceinline__ int taken_to(const int4& rec, int r) { return rec.x >= 0 && rec.x != r ? whole_of(rec) : 0; }

// The steps over pages: a warp takes one of `parts` parts of a request's columns, every `workers`-th of [worker, items).
template <class F>
__device__ __forceinline__ void each_part(const KvForkParams& p, int worker, int workers, int items, F f) {
    for (int item = worker; item < items; item += workers) {
        const int r = item / p.parts, c0 = (item - r * p.parts) * p.chunk;
        const int4 rec = __ldcg(p.rec + r);
        f(item, r, rec, c0, kv_part_end(c0, p.chunk));
    }
}

__device__ void fork_count_holders(const KvForkParams& p, int worker, int workers) {
    const int lane = threadIdx.x & 31;
    each_part(p, worker, workers, p.R * p.parts, [&](int, int r, const int4& rec, int c0, int c1) {
        const int32_t* const mine = p.pages.table + static_cast<size_t>(r) * p.max_pages;
        const int taken = taken_to(rec, r), whole = whole_of(rec), end = min(c1, max(taken, rec.y));
        const int32_t* const from = p.pages.table + static_cast<size_t>(taken ? rec.x : r) * p.max_pages;
        // the tail that is kept under a new name, and a fresh one (see fork_count_back)
        if (lane == 0 && whole >= c0 && whole < c1 && rec.w >= 0 && (rec.x != r || fresh_of(rec))) atomicAdd(p.others + rec.w, 1);
        const int kept = leaves_from(rec, r);
        for (int c = c0 + lane; c < end; c += 32 * kBatch) {
            int now[kBatch], old[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int at = c + k * 32;
                now[k] = at < min(c1, taken) ? __ldcg(from + at) : 0;
                old[k] = at < min(c1, rec.y) ? __ldcg(mine + at) : 0;
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int at = c + k * 32;
                const bool takes = at < min(c1, taken), had = at < min(c1, rec.y);
                if (takes) p.stage[static_cast<size_t>(r) * p.max_pages + at] = now[k];
                if ((takes && static_cast<unsigned>(now[k]) >= static_cast<unsigned>(p.n_pages)) ||
                    (had && static_cast<unsigned>(old[k]) >= static_cast<unsigned>(p.n_pages))) {
                    raise_status(p.status, QS_DEV_PAGES);
                }
                const bool stays = had && (at < kept || (takes && now[k] == old[k]));   // held before and after: nothing to count
                if (!stays && takes && static_cast<unsigned>(now[k]) < static_cast<unsigned>(p.n_pages)) atomicAdd(p.others + now[k], 1);
                if (had && static_cast<unsigned>(old[k]) < static_cast<unsigned>(p.n_pages)) {
                    if (!stays) atomicAdd(p.others + old[k], -1);
                    atomicMax(p.owner + old[k], r + 1);
                }
            }
        }
    });
}

// Columns c, c + 32, ... in front of `end`: their pages, whether request r is the last that held them, and holders beside the first
// (-1: nobody, so it comes back; less only where the counts did not agree with the tables).  Looked up together.
__device__ __forceinline__ void last_held(const KvForkParams& p, int r, int c, int end, int (&x)[kBatch], bool (&held)[kBatch],
                                          int (&others)[kBatch]) {
    const int32_t* const mine = p.pages.table + static_cast<size_t>(r) * p.max_pages;
    int who[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) x[k] = c + k * 32 < end ? __ldcg(mine + c + k * 32) : -1;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
        const bool there = static_cast<unsigned>(x[k]) < static_cast<unsigned>(p.n_pages);
        who[k] = there ? __ldcg(p.owner + x[k]) : 0;
        others[k] = there ? __ldcg(p.others + x[k]) : 0;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) held[k] = who[k] == r + 1;
}

// A CTA's run of the items, so that a sum over CTAs is all it needs of those before.
struct Run {
    int first, last;
    __device__ Run(int items, int cta, int ctas) {
        const int per = (items + ctas - 1) / ctas;
        first = min(items, cta * per);
        last = min(items, first + per);
    }
};
constexpr int kHeld = 1 << 30;   // beside a part's count: it has pages whose last holder the request is

__device__ void fork_count_back(const KvForkParams& p, int cta, int ctas, int* sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const Run run(p.R * p.parts, cta, ctas);
    int all = 0;
    // A page that no request held has nobody beside its first holder, a fresh one's, if it has one.  (One that was on the list although a
    // request held it is counted on.)
    constexpr int kPages = 8;   // of a thread that are read together
    const long long step = static_cast<long long>(ctas) * blockDim.x;
    for (long long x0 = cta * blockDim.x + threadIdx.x; x0 < p.n_pages; x0 += step * kPages) {
        int who[kPages], others[kPages];
#pragma unroll
        for (int k = 0; k < kPages; ++k) {
            const bool there = x0 + k * step < p.n_pages;
            who[k] = there ? __ldcg(p.owner + x0 + k * step) : 1;
            others[k] = there ? __ldcg(p.others + x0 + k * step) : 0;
        }
#pragma unroll
        for (int k = 0; k < kPages; ++k)
            if (who[k] == 0 && others[k] != 0) p.others[x0 + k * step] = 0;
    }
    each_part(p, run.first + warp, warps, run.last, [&](int item, int r, const int4& rec, int c0, int c1) {
        int n = 0;
        bool any = false;
        for (int c = c0 + lane; c < min(c1, rec.y); c += 32 * kBatch) {
            int x[kBatch], others[kBatch];
            bool held[kBatch];
            last_held(p, r, c, min(c1, rec.y), x, held, others);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                n += held[k] && others[k] == -1;
                any |= held[k];
            }
        }
        n = __reduce_add_sync(kFull, n);
        all += n;
        any = __any_sync(kFull, any);
        if (lane == 0) p.count[item] = n | (any ? kHeld : 0);
    });
    if (lane == 0) sums[warp] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < warps; ++w) all += sums[w];
        p.count[kKvMaxRequests + cta] = all;
    }
    __syncthreads();
}

// smem: an int for each item of a CTA's run.
__device__ void fork_place(const KvForkParams& p, int cta, int ctas, int* smem, int* sums) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const Run run(p.R * p.parts, cta, ctas);
    const int first = run.first, last = run.last, base = __ldcg(p.head);
    int before = 0;
#pragma unroll 4
    for (int i = tid; i < cta; i += blockDim.x) before += __ldcg(p.count + kKvMaxRequests + i);
    int total;
    block_sum(before, total, sums);   // of the items before
    for (int i0 = first; i0 < last; i0 += blockDim.x) {
        const int i = i0 + tid, n = i < last ? __ldcg(p.count + i) & ~kHeld : 0;
        int all;
        const int end = block_sum(n, all, sums);
        if (i < last) smem[i - first] = total + end - n;
        total += all;
    }
    __syncthreads();
    if (cta == ctas - 1 && tid == 0) p.pages.free_out[0] = min(base + total, p.n_pages);
    each_part(p, first + warp, warps, last, [&](int item, int r, const int4& rec, int c0, int c1) {
        int32_t* const mine = p.pages.table + static_cast<size_t>(r) * p.max_pages;
        const int end = min(c1, rec.y), whole = whole_of(rec), taken = taken_to(rec, r);
        int at = base + smem[item - first];
        const bool any = __ldcg(p.count + item) & kHeld;
        for (int c = c0; any && c < end; c += 32 * kBatch) {
            int x[kBatch], others[kBatch];
            bool held[kBatch];
            last_held(p, r, c + lane, end, x, held, others);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const bool back = held[k] && others[k] == -1;
                const unsigned mask = __ballot_sync(kFull, back);
                if (back) {
                    const int to = at + __popc(mask & ((1u << lane) - 1));
                    if (to < p.n_pages)
                        p.pages.free_list[to] = x[k];
                    else
                        raise_status(p.status, QS_DEV_PAGES);
                }
                if (held[k]) {
                    p.owner[x[k]] = 0;
                    if (others[k] < 0) p.others[x[k]] = 0;
                }
                at += __popc(mask);
            }
        }
        __syncwarp();   // the old pages of these columns are read
        for (int c = c0 + lane; c < min(c1, taken); c += 32 * kBatch) {
            int now[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (c + k * 32 < min(c1, taken)) now[k] = __ldcg(p.stage + static_cast<size_t>(r) * p.max_pages + c + k * 32);
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (c + k * 32 < min(c1, taken)) mine[c + k * 32] = now[k];
        }
        if (lane == 0 && whole >= c0 && whole < c1 && rec.w != kNoTail) mine[whole] = rec.w >= 0 ? rec.w : -1;
    });
}

// All four steps; CTAs of one cluster.
__global__ void __cluster_dims__(kForkCluster, 1, 1) __launch_bounds__(kForkThreads) kv_fork_kernel(const KvForkParams p) {
    extern __shared__ int smem[];
    __shared__ int sums[32];
    chain_wait();
    const int warps = blockDim.x >> 5, worker = blockIdx.x * warps + (threadIdx.x >> 5), workers = kForkCluster * warps;
    if (blockIdx.x == 0) fork_decide<1>(p, smem, sums);
    cluster_sync();
    fork_count_holders(p, worker, workers);
    cluster_sync();
    fork_count_back(p, blockIdx.x, kForkCluster, sums);
    cluster_sync();
    fork_place(p, blockIdx.x, kForkCluster, smem, sums);
}

// One step.
template <int kPer>
__global__ void __launch_bounds__(kForkThreads) kv_fork_step_kernel(const KvForkParams p, const int step) {
    extern __shared__ int smem[];
    __shared__ int sums[32];
    chain_wait();
    const int warps = blockDim.x >> 5, worker = blockIdx.x * warps + (threadIdx.x >> 5), workers = gridDim.x * warps;
    if (step == 0)
        fork_decide<kPer>(p, smem, sums);
    else if (step == 1)
        fork_count_holders(p, worker, workers);
    else if (step == 2)
        fork_count_back(p, blockIdx.x, gridDim.x, sums);
    else
        fork_place(p, blockIdx.x, gridDim.x, smem, sums);
}

cudaError_t launch_cluster(const KvForkParams& p, cudaStream_t stream) {
    // a thread a request in the first step, then a warp an item, as far as there are items
    const int items = p.R * p.parts;
    int threads = 256;
    while (threads < kForkThreads && threads / 32 * kForkCluster < items) threads *= 2;
    const int ints = 2 * p.R > items ? 2 * p.R : items;   // of the first and of the last step
    return launch_chained(kv_fork_kernel, kForkCluster, threads, sizeof(int) * static_cast<size_t>(ints), stream, true, p);
}

template <int kPer>
cudaError_t launch_steps(const KvForkParams& p, cudaStream_t stream) {
    // The limit is the kernel's, not the call's: every call sets the same one.
    cudaError_t e = cudaFuncSetAttribute(kv_fork_step_kernel<kPer>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         2 * sizeof(int) * kKvMaxRequests);
    constexpr int kStepThreads = 256;
    const int items = p.R * p.parts;
    // a warp an item, and no more than some pages a thread
    const int for_items = (items + kStepThreads / 32 - 1) / (kStepThreads / 32), for_pages = p.n_pages / (kStepThreads * 8);
    const int need = for_items > for_pages ? for_items : for_pages, most = 8 * device_sm_count();
    const int grid = need < 1 ? 1 : need < most ? need : most;
    const size_t decide = 2 * sizeof(int) * static_cast<size_t>(p.R), place = sizeof(int) * static_cast<size_t>((items + grid - 1) / grid);
    for (int step = 0; step < 4 && e == cudaSuccess; ++step)
        e = launch_chained(kv_fork_step_kernel<kPer>, step == 0 ? 1 : grid, step == 0 ? kForkThreads : kStepThreads,
                           step == 0 ? decide : step == 3 ? place : 0, stream, true, p, step);
    return e;
}

}  // namespace

// Parts of a request's columns, a power of two with R parts <= kKvMaxRequests, of 64 columns or more.
int kv_column_parts(int R, int max_pages) {
    int parts = 1;
    while (2LL * parts * (R < 1 ? 1 : R) <= kKvMaxRequests && 2LL * parts * 64 <= max_pages) parts *= 2;
    return parts;
}

cudaError_t launch_kv_fork(const KvForkParams& p, cudaStream_t stream) {
    // an item or so for each warp of the cluster, few columns to an item, eight pages a thread
    if (p.R <= kForkClusterRequests && static_cast<long long>(p.R) * p.max_pages <= kForkClusterEntries && p.n_pages <= kForkClusterPages)
        return launch_cluster(p, stream);
    return p.R <= kForkThreads ? launch_steps<1>(p, stream) : launch_steps<kKvMaxRequests / kForkThreads>(p, stream);
}

}  // namespace qs
