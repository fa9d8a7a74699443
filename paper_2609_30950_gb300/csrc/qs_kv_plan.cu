// qs_kv_plan.cu -- block table, slots and free list of a serving step, from the requests' lengths.
//
// With n_r tokens cached and a_r to come (a_r < 0: the request has ended), pages(n) = ceil(n / page):
//     cu = exclusive prefix sum of max(a, 0)
//     back_r = pages(n_r) where the request has ended, else 0
//     need_r = pages(n_r + a_r) - pages(n_r) where its rows and columns are there, else 0
//     stack  = free list with the pages that come back on top, height h = free + sum back
//     granted where need_r = 0 or (inclusive prefix sum of need)_r <= h; the j-th page is stack[h - 1 - j].
// The prefix sum does not go back behind a refusal, so the granted pages are the first
// max{prefix sum : granted} of the stack's top and every answer follows from three prefix sums over
// the requests.  Each CTA makes those for itself (R <= 8192: a few loads a thread) and then writes
// its share of the rows, the table and the list: one launch, no CTA waits for another.  Pages are
// read from stack places below the new height only where nothing is written and the other way
// round: the list is written at [free, new height) and read at [new height, free), the table is
// written behind a request's old pages and read in front of them.
#include "qs_common.cuh"

namespace qs {
namespace {

constexpr int kThreads = 1024;

__device__ __forceinline__ int held(long long x) { return x > 0x7fffffffLL ? 0x7fffffff : static_cast<int>(x); }

// Exclusive prefix sums over the CTA's threads of a and b, and their totals.
__device__ __forceinline__ void block_scan(long long& a, long long& b, long long& all_a, long long& all_b,
                                           long long (*warp_sums)[2]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long a0 = a, b0 = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(kFull, a, o), y = __shfl_up_sync(kFull, b, o);
        if (lane >= o) a += x, b += y;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp][0] = a, warp_sums[warp][1] = b;
    __syncthreads();
    long long wa = warp_sums[lane][0], wb = warp_sums[lane][1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(kFull, wa, o), y = __shfl_up_sync(kFull, wb, o);
        if (lane >= o) wa += x, wb += y;
    }
    all_a = __shfl_sync(kFull, wa, 31);
    all_b = __shfl_sync(kFull, wb, 31);
    const long long pa = __shfl_sync(kFull, wa, (warp + 31) & 31), pb = __shfl_sync(kFull, wb, (warp + 31) & 31);
    a += (warp ? pa : 0) - a0;
    b += (warp ? pb : 0) - b0;
}

// First r in [0, n) with ends[r] > x (n if there is none); ends does not fall.
__device__ __forceinline__ int first_above(const int* ends, int n, int x) {
    int lo = 0;
    while (n > 0) {
        const int half = n >> 1;
        if (ends[lo + half] > x) {
            n = half;
        } else {
            lo += half + 1;
            n -= half + 1;
        }
    }
    return lo;
}

__global__ void __launch_bounds__(kThreads) kv_plan_kernel(const KvPlanParams p) {
    extern __shared__ int smem[];
    __shared__ long long warp_sums[32][2];
    __shared__ int s_granted, s_last;
    const int R = p.R, tid = threadIdx.x, sh = p.page_shift;
    int* const s_len = smem;
    int* const s_end = s_len + R;     // inclusive prefix sums: rows, pages asked for, pages back
    int* const s_need = s_end + R;
    int* const s_back = s_need + R;
    int* const s_ok = s_back + R;     // 1: granted, 2: ended, 0: refused
    const long long most = static_cast<long long>(p.max_pages) << sh;
    auto pages = [&](long long n) { return (n + (1LL << sh) - 1) >> sh; };

    if (tid == 0) s_granted = 0;
    const int per = (R + kThreads - 1) / kThreads, r0 = min(R, tid * per), r1 = min(R, r0 + per);
    long long rows = 0, none = 0, all_rows, all_none;
    for (int r = r0; r < r1; ++r) {
        int n = p.pages.lens[r];
        const int a = p.n_new[r];
        if (n < 0 || n > most) {
            raise_status(p.status, QS_DEV_PAGES);
            n = n < 0 ? 0 : static_cast<int>(most);
        }
        s_len[r] = n;
        s_end[r] = a;
        rows += max(a, 0);
    }
    block_scan(rows, none, all_rows, all_none, warp_sums);
    long long need = 0, back = 0, all_need, all_back;
    {
        long long end = rows;
        for (int r = r0; r < r1; ++r) {
            const int n = s_len[r], a = s_end[r];
            end += max(a, 0);
            const bool valid = a >= 0 && end <= p.slots.T && pages(static_cast<long long>(n) + a) <= p.max_pages;
            const int nd = valid ? static_cast<int>(pages(static_cast<long long>(n) + a) - pages(n)) : 0;
            s_end[r] = held(end);
            s_need[r] = nd;
            s_back[r] = a < 0 ? static_cast<int>(pages(n)) : 0;
            s_ok[r] = a < 0 ? 2 : valid;
            need += nd;
            back += s_back[r];
        }
    }
    block_scan(need, back, all_need, all_back, warp_sums);
    int free_n = p.pages.free_count[0];
    if (free_n < 0 || free_n + all_back > p.n_pages) {
        if (tid == 0) raise_status(p.status, QS_DEV_PAGES);
        free_n = min(max(free_n, 0), p.n_pages);
    }
    const int avail = static_cast<int>(min(free_n + all_back, static_cast<long long>(p.n_pages)));
    {
        int top = 0;
        for (int r = r0; r < r1; ++r) {
            const int nd = s_need[r];
            need += nd;
            back += s_back[r];
            if (s_ok[r] == 1 && nd > 0) {
                if (need <= avail)
                    top = static_cast<int>(need);
                else
                    s_ok[r] = 0;
            }
            s_need[r] = held(need);
            s_back[r] = held(back);
        }
        if (top) atomicMax(&s_granted, top);
    }
    __syncthreads();
    if (p.in_place && gridDim.x > 1) {
        // the last CTA to have read the old lengths and count writes the new ones
        if (tid == 0) {
            __threadfence();
            s_last = atomicAdd(p.ticket, 1) == static_cast<int>(gridDim.x) - 1;
            if (s_last) *p.ticket = 0;
        }
        __syncthreads();
    }
    const int granted = s_granted, height = avail - granted;
    const int cta = blockIdx.x, step = gridDim.x * kThreads, first = cta * kThreads + tid;
    const bool alone = p.in_place && gridDim.x > 1;

    // page at a place of the stack
    auto stack = [&](int at) {
        int id;
        if (at < free_n) {
            id = p.pages.free_list[at];
        } else {
            const int x = at - free_n, r = first_above(s_back, R, x);
            if (r >= R) return -1;
            const int start = s_back[r] - static_cast<int>(pages(s_len[r]));
            id = p.pages.table[static_cast<size_t>(r) * p.max_pages + (x - start)];
        }
        if (id < 0 || id >= p.n_pages) {
            raise_status(p.status, QS_DEV_PAGES);
            id = -1;
        }
        return id;
    };
    // j-th page asked for belongs to request r, whose pages are [need_start, need_end)
    auto need_start = [&](int r) { return r > 0 ? s_need[r - 1] : 0; };

    if (!alone || s_last) {
        for (int r = alone ? tid : first; r < R; r += alone ? kThreads : step) {
            const int ok = s_ok[r], a = r > 0 ? s_end[r] - s_end[r - 1] : s_end[0];
            p.pages.lens_out[r] = ok == 2 ? 0 : s_len[r] + (ok ? a : 0);
        }
        if (tid == 0 && (alone || cta == 0)) p.pages.free_out[0] = height;
    }
    for (int r = first; r < R; r += step) {
        p.slots.cu[r + 1] = s_end[r];
        p.slots.ok[r] = s_ok[r] != 0;
    }
    if (first == 0) p.slots.cu[0] = 0;
    for (int j = first; j < granted; j += step) {
        const int r = first_above(s_need, R, j);
        const size_t col = static_cast<size_t>(pages(s_len[r])) + (j - need_start(r));
        p.pages.table[static_cast<size_t>(r) * p.max_pages + col] = stack(avail - 1 - j);
    }
    for (int at = free_n + first; at < height; at += step) p.pages.free_list[at] = stack(at);
    const int rows_all = R > 0 ? s_end[R - 1] : 0;
    for (int t = first; t < p.slots.T; t += step) {
        int slot = -1, pos = -1, req = -1;
        if (t < rows_all) {
            req = first_above(s_end, R, t);
            pos = s_len[req] + t - (req > 0 ? s_end[req - 1] : 0);
            if (s_ok[req] == 1) {
                const int col = pos >> sh, have = static_cast<int>(pages(s_len[req]));
                int id;
                if (col < have) {
                    id = p.pages.table[static_cast<size_t>(req) * p.max_pages + col];
                    if (id < 0 || id >= p.n_pages) {
                        raise_status(p.status, QS_DEV_PAGES);
                        id = -1;
                    }
                } else {
                    id = stack(avail - 1 - (need_start(req) + col - have));
                }
                if (id >= 0) slot = (id << sh) + (pos & ((1 << sh) - 1));
            }
        }
        p.slots.slot[t] = slot;
        if (p.slots.pos) p.slots.pos[t] = pos;
        if (p.slots.req) p.slots.req[t] = req;
    }
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanParams& p, cudaStream_t stream) {
    const size_t smem = 5 * sizeof(int) * static_cast<size_t>(p.R);
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kv_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   static_cast<int>(smem));
        if (e != cudaSuccess) return e;
    }
    int grid = (p.slots.T + 2 * kThreads - 1) / (2 * kThreads);
    grid = grid < 1 ? 1 : grid > device_sm_count() ? device_sm_count() : grid;
    kv_plan_kernel<<<grid, kThreads, smem, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace qs
