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
// written behind a request's old pages and read in front of them.  A chain of latencies (lengths, three scans,
// a search, a page): 256 requests with a token each 4.6 us; with 700 requests' prompts, some hundred thousand rows, 9.7.
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

// Sums are held at 2^32 - 1: every term is under 2^31 and so is everything they are compared with, and a sum
// that is held stays so, whichever way its terms are grouped.
__device__ __forceinline__ unsigned held_add(unsigned a, unsigned b) {
    const unsigned c = a + b;
    return c < a ? 0xffffffffu : c;
}

// Exclusive prefix sums of a and b over the CTA's threads, and b's total.  sums: 2 x 32 of shared memory.
__device__ __forceinline__ void block_scan(unsigned& a, unsigned& b, unsigned& all_b, unsigned (*sums)[32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    unsigned x = a, y = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned u = __shfl_up_sync(kFull, x, o), v = __shfl_up_sync(kFull, y, o);
        if (lane >= o) x = held_add(x, u), y = held_add(y, v);
    }
    if (lane == 31) sums[0][warp] = x, sums[1][warp] = y;
    __syncthreads();
    unsigned wx = lane < warps ? sums[0][lane] : 0u, wy = lane < warps ? sums[1][lane] : 0u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned u = __shfl_up_sync(kFull, wx, o), v = __shfl_up_sync(kFull, wy, o);
        if (lane >= o) wx = held_add(wx, u), wy = held_add(wy, v);
    }
    all_b = __shfl_sync(kFull, wy, 31);
    const unsigned px = __shfl_sync(kFull, wx, (warp + 31) & 31), py = __shfl_sync(kFull, wy, (warp + 31) & 31);
    const unsigned ex = __shfl_up_sync(kFull, x, 1), ey = __shfl_up_sync(kFull, y, 1);
    a = held_add(warp ? px : 0u, lane ? ex : 0u);
    b = held_add(warp ? py : 0u, lane ? ey : 0u);
}

// First r in [0, n) with ends[r] > x (n if there is none); ends does not fall.
__device__ __forceinline__ int first_above(const unsigned* ends, int n, unsigned x) {
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

template <int kRows>
__global__ void __launch_bounds__(256) kv_plan_kernel(const KvPlanParams p) {
    extern __shared__ int smem[];
    chain_wait();
    __shared__ unsigned sums[4][32];
    __shared__ unsigned s_granted;
    __shared__ int s_last;
    const int R = p.R, tid = threadIdx.x, sh = p.page_shift;
    int* const s_len = smem;
    unsigned* const s_end = reinterpret_cast<unsigned*>(s_len + R);   // inclusive prefix sums: rows, pages asked for, pages back
    unsigned* const s_need = s_end + R;
    unsigned* const s_back = s_need + R;
    int* const s_ok = reinterpret_cast<int*>(s_back + R);             // 1: granted, 2: ended, 0: refused
    const long long most = static_cast<long long>(p.max_pages) << sh;
    auto pages = [&](unsigned n) { return (n + (1u << sh) - 1) >> sh; };   // n < 2^31

    const int threads = blockDim.x, per = (R + threads - 1) / threads, r0 = min(R, tid * per), r1 = min(R, r0 + per);
    int free_n = __ldcg(p.pages.free_count);
    unsigned rows = 0, none = 0, all;
    if (tid == 0) s_granted = 0;
#pragma unroll 4
    for (int r = tid; r < R; r += threads) {
        s_len[r] = __ldcg(p.pages.lens + r);
        s_ok[r] = __ldcg(p.n_new + r);
    }
    __syncthreads();
    for (int r = r0; r < r1; ++r) {
        const int n = s_len[r];
        if (n < 0 || n > most) {
            raise_status(p.status, QS_DEV_PAGES);
            s_len[r] = n < 0 ? 0 : static_cast<int>(most);
        }
        rows = held_add(rows, max(s_ok[r], 0));
    }
    block_scan(rows, none, all, sums);
    unsigned need = 0, back = 0;
    for (int r = r0; r < r1; ++r) {
        const int n = s_len[r], a = s_ok[r];
        rows = held_add(rows, max(a, 0));
        const long long want = static_cast<long long>(n) + a;
        const bool valid = a >= 0 && rows <= static_cast<unsigned>(p.slots.T) && want <= most;
        const unsigned nd = valid ? pages(static_cast<unsigned>(want)) - pages(n) : 0u, bk = a < 0 ? pages(n) : 0u;
        s_end[r] = rows;
        s_need[r] = nd;
        s_back[r] = bk;
        s_ok[r] = a < 0 ? 2 : valid;
        need = held_add(need, nd);
        back = held_add(back, bk);
    }
    block_scan(need, back, all, sums + 2);
    const unsigned n_pages = static_cast<unsigned>(p.n_pages);
    if (free_n < 0 || held_add(static_cast<unsigned>(free_n), all) > n_pages) {
        if (tid == 0) raise_status(p.status, QS_DEV_PAGES);
        free_n = min(max(free_n, 0), p.n_pages);
    }
    const int avail = static_cast<int>(min(held_add(static_cast<unsigned>(free_n), all), n_pages));
    unsigned top = 0;
    for (int r = r0; r < r1; ++r) {
        const unsigned nd = s_need[r];
        need = held_add(need, nd);
        back = held_add(back, s_back[r]);
        if (s_ok[r] == 1 && nd > 0) {
            if (need <= static_cast<unsigned>(avail))
                top = need;
            else
                s_ok[r] = 0;
        }
        s_need[r] = need;
        s_back[r] = back;
    }
    if (top) atomicMax(&s_granted, top);
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
    const int granted = static_cast<int>(s_granted), height = avail - granted;
    const int cta = blockIdx.x, step = gridDim.x * threads, first = cta * threads + tid;
    const bool alone = p.in_place && gridDim.x > 1;

    // page at a place of the stack
    auto stack = [&](int at) {
        int id;
        if (at < free_n) {
            id = p.pages.free_list[at];
        } else {
            const int x = at - free_n, r = first_above(s_back, R, x);
            if (r >= R) return -1;
            const int start = static_cast<int>(s_back[r]) - static_cast<int>(pages(s_len[r]));
            id = p.pages.table[static_cast<size_t>(r) * p.max_pages + (x - start)];
        }
        if (id < 0 || id >= p.n_pages) {
            raise_status(p.status, QS_DEV_PAGES);
            id = -1;
        }
        return id;
    };
    // j-th page asked for belongs to request r, whose pages are [need_start, need_end)
    auto need_start = [&](int r) { return r > 0 ? static_cast<int>(s_need[r - 1]) : 0; };

    if (!alone || s_last) {
        for (int r = alone ? tid : first; r < R; r += alone ? threads : step) {
            const int ok = s_ok[r], a = static_cast<int>(r > 0 ? s_end[r] - s_end[r - 1] : s_end[0]);
            p.pages.lens_out[r] = ok == 2 ? 0 : s_len[r] + (ok ? a : 0);
        }
        if (tid == 0 && (alone || cta == 0)) p.pages.free_out[0] = height;
    }
    for (int r = first; r < R; r += step) {
        p.slots.cu[r + 1] = static_cast<int>(min(s_end[r], 0x7fffffffu));
        p.slots.ok[r] = s_ok[r] != 0;
    }
    if (first == 0) p.slots.cu[0] = 0;
    // pages that are taken and pages that come back, by the threads from the far end, so that few rows and few
    // pages are worked side by side
    const int pushed = max(height - free_n, 0);
    for (int i = step - 1 - first; i < granted + pushed; i += step) {
        if (i < granted) {
            const int r = first_above(s_need, R, i);
            const size_t col = static_cast<size_t>(pages(s_len[r])) + (i - need_start(r));
            p.pages.table[static_cast<size_t>(r) * p.max_pages + col] = stack(avail - 1 - i);
        } else {
            const int at = free_n + i - granted;
            p.pages.free_list[at] = stack(at);
        }
    }
    // kRows rows by a thread: one search, and one page where they share it
    const unsigned rows_all = R > 0 ? s_end[R - 1] : 0u;
    const int T = p.slots.T;
    for (long long q = first; q * kRows < T; q += step) {
        const int t0 = static_cast<int>(q * kRows);
        int slot[kRows], pos[kRows], req[kRows], r = R, page = -1, id = -1;
        if (static_cast<unsigned>(t0) < rows_all) r = first_above(s_end, R, t0);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const unsigned t = static_cast<unsigned>(t0) + k;
            slot[k] = pos[k] = req[k] = -1;
            if (t >= rows_all || t >= static_cast<unsigned>(T)) continue;
            if (t >= s_end[r]) {
                while (t >= s_end[r]) ++r;
                page = -1;
            }
            req[k] = r;
            pos[k] = s_len[r] + static_cast<int>(t - (r > 0 ? s_end[r - 1] : 0u));
            if (s_ok[r] != 1) continue;
            const int col = pos[k] >> sh, have = static_cast<int>(pages(s_len[r]));
            if (col != page) {
                page = col;
                if (col < have) {
                    id = p.pages.table[static_cast<size_t>(r) * p.max_pages + col];
                    if (id < 0 || id >= p.n_pages) {
                        raise_status(p.status, QS_DEV_PAGES);
                        id = -1;
                    }
                } else {
                    id = stack(avail - 1 - (need_start(r) + col - have));
                }
            }
            if (id >= 0) slot[k] = (id << sh) + (pos[k] & ((1 << sh) - 1));
        }
        auto put = [&](int* out, const int* v) {
            if (!out) return;
            if (kRows % 4 == 0 && p.aligned && t0 + kRows <= T) {
#pragma unroll
                for (int k = 0; k < kRows; k += 4)
                    *reinterpret_cast<int4*>(out + t0 + k) = make_int4(v[k], v[(k + 1) % kRows], v[(k + 2) % kRows], v[(k + 3) % kRows]);
            } else {
#pragma unroll
                for (int k = 0; k < kRows; ++k)
                    if (t0 + k < T) out[t0 + k] = v[k];
            }
        };
        put(p.slots.slot, slot);
        put(p.slots.pos, pos);
        put(p.slots.req, req);
    }
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanParams& p, cudaStream_t stream) {
    const size_t smem = 5 * sizeof(int) * static_cast<size_t>(p.R);
    // Four rows in a row by a thread where requests have many: one search and mostly one page look-up for them.  With
    // a row or so for each request the look-ups would follow one another (256 requests: 6.8 us against 4.6).
    const bool many = p.slots.T > 16LL * p.R;
    auto* const kernel = many ? kv_plan_kernel<4> : kv_plan_kernel<1>;
    // 48 KB without asking count the kernel's own arrays (some 500 bytes) too.  The limit is the kernel's, not the
    // call's: every call sets the same one, so that none takes it away from another thread's between its two steps.
    constexpr int kAsk = 40 * 1024, kMost = 5 * sizeof(int) * kKvMaxRequests;
    if (smem > kAsk) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
    }
    // CTAs of 8 warps, four at least: a decode step's few rows, and the pages that ended requests give back, are
    // worked side by side.
    constexpr int kThreads = 256, kMostPerSm = 4;
    const long long threads = (static_cast<long long>(p.slots.T) + (many ? 3 : 0)) / (many ? 4 : 1);
    long long grid = (threads + kThreads - 1) / kThreads;
    if (grid < 4) grid = 4;
    if (grid > kMostPerSm * device_sm_count()) grid = kMostPerSm * device_sm_count();
    return launch_chained(kernel, static_cast<int>(grid), kThreads, smem, stream, true, p);
}

}  // namespace qs
