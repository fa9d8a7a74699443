// qs_kv_tiles.cuh -- what the attention kernels over the paged cache share: how the work is divided and
// how the parts of a row are joined.
//
// A row of work is one request and one group of its heads; its unit is a tile of tokens.  The units of all
// rows, request after request, are dealt out evenly: CTA c of n takes a contiguous range of them,
// so that a long row is split and short ones are strung together, whatever the lengths are, and no
// length has to be known on the host.  A row that several CTAs share is joined by the last of them
// to finish (a counter says who that is), in the order of the tokens: the sum does not depend on which it
// was.
#pragma once

#include "qs_common.cuh"

namespace qs {
namespace kv {

// Tokens of a request that are seen: [begin, end); tiles start at base, a multiple of `grain`.
struct Span {
    int begin, end, base, tiles;
};

__device__ __forceinline__ int clamped_len(const KvAttendParams& p, int r, bool report) {
    const int n = __ldg(p.lens + r);
    const long long most = static_cast<long long>(p.max_pages) << p.page_shift;
    if (n >= 0 && n <= most) return n;
    if (report) raise_status(p.status, QS_DEV_PAGES);
    return n < 0 ? 0 : static_cast<int>(most);
}

template <int kTile, int kGrain>
__device__ __forceinline__ Span span_of(const KvAttendParams& p, int n) {
    Span s;
    s.end = n;
    s.begin = p.window > 0 && n > p.window ? n - p.window : 0;
    s.base = s.begin & ~(kGrain - 1);
    s.tiles = (n - s.base + kTile - 1) / kTile;
    return s;
}

// A CTA's share of the units.
struct Share {
    long long total;        // units of all rows
    long long u0, u1;       // this CTA's
    int r, group, tile;     // where u0 is
};

__device__ __forceinline__ long long share_start(long long total, int cta, int ctas) {
    const long long q = total / ctas, rem = total - q * ctas;
    return q * cta + (cta < rem ? cta : rem);
}
// CTA whose share holds unit u.
__device__ __forceinline__ int share_owner(long long total, long long u, int ctas) {
    const long long q = total / ctas, rem = total - q * ctas, cut = rem * (q + 1);
    return static_cast<int>(u < cut ? u / (q + 1) : rem + (u - cut) / q);
}

// All threads of the CTA; `groups` rows a request.  scratch: kThreads / 32 + 4 long longs of shared memory.
template <int kThreads, int kTile, int kGrain>
__device__ Share make_share(const KvAttendParams& p, int groups, int worker, int workers, long long* scratch) {
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.R + kThreads - 1) / kThreads, r0 = min(p.R, tid * per), r1 = min(p.R, r0 + per);
    long long mine = 0;
    for (int r = r0; r < r1; ++r) mine += span_of<kTile, kGrain>(p, clamped_len(p, r, blockIdx.x == 0)).tiles;
    long long before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(kFull, before, o);
        if (lane >= o) before += x;
    }
    if (lane == 31) scratch[warp] = before;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += scratch[w];
        all += scratch[w];
    }
    before -= mine;
    Share s;
    s.total = all * groups;
    s.u0 = share_start(s.total, worker, workers);
    s.u1 = share_start(s.total, worker + 1, workers);
    long long* const found = scratch + kWarps;
    const long long first = before * groups;
    if (s.u0 < s.u1 && s.u0 >= first && s.u0 < first + mine * groups) {
        long long at = s.u0 - first;
        for (int r = r0; r < r1; ++r) {
            const int tiles = span_of<kTile, kGrain>(p, clamped_len(p, r, false)).tiles;
            if (at < static_cast<long long>(tiles) * groups) {
                found[0] = r;
                found[1] = at / tiles;
                found[2] = at % tiles;
                break;
            }
            at -= static_cast<long long>(tiles) * groups;
        }
    }
    __syncthreads();
    s.r = static_cast<int>(found[0]);
    s.group = static_cast<int>(found[1]);
    s.tile = static_cast<int>(found[2]);
    return s;
}

// Walks the units of a share; rows without tiles are stepped over.
template <int kTile, int kGrain>
struct Walk {
    int r, group, tile;
    Span span;

    __device__ __forceinline__ void start(const KvAttendParams& p, const Share& s) {
        r = s.r;
        group = s.group;
        tile = s.tile;
        span = span_of<kTile, kGrain>(p, clamped_len(p, r, false));
    }
    // to the next unit; the share must hold one
    __device__ __forceinline__ void next(const KvAttendParams& p, int groups) {
        if (++tile < span.tiles) return;
        tile = 0;
        if (++group < groups) return;
        group = 0;
        do {
            span = span_of<kTile, kGrain>(p, clamped_len(p, ++r, false));
        } while (span.tiles == 0);
    }
};

// Contributors of a split row: CTAs first .. first + n - 1; the first holds its part in slot 1, the others
// in slot 0 (a CTA has at most one row that began before its share and one that goes on behind it).
struct Joint {
    int first, n;
};

__device__ __forceinline__ Joint joint_of(long long total, long long row_start, int tiles, int workers) {
    Joint j;
    j.first = share_owner(total, row_start, workers);
    j.n = share_owner(total, row_start + tiles - 1, workers) - j.first + 1;
    return j;
}

// Parts that one CTA adds up at most; more contributors are joined in groups of so many first, each by the
// last CTA of its group, then the groups' sums.  (One CTA reading all of 304 parts of 8 KB: about 20 us.)
constexpr int kJoinFan = 16;

__device__ __forceinline__ int part_slot(int cta, bool first) { return cta * 2 + (first ? 1 : 0); }

// Counts this CTA in and tells whether it is the last of n.  What the CTA wrote before is visible to the last.
__device__ __forceinline__ bool arrive_last(int* counter, int n, int* flag) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const int last = atomicAdd(counter, 1) == n - 1;
        if (last) *counter = 0;
        *flag = last;
    }
    __syncthreads();
    const bool last = *flag != 0;
    if (last) __threadfence();
    return last;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Weight of a part whose reference is m in a sum whose reference is M; nothing at all has m = -inf.
__device__ __forceinline__ float part_weight(float m, float M) { return m == -INFINITY ? 0.0f : exp2_fast(m - M); }

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// c += a b, 16 x 8 x 16, FP32 sums
template <bool kF16>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// {lo, hi} as a pair of 16-bit values
template <bool kF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (kF16)
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool kF16>
__device__ __forceinline__ float2 unpack2(uint32_t x) {
    if (kF16) return __half22float2(*reinterpret_cast<const __half2*>(&x));
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ float max4(float x) {   // over the four lanes of a fragment's row
    x = fmaxf(x, __shfl_xor_sync(kFull, x, 1));
    return fmaxf(x, __shfl_xor_sync(kFull, x, 2));
}
__device__ __forceinline__ float sum4(float x) {
    x += __shfl_xor_sync(kFull, x, 1);
    return x + __shfl_xor_sync(kFull, x, 2);
}

}  // namespace kv
}  // namespace qs
