// qs_kv_tiles.cuh -- what the attention kernels over the paged cache share: how the work is divided, how the
// parts of a row are joined, and the instructions that they use.
//
// A row of work is one request and one group of its heads; its unit is a tile of tokens, and kRowUnits more
// stand for what a row costs by itself (its queries, its end).  The units of all rows, request after
// request, are dealt out evenly: worker c of n takes a contiguous range of them, so that a long row is
// split and short ones are strung together, whatever the lengths are, and no length has to be known on
// the host.  Parts of a row that several workers share go to memory, and a second
// kernel, already placed and waiting when the first ends, joins them in the order of the tokens.  (Joined in
// the first kernel by the last worker of a row, 25 parts of 8 KB took 23 us of one CTA's latencies.)
// Where the table is so narrow that no row has more than kWholeTiles tiles, workers take whole rows in
// turn instead: nothing to sum up over the requests first, nothing to join (40 tokens cached: 4.1 us
// against 5.1 with heads, 7.4 against 11.4 with latents).
#pragma once

#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace kv {

// Tokens of a request that are seen: [begin, end); tiles start at base, a multiple of `grain`.
struct Span {
    int begin, end, base, tiles;
};

__device__ __forceinline__ int clamped_len(const KvAttendParams& p, int r, bool report) {
    const int n = p.lens[r];
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

constexpr int kWholeTiles = 4;
constexpr int kRowUnits = 1;

// A worker's share of the units, [u0, u1), and where it begins.  A worker goes through it from u0 to u1, in the order
// of rows and tokens, so the parts of a split row belong to workers in a row, in the order of its tokens.
struct Share {
    long long total;        // units of all rows
    long long u0, u1;
    int r, group, pos;      // where u0 is; tile t of a row is at pos kRowUnits + t
};

__device__ __forceinline__ long long share_start(long long total, int worker, int workers) {
    const long long q = total / workers, rem = total - q * workers;
    return q * worker + (worker < rem ? worker : rem);
}
// Worker whose share holds unit u.
__device__ __forceinline__ int share_owner(long long total, long long u, int workers) {
    const long long q = total / workers, rem = total - q * workers, cut = rem * (q + 1);
    return static_cast<int>(u < cut ? u / (q + 1) : rem + (u - cut) / q);
}

__device__ __forceinline__ int row_units(int tiles) { return tiles > 0 ? tiles + kRowUnits : 0; }

// All threads of the CTA; `groups` rows a request.  scratch: kThreads / 32 + 2 long longs of shared memory; *out too.
template <int kThreads, int kTile, int kGrain>
__device__ __forceinline__ void make_share(const KvAttendParams& p, int groups, int worker, long long* scratch, Share* out) {
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.R + kThreads - 1) / kThreads, r0 = min(p.R, tid * per), r1 = min(p.R, r0 + per);
    long long mine = 0;
    int tiles = 0;
    for (int r = r0; r < r1; ++r) {
        tiles = row_units(span_of<kTile, kGrain>(p, clamped_len(p, r, false)).tiles);
        mine += tiles;
    }
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
        const long long x = scratch[w];
        if (w < warp) before += x;
        all += x;
    }
    before -= mine;
    const long long total = all * groups, u0 = share_start(total, worker, p.workers), u1 = share_start(total, worker + 1, p.workers);
    if (tid == 0) {
        out->total = total;
        out->u0 = u0;
        out->u1 = u1;
    }
    const long long first = before * groups;
    if (u0 >= first && u0 < first + mine * groups) {
        long long at = u0 - first;
        int r = r0;
        if (per > 1)
            for (; r < r1; ++r) {
                tiles = row_units(span_of<kTile, kGrain>(p, clamped_len(p, r, false)).tiles);
                if (at < static_cast<long long>(tiles) * groups) break;
                at -= static_cast<long long>(tiles) * groups;
            }
        const int group = static_cast<int>(at / tiles);
        out->r = r;
        out->group = group;
        out->pos = static_cast<int>(at - static_cast<long long>(group) * tiles);
    }
    __syncthreads();
}

// Walks the units of a worker: those of its share, or, with p.whole_rows, every p.workers-th row.  Rows without
// tiles are stepped over.
template <int kTile, int kGrain>
struct Walk {
    int r, group, tile;
    int left;      // units to the share's end, this one among them; whole rows: the row
    Span span;

    // false: no tile at all
    __device__ __forceinline__ bool start(const KvAttendParams& p, const Share& s, int groups, int worker) {
        tile = 0;
        if (p.whole_rows) {
            left = worker - p.workers;
            return next_row(p, groups);
        }
        left = static_cast<int>(s.u1 - s.u0);
        if (left <= 0) return false;
        r = s.r;
        group = s.group;
        tile = s.pos - kRowUnits;
        span = span_of<kTile, kGrain>(p, clamped_len(p, r, false));
        if (tile < 0) {
            left += tile;
            tile = 0;
        }
        return left > 0;
    }
    __device__ __forceinline__ bool next_row(const KvAttendParams& p, int groups) {
        tile = 0;
        do {
            left += p.workers;
            if (left >= p.R * groups) return false;
            r = left / groups;
            group = left - r * groups;
            span = span_of<kTile, kGrain>(p, clamped_len(p, r, false));
        } while (span.tiles == 0);
        return true;
    }
    // to the next unit, if there is one
    __device__ __forceinline__ bool next(const KvAttendParams& p, int groups) {
        if (p.whole_rows) return ++tile < span.tiles || next_row(p, groups);
        if (--left <= 0) return false;
        if (++tile < span.tiles) return true;
        tile = 0;
        left -= kRowUnits;
        if (left <= 0) return false;
        if (++group < groups) return true;
        group = 0;
        do {
            span = span_of<kTile, kGrain>(p, clamped_len(p, ++r, false));
        } while (span.tiles == 0);
        return true;
    }
    // Whether this is the last unit of its row here.
    __device__ __forceinline__ bool ends(const KvAttendParams& p) const {
        return tile == span.tiles - 1 || (!p.whole_rows && left == 1);
    }
};

// A row that several workers share: the one that begins it holds its part in slot 1, the others in slot 0 (a worker has
// at most one row that began before its share and one that goes on behind it).
__device__ __forceinline__ int part_slot(int worker, bool first) { return worker * 2 + (first ? 1 : 0); }

// Parts of a row whose tile `tile` is where the worker's share ends, for the worker that begins the row.
__device__ __forceinline__ int row_parts(const KvAttendParams& p, const Share& s, int worker, int left, int tile, int tiles) {
    return share_owner(s.total, s.u1 - left - tile + tiles - 1, p.workers) - worker + 1;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Weight of a part whose reference is m in a sum whose reference is M; nothing at all has m = -inf.
__device__ __forceinline__ float part_weight(float m, float M) { return m == -INFINITY ? 0.0f : exp2_fast(m - M); }

// log of a sum of 2^z against the reference ref; the sum's exponent goes to the reference, so that log2f adds nothing to
// the rounding of the result.
__device__ __forceinline__ float log_sum(float ref, float sum) {
    if (sum == 0.0f) return -INFINITY;
    int e = 0;
    const float f = frexpf(sum, &e);   // infinities and NaN stay what they are
    return (ref + static_cast<float>(e) + log2f(f)) * 0.6931471805599453f;
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
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

// ---- joining the parts of split rows ------------------------------------------------------------------
// A part: the sums of values [rows][DV], and for each row the references of values and of weights, the sum of
// weights (for lse), and the sum that o is divided by.  The worker that begins a row has left the number of parts
// and the row.  An item is one head of a row of many parts, whose parts the block's warps share out, or eight
// heads of a row of few, one a warp: either way some dozen loads are in flight for each warp.  The kernel is a
// chain of latencies (which row an item is of, its parts, their sum), so each step asks for all that it needs
// at once.
struct JoinGeo {
    int columns;         // CTAs a worker has, each with its own heads (latents), else 1
    int rows;            // rows of a part
    int per_group;       // heads of a group
    int G, groups_per_kv;
};
constexpr int kJoinWarps = 8, kFewParts = 8;

__device__ __forceinline__ float warp_top(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kFull, x, o));
    return x;
}

template <int DV, bool kF16>
__global__ void __launch_bounds__(kJoinWarps * 32) kv_join_kernel(const KvAttendParams p, const JoinGeo g) {
    constexpr int kThreads = kJoinWarps * 32, kPer = (kKvWorkers + kThreads - 1) / kThreads;
    constexpr int kPieces = DV / 128 > 0 ? DV / 128 : 1, kLanes = DV / 4 < 32 ? DV / 4 : 32;   // a lane's float4 of a row
    constexpr int kBatch = DV >= 512 ? 4 : 8;                                                  // parts in flight for a warp
    __shared__ int s_warp[kJoinWarps];
    __shared__ int4 s_item;
    __shared__ float4 s_ml[kJoinWarps], s_acc[kJoinWarps][DV / 4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    chain_wait();
    // items of each worker, summed up
    int parts[kPer], rows[kPer], ends[kPer], mine_items = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int w = tid * kPer + k;
        parts[k] = w < p.workers ? __ldcg(p.split + w) : 0;
        rows[k] = w < p.workers ? __ldcg(p.split + kKvWorkers + w) : 0;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        mine_items += parts[k] < 2 ? 0 : g.columns * (parts[k] <= kFewParts ? (g.per_group + 7) / 8 : g.per_group);
        ends[k] = mine_items;
    }
    int before = mine_items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, before, o);
        if (lane >= o) before += y;
    }
    if (lane == 31) s_warp[warp] = before;
    __syncthreads();
    int items = 0;
    before -= mine_items;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
        if (w < warp) before += s_warp[w];
        items += s_warp[w];
    }
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int rel = item - before - (k > 0 ? ends[k - 1] : 0);
            if (rel >= 0 && item < before + ends[k]) s_item = make_int4(tid * kPer + k, parts[k], rows[k], rel);
        }
        __syncthreads();
        const int worker = s_item.x, n = s_item.y, row = s_item.z, rel = s_item.w;
        const bool few = n <= kFewParts;
        const int per = few ? (g.per_group + 7) / 8 : g.per_group;
        const int column = rel / per, h = few ? (rel - column * per) * 8 + warp : rel - column * per;
        // request and query head
        const int groups = p.Hq / g.G * g.groups_per_kv, r = row / groups, group = row - r * groups + column;
        const int kv = group / g.groups_per_kv, in_kv = (group - kv * g.groups_per_kv) * g.per_group + h;
        const bool mine = h < g.per_group && in_kv < g.G;
        // this warp's parts: i0, i0 + step ...
        const int i0 = few ? 0 : warp, step = few ? 1 : kJoinWarps, count = !mine ? 0 : few ? n : (n - warp + kJoinWarps - 1) / kJoinWarps;
        auto at = [&](int j) {
            const int i = i0 + j * step;
            return (static_cast<size_t>(part_slot(worker + i, i == 0)) * g.columns + column) * g.rows + h;
        };
        float Mo = -INFINITY, M = -INFINITY, L = 0.0f, Lo = 0.0f;
        float4 acc[kPieces] = {};
        for (int base = 0; base < count; base += 32) {
            const int many = min(32, count - base);
            float4 y = make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);   // a lane's part's
            if (lane < many) y = __ldcg(reinterpret_cast<const float4*>(p.part_ml) + at(base + lane));
            float c = 0.0f;
            for (int j = 0; j < many; j += kBatch) {
                float4 v[kBatch][kPieces];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const float4* const src = reinterpret_cast<const float4*>(p.part + at(base + j + b) * DV) + lane;
#pragma unroll
                    for (int k = 0; k < kPieces; ++k)
                        v[b][k] = j + b < many && lane < kLanes ? __ldcg(src + k * 32) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
                if (j == 0) {
                    const float to = fmaxf(Mo, warp_top(y.x)), tm = fmaxf(M, warp_top(y.y));
                    const float co = part_weight(Mo, to), cm = part_weight(M, tm), cy = part_weight(y.y, tm);
                    L = L * cm + warp_sum(y.z * cy);
                    Lo = Lo * cm + warp_sum(y.w * cy);
                    Mo = to;
                    M = tm;
                    c = part_weight(y.x, to);
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) acc[k] = make_float4(acc[k].x * co, acc[k].y * co, acc[k].z * co, acc[k].w * co);
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const float cb = __shfl_sync(kFull, c, j + b);
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) {
                        acc[k].x += cb * v[b][k].x;
                        acc[k].y += cb * v[b][k].y;
                        acc[k].z += cb * v[b][k].z;
                        acc[k].w += cb * v[b][k].w;
                    }
                }
            }
        }
        const size_t out = static_cast<size_t>(r) * p.Hq + kv * g.G + in_kv;
        // values and weights have references of their own where values carry powers of two
        auto put = [&](int piece, const float4& x) {
            const float inv = (Lo == 0.0f ? 0.0f : 1.0f / Lo) * (Mo == M ? 1.0f : exp2_fast(Mo - M));
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o) + out * DV + piece * 4) =
                make_uint2(pack2<kF16>(x.x * inv, x.y * inv), pack2<kF16>(x.z * inv, x.w * inv));
        };
        if (few) {
            if (mine && lane < kLanes)
#pragma unroll
                for (int k = 0; k < kPieces; ++k) put(k * 32 + lane, acc[k]);
        } else {
            if (lane < kLanes)
#pragma unroll
                for (int k = 0; k < kPieces; ++k) s_acc[warp][k * 32 + lane] = acc[k];
            if (lane == 0) s_ml[warp] = make_float4(Mo, M, L, Lo);
            __syncthreads();
            Mo = M = -INFINITY;
            L = Lo = 0.0f;
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) {
                Mo = fmaxf(Mo, s_ml[w].x);
                M = fmaxf(M, s_ml[w].y);
            }
            if (mine && tid < DV / 4) {
#pragma unroll
                for (int w = 0; w < kJoinWarps; ++w) {
                    const float4 z = s_acc[w][tid], y = s_ml[w];
                    const float co = part_weight(y.x, Mo), cm = part_weight(y.y, M);
                    L += y.z * cm;
                    Lo += y.w * cm;
                    x.x += co * z.x;
                    x.y += co * z.y;
                    x.z += co * z.z;
                    x.w += co * z.w;
                }
                put(tid, x);
            }
        }
        if (mine && lane == 0 && (few || warp == 0) && p.lse) p.lse[out] = log_sum(M, L);
        __syncthreads();
    }
}

template <int DV, bool kF16>
cudaError_t launch_join(const KvAttendParams& p, const JoinGeo& g, cudaStream_t stream) {
    return launch_chained(kv_join_kernel<DV, kF16>, 2 * device_sm_count(), kJoinWarps * 32, 0, stream, true, p, g);
}

}  // namespace kv
}  // namespace qs
