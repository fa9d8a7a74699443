// qs_kv_join.cuh -- joins what a request made of its own tokens with its rows of the tokens that its group shares.
//
// o = sum_parts 2^{m - M} sums / sum_parts 2^{m - M} l over the parts of both, each one unsplit row in a store or a run of
// slots in the order of the tokens.  A CTA takes eight rows (requests and query heads of one key head, as they lie in a block
// of rows), a warp 32 columns of them: the parts of shared tokens lie column by column, as the tensor memory's lanes
// write them, so that eight rows are a line.  Where there are few rows and so many parts of each, two to eight warps share the
// parts out and join in shared memory.  A row is read once and o written once: a chain of latencies (lengths and records, where
// the parts are, the parts, four at a time).  8192 rows of 128 take 6 us; with 64 registers and two CTAs an SM it took 2 more.
#pragma once

#include <type_traits>

#include "qs_kv_tiles.cuh"

namespace qs {
namespace kv {

constexpr int kJoinRows = 8, kJoinBatch = 4;   // rows of a CTA, parts in flight
// Warps that share a row's parts: 512 threads at most, which leave them their registers.
template <int D>
__host__ __device__ constexpr int join_shares() { return D == 64 ? 8 : D == 128 ? 4 : 2; }

// Whether a row's parts (KvAttendParams::dir), where it has any, lie with the workers that there are.
__device__ __forceinline__ bool has_place(const int2& dir, bool any, int workers) {
    return !any || (dir.x < 0 ? dir.x >= -2 && dir.y == (dir.x == -1 ? 1 : 0) : dir.y > 0 && dir.x + static_cast<unsigned>(dir.y) <= static_cast<unsigned>(workers));
}

template <int D, bool kF16, bool kMany>
__global__ void __launch_bounds__(D * (kMany ? join_shares<D>() : 1)) kv_join_shared_kernel(const KvAttendParams p, const JoinGeo g) {
    constexpr int kColumns = D / 32, kShares = kMany ? join_shares<D>() : 1, kRows = kv_shared_rows(D);
    __shared__ float4 s_ml[kShares][kJoinRows], s_acc[kMany ? kShares : 1][kMany ? kJoinRows : 1][D / 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = warp / kColumns;
    const int chunks = (p.R * g.G + kJoinRows - 1) / kJoinRows, groups = p.Hkv * g.groups_per_kv;
    const int kv = blockIdx.x / chunks, rr = lane & 7, v = (blockIdx.x - kv * chunks) * kJoinRows + rr;
    const int c = (warp % kColumns) * 8 + (lane >> 3);   // the lane's columns: 4 c ... 4 c + 3 and 16 more on
    const bool mine = v < p.R * g.G;
    const int r = mine ? v / g.G : 0, in_kv = mine ? v - r * g.G : 0;
    const size_t rows = static_cast<size_t>(p.R) * p.Hq, row = static_cast<size_t>(r) * p.Hq + kv * g.G + in_kv;
    int4 rec = __ldcg(p.shared + r);
    if (!groups_fit(p)) rec = make_int4(0, 0, 0, 0);
    // records and lengths are older than the kernels that this one waits for
    const int n = clamped_len(p, r, false), begin = min(max(p.window > 0 && n > p.window ? n - p.window : 0, rec.x), n);
    const bool has_own = mine && begin < n, has_pre = mine && rec.x > 0;
    int2 own_dir = make_int2(0, 0), pre_dir = own_dir;
    chain_wait();
    if (has_own) own_dir = __ldcg(p.dir + static_cast<size_t>(r) * groups + kv * g.groups_per_kv + in_kv / g.per_group);
    if (has_pre) pre_dir = __ldcg(p.pre_dir + rec.y + kv * rec.z + (rec.w + in_kv) / kRows);
    // Places that no worker has: calls that use the work space at once, from two streams.  They are not followed.
    const bool bad = !has_place(own_dir, has_own, p.workers) || !has_place(make_int2(pre_dir.x, abs(pre_dir.y)), has_pre, kKvSms) || pre_dir.x < -1;
    if (bad) {
        raise_status(p.status, QS_DEV_PAGES);
        own_dir = pre_dir = make_int2(0, 0);
    }
    // The parts' places, in float4 of references (of sums: D / 4 times as much, but that shared tokens' parts lie column by
    // column in a slot): 32 bits, and few instructions, whose latencies are what a join takes.  Part 0 of a split row is in the first
    // worker's slot 1, part k behind it in slot 0 of the k-th worker on.
    auto slot_of = [](int worker, int k) { return static_cast<unsigned>(part_slot(worker + k, k == 0)); };
    const bool done = own_dir.x == -2;   // by the kernel before
    if (__all_sync(kFull, done || !mine) && !kMany) return;
    const unsigned own_at = in_kv % g.per_group, pre_at = (rec.w + in_kv) % kRows, row32 = static_cast<unsigned>(row);
    const float4* const own_ml = own_dir.x < 0 ? p.store_ml : reinterpret_cast<const float4*>(p.part_ml);
    const float4* const own_sums = reinterpret_cast<const float4*>(own_dir.x < 0 ? p.store : p.part) + c;
    const bool pre_whole = pre_dir.x < 0;
    const float4* const pre_ml = pre_whole ? p.pre_store_ml : p.pre_ml;
    const float4* const pre_sums = reinterpret_cast<const float4*>(pre_whole ? p.pre_store : p.pre_part) + c * (pre_whole ? 1 : kRows);
    const int pair = pre_dir.y < 0 ? 1 : 0, pre_n = abs(pre_dir.y) << pair;   // two streams of one half
    const unsigned column = 4 * (pre_whole ? 1 : kRows);                     // to the lane's other columns
    auto load_own = [&](int k, float4& y, float4 (&x)[2]) {
        const unsigned ml = own_dir.x < 0 ? row32 : slot_of(own_dir.x, k) * g.rows + own_at;
        y = __ldcg(own_ml + ml);
        const float4* const src = own_sums + static_cast<size_t>(ml) * (D / 4);
        x[0] = __ldcg(src);
        x[1] = __ldcg(src + 4);
    };
    auto load_pre = [&](int i, float4& y, float4 (&x)[2]) {
        const int k = i >> pair, s = i & pair;
        const unsigned slot = pre_whole ? 0u : slot_of(pre_dir.x, k) * kRows;
        const unsigned at = pre_whole ? row32 + (s ? static_cast<unsigned>(rows) : 0u) : pre_at + s * 128u;
        y = __ldcg(pre_ml + slot + at);
        const float4* const src = pre_sums + (pre_whole ? static_cast<size_t>(at) * (D / 4) : static_cast<size_t>(slot) * (D / 4) + at);
        x[0] = __ldcg(src);
        x[1] = __ldcg(src + column);
    };
    float Mo = -INFINITY, M = -INFINITY, L = 0.0f, Lo = 0.0f;
    float4 acc[2] = {};
    // n parts at once: one reference for all, so that their weights do not wait for one another
    auto take = [&](auto count, const float4* y, const float4 (*x)[2]) {
        constexpr int n = decltype(count)::value;
        float to = Mo, tm = M;
#pragma unroll
        for (int b = 0; b < n; ++b) to = fmaxf(to, y[b].x), tm = fmaxf(tm, y[b].y);
        const float co = part_weight(Mo, to), cm = part_weight(M, tm);
        L *= cm;
        Lo *= cm;
#pragma unroll
        for (int k = 0; k < 2; ++k) acc[k] = make_float4(acc[k].x * co, acc[k].y * co, acc[k].z * co, acc[k].w * co);
        Mo = to;
        M = tm;
#pragma unroll
        for (int b = 0; b < n; ++b) {
            const float cy = part_weight(y[b].x, to), cl = part_weight(y[b].y, tm);
            if (y[b].x == -INFINITY && y[b].w == 0.0f) continue;   // no token, or none that weighs anything: no sums (NaN are none of these)
            L += y[b].z * cl;
            Lo += y[b].w * cl;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                acc[k].x += cy * x[b][k].x;
                acc[k].y += cy * x[b][k].y;
                acc[k].z += cy * x[b][k].z;
                acc[k].w += cy * x[b][k].w;
            }
        }
    };
    using One = std::integral_constant<int, 1>;
    using Batch = std::integral_constant<int, kJoinBatch>;
    const float4 none = make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);
    const int most = __reduce_max_sync(kFull, pre_n), most_own = __reduce_max_sync(kFull, own_dir.y);
    // own parts by the shares from the last on, so that the one that has the fewest of the others begins
    float4 y0[1] = {none}, x0[1][2];
    const int own_first = kShares - 1 - share;
    if (own_first < own_dir.y) load_own(own_first, y0[0], x0[0]);
#pragma unroll 1
    for (int i0 = share * kJoinBatch; i0 < most; i0 += kShares * kJoinBatch) {
        float4 y[kJoinBatch], x[kJoinBatch][2];
#pragma unroll
        for (int b = 0; b < kJoinBatch; ++b) {
            y[b] = none;
            if (i0 + b < pre_n) load_pre(i0 + b, y[b], x[b]);
        }
        take(Batch{}, y, x);
    }
    take(One{}, y0, x0);
#pragma unroll 1
    for (int i0 = own_first + kShares; i0 < most_own; i0 += kShares * kJoinBatch) {
        float4 y[kJoinBatch], x[kJoinBatch][2];
#pragma unroll
        for (int b = 0; b < kJoinBatch; ++b) {
            y[b] = none;
            if (i0 + b * kShares < own_dir.y) load_own(i0 + b * kShares, y[b], x[b]);
        }
        take(Batch{}, y, x);
    }
    if constexpr (kMany) {
        s_acc[share][rr][c] = acc[0];
        s_acc[share][rr][c + 4] = acc[1];
        if (c == 0) s_ml[share][rr] = make_float4(Mo, M, L, Lo);
        __syncthreads();
        if (share > 0) return;
        Mo = M = -INFINITY;
        L = Lo = 0.0f;
        acc[0] = acc[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kShares; ++w) {
            Mo = fmaxf(Mo, s_ml[w][rr].x);
            M = fmaxf(M, s_ml[w][rr].y);
        }
#pragma unroll
        for (int w = 0; w < kShares; ++w) {
            const float4 y = s_ml[w][rr];
            const float cl = part_weight(y.y, M), co = part_weight(y.x, Mo);
            L += y.z * cl;
            Lo += y.w * cl;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float4 z = s_acc[w][rr][c + 4 * k];
                acc[k].x += co * z.x;
                acc[k].y += co * z.y;
                acc[k].z += co * z.z;
                acc[k].w += co * z.w;
            }
        }
    }
    if (!mine || done) return;
    // values and weights have references of their own where values carry powers of two
    const float inv = (Lo == 0.0f ? 0.0f : 1.0f / Lo) * (Mo == M ? 1.0f : exp2_fast(Mo - M));
#pragma unroll
    for (int k = 0; k < 2; ++k)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o) + row * D + (c + 4 * k) * 4) =
            make_uint2(pack2<kF16>(acc[k].x * inv, acc[k].y * inv), pack2<kF16>(acc[k].z * inv, acc[k].w * inv));
    if (c == 0 && p.lse) p.lse[row] = log_sum(M, L);
}

template <int D, bool kF16>
cudaError_t launch_join_shared(const KvAttendParams& p, const JoinGeo& g, cudaStream_t stream) {
    const int items = (p.R * g.G + kJoinRows - 1) / kJoinRows * p.Hkv;
    // rows of half the SMs and fewer: a block's have a part from many SMs
    if (items < 2 * device_sm_count())
        return launch_chained(kv_join_shared_kernel<D, kF16, true>, items, D * join_shares<D>(), 0, stream, true, p, g);
    return launch_chained(kv_join_shared_kernel<D, kF16, false>, items, D, 0, stream, true, p, g);
}

}  // namespace kv
}  // namespace qs
