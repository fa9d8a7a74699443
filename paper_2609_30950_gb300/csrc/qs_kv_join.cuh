// qs_kv_join.cuh -- joins what a request made of its own tokens with its rows of the tokens that its group shares.
//
// o = sum_parts 2^{m - M} sums / sum_parts 2^{m - M} l over the parts of both, each one unsplit row in a store or a run of
// slots in the order of the tokens.  A CTA takes eight rows (requests and query heads of one key head, as they lie in a block
// of rows), a warp 32 columns of them: the parts of shared tokens lie column by column, as the tensor memory's lanes
// write them, so that eight rows are a line.  Where there are few rows and so many parts of each, two to eight warps share the
// parts out and join in shared memory.  A row is read once and o written once: a chain of latencies (lengths and records, where
// the parts are, the parts, four at a time).
#pragma once

#include "qs_kv_tiles.cuh"

namespace qs {
namespace kv {

// The parts of a row, addresses in float4: part i of the columns 4 c ... 4 c + 3 is at sums + at(i) + c * column.
struct PartList {
    const float4* sums;
    const float4* ml;
    size_t slot, offset, ml_slot, ml_offset;   // sizes of a slot, place of the row in one
    size_t pair, ml_pair;                      // from a part's first stream to its second
    int column, worker, n, streams;

    __device__ __forceinline__ size_t slot_of(int i) const { return worker < 0 ? 0 : part_slot(worker + i, i == 0); }
    __device__ __forceinline__ const float4* sums_at(int i) const {
        const int s = streams == 2 ? i & 1 : 0;
        return sums + slot_of(streams == 2 ? i >> 1 : i) * slot + offset + s * pair;
    }
    __device__ __forceinline__ const float4* ml_at(int i) const {
        const int s = streams == 2 ? i & 1 : 0;
        return ml + slot_of(streams == 2 ? i >> 1 : i) * ml_slot + ml_offset + s * ml_pair;
    }
};

constexpr int kJoinRows = 8, kJoinBatch = 4;   // rows of a CTA, parts in flight
// Warps that share a row's parts: 512 threads at most, which leave them their registers.
template <int D>
__host__ __device__ constexpr int join_shares() { return D == 64 ? 8 : D == 128 ? 4 : 2; }

template <int D, bool kF16, bool kMany>
__global__ void __launch_bounds__(D * (kMany ? join_shares<D>() : 1)) kv_join_shared_kernel(const KvAttendParams p, const JoinGeo g) {
    constexpr int kColumns = D / 32, kShares = kMany ? join_shares<D>() : 1, kRows = kv_shared_rows(D);
    __shared__ float4 s_ml[kShares][kJoinRows], s_acc[kMany ? kShares : 1][kMany ? kJoinRows : 1][D / 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = warp / kColumns;
    chain_wait();
    const int chunks = (p.R * g.G + kJoinRows - 1) / kJoinRows, groups = p.Hkv * g.groups_per_kv;
    const int kv = blockIdx.x / chunks, rr = lane & 7, v = (blockIdx.x - kv * chunks) * kJoinRows + rr;
    const int c = (warp % kColumns) * 8 + (lane >> 3);   // the lane's columns: 4 c ... 4 c + 3 and 16 more on
    const bool mine = v < p.R * g.G;
    const int r = mine ? v / g.G : 0, in_kv = mine ? v - r * g.G : 0;
    const size_t rows = static_cast<size_t>(p.R) * p.Hq, row = static_cast<size_t>(r) * p.Hq + kv * g.G + in_kv;
    const int4 rec = __ldcg(p.shared + r);
    const int n = clamped_len(p, r, false), begin = min(max(p.window > 0 && n > p.window ? n - p.window : 0, rec.x), n);
    const bool has_own = mine && begin < n, has_pre = mine && rec.x > 0;
    int2 own_dir = make_int2(0, 0), pre_dir = own_dir;
    if (has_own) own_dir = __ldcg(p.dir + static_cast<size_t>(r) * groups + kv * g.groups_per_kv + in_kv / g.per_group);
    if (has_pre) pre_dir = __ldcg(p.pre_dir + rec.y + kv * rec.z + (rec.w + in_kv) / kRows);
    PartList own{}, pre{};
    if (has_own) {
        const size_t at = in_kv % g.per_group;
        own = own_dir.x < 0
                  ? PartList{reinterpret_cast<const float4*>(p.store), p.store_ml, 0, row * (D / 4), 0, row, 0, 0, 1, -1, 1, 1}
                  : PartList{reinterpret_cast<const float4*>(p.part), reinterpret_cast<const float4*>(p.part_ml),
                             static_cast<size_t>(g.rows) * (D / 4), at * (D / 4), static_cast<size_t>(g.rows), at, 0, 0, 1, own_dir.x, own_dir.y, 1};
    }
    if (has_pre) {
        const size_t at = (rec.w + in_kv) % kRows;
        const int streams = pre_dir.y < 0 ? 2 : 1, many = abs(pre_dir.y) * streams;
        pre = pre_dir.x < 0
                  ? PartList{reinterpret_cast<const float4*>(p.pre_store), p.pre_store_ml, 0, row * (D / 4), 0, row, rows * (D / 4), rows, 1,
                             -1, many, streams}
                  : PartList{reinterpret_cast<const float4*>(p.pre_part), p.pre_ml, static_cast<size_t>(kRows) * (D / 4), at,
                             static_cast<size_t>(kRows), at, 128, 128, kRows, pre_dir.x, many, streams};
    }
    const int all = own.n + pre.n, most = __reduce_max_sync(kFull, all);
    float Mo = -INFINITY, M = -INFINITY, L = 0.0f, Lo = 0.0f;
    float4 acc[2] = {};
    for (int i0 = share * kJoinBatch; i0 < most; i0 += kShares * kJoinBatch) {
        float4 y[kJoinBatch], x[kJoinBatch][2];
#pragma unroll
        for (int b = 0; b < kJoinBatch; ++b) {
            const int i = i0 + b;
            const bool shared = i < pre.n;
            y[b] = make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);
            if (i >= all) continue;
            y[b] = __ldcg(shared ? pre.ml_at(i) : own.ml_at(i - pre.n));
            const float4* const src = shared ? pre.sums_at(i) : own.sums_at(i - pre.n);
            const int column = shared ? pre.column : own.column;
            x[b][0] = __ldcg(src + c * column);
            x[b][1] = __ldcg(src + (c + 4) * column);
        }
#pragma unroll
        for (int b = 0; b < kJoinBatch; ++b) {
            if (y[b].x == -INFINITY && y[b].w == 0.0f) continue;   // no token, or none that weighs anything: no sums (NaN are none of these)
            const float to = fmaxf(Mo, y[b].x), tm = fmaxf(M, y[b].y);
            const float co = part_weight(Mo, to), cy = part_weight(y[b].x, to), cm = part_weight(M, tm), cl = part_weight(y[b].y, tm);
            L = L * cm + y[b].z * cl;
            Lo = Lo * cm + y[b].w * cl;
            Mo = to;
            M = tm;
#pragma unroll
            for (int k = 0; k < 2; ++k)
                acc[k] = make_float4(acc[k].x * co + cy * x[b][k].x, acc[k].y * co + cy * x[b][k].y, acc[k].z * co + cy * x[b][k].z,
                                     acc[k].w * co + cy * x[b][k].w);
        }
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
    if (!mine) return;
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
