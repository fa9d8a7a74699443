// qs_kv_join.cuh -- joins what a request made of its own tokens with its rows of the tokens that its group shares.
//
// o = sum_parts 2^{m - M} sums / sum_parts 2^{m - M} l over the parts of both, each one unsplit row in a store or a run of
// slots in the order of the tokens.  A warp takes a row (request and query head), or, where there are few rows and so many
// parts of each, a block of eight warps; either way a lane's loads of eight parts are in flight together.  A row is read
// once and o written once: some bytes from L2, and a chain of three latencies (the row's records, its parts' references, its parts).
#pragma once

#include "qs_kv_tiles.cuh"

namespace qs {
namespace kv {

struct PartList {
    const float* sums;       // rows of D
    const float4* ml;
    size_t row, step, step1; // the first part's row; rows between parts (from the second on), and from the first to the second
    size_t pair;             // rows between the two streams of a part
    int n, streams;
};

// The parts of a row: unsplit in the store, or in slots of `rows` rows from `worker` on.
__device__ __forceinline__ PartList part_list(int2 dir, const float* store, const float4* store_ml, size_t out_row, const float* part,
                                              const float4* part_ml, int rows, int row) {
    if (dir.x < 0) return {store, store_ml, out_row, 0, 0, 0, 1, 1};
    // the first is in slot 2 worker + 1, part i behind it in slot 2 (worker + i)
    return {part, part_ml, static_cast<size_t>(part_slot(dir.x, true)) * rows + row, 2 * static_cast<size_t>(rows),
            static_cast<size_t>(rows), 0, dir.y, 1};
}
__device__ __forceinline__ size_t part_row(const PartList& p, int i) {
    size_t at = p.row;
    if (p.streams == 2) {
        at += (i & 1) * p.pair;
        i >>= 1;
    }
    return i == 0 ? at : at + p.step1 + (i - 1) * p.step;
}

template <int D, bool kF16, int kWarpsPer>
__global__ void __launch_bounds__(kJoinWarps * 32) kv_join_shared_kernel(const KvAttendParams p, const JoinGeo g) {
    constexpr int kPieces = D / 128 > 0 ? D / 128 : 1, kLanes = D / 4 < 32 ? D / 4 : 32, kBatch = 8;
    constexpr int kRowsPer = kJoinWarps / kWarpsPer;
    __shared__ float4 s_ml[kJoinWarps], s_acc[kWarpsPer > 1 ? kJoinWarps : 1][D / 4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    chain_wait();
    const int rows = p.R * p.Hq, groups = p.Hkv * g.groups_per_kv;
    for (int row0 = blockIdx.x * kRowsPer; row0 < rows; row0 += gridDim.x * kRowsPer) {
        const int row = row0 + warp / kWarpsPer;
        const bool mine = row < rows;
        const int r = mine ? row / p.Hq : 0, h = mine ? row - r * p.Hq : 0, kv = h / g.G, in_kv = h - kv * g.G;
        const int4 rec = __ldcg(p.shared + r);
        const int n = clamped_len(p, r, false), begin = min(max(p.window > 0 && n > p.window ? n - p.window : 0, rec.x), n);
        const int group = kv * g.groups_per_kv + in_kv / g.per_group, at = rec.w + in_kv;
        PartList own{}, pre{};
        if (mine && begin < n)
            own = part_list(__ldcg(p.dir + static_cast<size_t>(r) * groups + group), p.store, p.store_ml, row, p.part,
                               reinterpret_cast<const float4*>(p.part_ml), g.rows, in_kv % g.per_group);
        if (mine && rec.x > 0) {
            int2 dir = __ldcg(p.pre_dir + rec.y + kv * rec.z + at / kv_shared_rows(D));
            const bool pair = dir.y < 0;   // two streams of one half
            dir.y = abs(dir.y);
            pre = part_list(dir, p.pre_store, p.pre_store_ml, row, p.pre_part, p.pre_ml, kv_shared_rows(D), at % kv_shared_rows(D));
            if (pair) {
                pre.streams = 2;
                pre.n *= 2;
                pre.pair = dir.x < 0 ? static_cast<size_t>(rows) : 128;
            }
        }
        const int first = warp % kWarpsPer, all = own.n + pre.n, count = all > first ? (all - first + kWarpsPer - 1) / kWarpsPer : 0;
        float Mo = -INFINITY, M = -INFINITY, L = 0.0f, Lo = 0.0f;
        float4 acc[kPieces] = {};
        for (int base = 0; base < count; base += 32) {
            const int many = min(32, count - base);
            float4 y = make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);   // a lane's part's
            if (lane < many) {
                const int i = first + (base + lane) * kWarpsPer;
                y = __ldcg(i < pre.n ? pre.ml + part_row(pre, i) : own.ml + part_row(own, i - pre.n));
            }
            float c = 0.0f;
            for (int j = 0; j < many; j += kBatch) {
                float4 v[kBatch][kPieces];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int i = first + (base + j + b) * kWarpsPer;
                    const bool on = j + b < many && lane < kLanes;
                    const float4* const src =
                        reinterpret_cast<const float4*>(i < pre.n ? pre.sums + part_row(pre, i) * D : own.sums + part_row(own, i - pre.n) * D) + lane;
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) v[b][k] = on ? __ldcg(src + k * 32) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
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
                    const float cb = __shfl_sync(kFull, c, j + b), ref = __shfl_sync(kFull, y.x, j + b);
                    if (ref == -INFINITY) continue;   // no token, and no sums
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
        // values and weights have references of their own where values carry powers of two
        auto put = [&](int piece, const float4& x) {
            const float inv = (Lo == 0.0f ? 0.0f : 1.0f / Lo) * (Mo == M ? 1.0f : exp2_fast(Mo - M));
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o) + static_cast<size_t>(row) * D + piece * 4) =
                make_uint2(pack2<kF16>(x.x * inv, x.y * inv), pack2<kF16>(x.z * inv, x.w * inv));
        };
        if constexpr (kWarpsPer == 1) {
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
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) {
                Mo = fmaxf(Mo, s_ml[w].x);
                M = fmaxf(M, s_ml[w].y);
            }
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (tid < D / 4) {
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
            __syncthreads();
        }
        if (mine && lane == 0 && first == 0 && p.lse) p.lse[row] = log_sum(M, L);
    }
}

template <int D, bool kF16>
cudaError_t launch_join_shared(const KvAttendParams& p, const JoinGeo& g, cudaStream_t stream) {
    // A warp a row where the rows keep every SM's warps busy; their parts are few then (two blocks' rows have at most a part
    // from each SM).
    const int sms = device_sm_count(), rows = p.R * p.Hq;
    if (rows < 8 * sms) return launch_chained(kv_join_shared_kernel<D, kF16, kJoinWarps>, rows, kJoinWarps * 32, 0, stream, true, p, g);
    const int blocks = (rows + kJoinWarps - 1) / kJoinWarps;
    return launch_chained(kv_join_shared_kernel<D, kF16, 1>, blocks, kJoinWarps * 32, 0, stream, true, p, g);
}

}  // namespace kv
}  // namespace qs
