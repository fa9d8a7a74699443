// qs_kv_heads.cuh -- one new token of each request against keys and values per head.
//
// z_t = scale q.k_t, o = sum_t e^{z_t} v_t / sum_t e^{z_t}, in base 2 and against a running reference m:
// p_t = 2^{z_t - m}.  Every key and value is used once by the G query heads that share it, G
// operations a byte in 16 bits and 2 G in e4m3, so the cache's bytes are the bound far beyond the heads that share
// one in practice.  In 16 bits the kernel runs at 87 to 92 % of the copy rate (0.61 GB in 104 us, 1.08 GB in 174); codes take an
// instruction more each, and what issues is the bound (0.81 GB in 150 us, 79 %); few or short rows are bound by the
// latencies of two launches (1 request of 3001 tokens: 9.1 us).
//
// Tiles (qs_kv_tiles.cuh) of 64 tokens (128 in e4m3) of one request and key head, up to 16 query heads
// as the 16 rows of the matrix products; more query heads are further rows of work, which read the
// tile again.  A tile is four chunks, one a warp.  Each warp keeps its own ring of chunks (cp.async, zeros in
// place of what is not to be seen, rows swizzled so that neither the copies nor the fragment loads
// meet in a bank) and its own m, sums and o, so that warps meet only where a row of work ends: there
// they lay their o into the ring's slot just used and join it.
//  - m follows a row's maximum only when that has grown by more than 2^8: a vote, no reduction, on the
//    way.  p is at most 2^8 then, which changes nothing about its relative precision.
//  - p goes into the second product as hi + lo of two 16-bit values: one alone would add as much
//    error as the rounding of o itself.  With up to 8 heads lo takes the rows that are left over,
//    at no cost.
//  - products in f16 (f16 layers and e4m3): f16 ends at 2^-24, so a weight of the reference enters as 2^7, and
//    where the largest of a block of 16 tokens is under 2^-16 of it, the values' reference goes down to that one (o's sums
//    are FP32 and have room above), at most 2^48 under the highest it was.  Otherwise what lies far under one large
//    weight would be lost beside it, and where that one's value is zero it is all there is.  In a block a weight loses at most
//    2^-16 of the largest there.  (256 requests of 32 heads 172 us with and without; e4m3 above 150 against 145.)
//  - e4m3: codes are exact in f16, so both products run in f16.  q is scaled by a power of two for
//    each head first: entries over 2^-14 of the head's largest are exact, smaller ones are off by up to 2^-25 of the
//    largest (a score notices only where keys are next to nothing at q's largest entries); the keys' powers multiply the scores, and the values' powers are added to them in
//    base 2, with a reference of their own, so that p times the power stays in f16's range.
#pragma once

#include <cuda_bf16.h>

#include "qs_kv_join.cuh"

namespace qs {
namespace kv {

constexpr int kHeadRows = 16;
constexpr float kLazy = 8.0f;
// Products in f16: a weight of the reference enters as 2^kLift, one of 2^kLazy more as 2^15; the reference goes down to a
// block's largest where that is under 2^-kFar of it, but not under 2^-kDeep of the highest it was.
constexpr float kLift = 7.0f, kFar = 16.0f, kDeep = 48.0f;

// A word's codes 0, 1 and 2, 3 as pairs of f16.
__device__ __forceinline__ void e4m3_cvt(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}" : "=r"(lo), "=r"(hi) : "r"(w));
}

template <int D, bool kE4M3, int kStages>
struct HeadsShape {
    static constexpr int kWarps = 4, kThreads = kWarps * 32;
    static constexpr int kChunk = kE4M3 ? 32 : 16, kTile = kWarps * kChunk;
    static constexpr int kRow = kE4M3 ? D : 2 * D, kSeg = kRow / 16;
    static constexpr int kTensor = kChunk * kRow, kSlot = 2 * kTensor;   // 64 D bytes: 16 x D floats
    static constexpr int kRing = kWarps * kStages * kSlot;
    // queries: of the row that begins in a stage, and at 256 entries, too many to hold in registers, of this row
    static constexpr int kQBytes = kHeadRows * 2 * D, kQ = kRing, kQRow = kQ + kStages * kQBytes;
    static constexpr int kExps = kQRow + (D > 128 ? kQBytes : 0);
    static constexpr int kMl = kExps + (kE4M3 ? kWarps * kStages * 64 : 0);
    static constexpr int kQScale = kMl + kWarps * kHeadRows * 16;
    static constexpr int kMasks = kQScale + kHeadRows * 4;
    static constexpr int kScratch = kMasks + kWarps * kStages * 4 + 16 - (kWarps * kStages * 4) % 16;
    static constexpr int kShare = kScratch + 8 * 8;
    static constexpr int kBytes = kShare + (sizeof(Share) + 15) / 16 * 16;

    // byte of 16-byte piece `seg` of a row in a tile: eight rows at one piece, and two rows at four pieces,
    // lie in different banks
    static __device__ __forceinline__ int at(int row, int seg) {
        if (kSeg == 4) return row * kRow + ((seg ^ ((row >> 1) & 3)) << 4);
        return row * kRow + ((seg ^ (((row & 1) << 2) | ((row >> 1) & 3))) << 4);
    }
    static __device__ __forceinline__ int q_at(int row, int seg) {
        return row * 2 * D + ((seg ^ (((row & 1) << 2) | ((row >> 1) & 3))) << 4);
    }
    // float of (row, column) where a warp lays its o down
    static __device__ __forceinline__ int o_at(int row, int col) {
        return row * D + (col ^ (kE4M3 ? (row & 1) << 4 : (row & 3) << 3));
    }
};

// kShared: requests leave the tokens that they share to another kernel, and what they make of the others goes to memory, to be
// joined with that kernel's part.
template <int D, bool kF16, bool kE4M3, bool kHalf, int kStages, int kCtas, bool kShared>
__global__ void __launch_bounds__(128, kCtas) kv_heads_kernel(const KvAttendParams p, const int per_group, const int groups_per_kv) {
    using S = HeadsShape<D, kE4M3, kStages>;
    constexpr bool kProd16 = kF16 || kE4M3;         // products in f16
    constexpr bool kQInRegs = D <= 128;
    constexpr int kSteps = D / 16, kOut = D / 8;
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(128) char smem[];
    // kShared: nothing here needs the kernel before, which works on the shared tokens and has itself waited for all that came
    // before it: CTAs begin where its CTAs end, and the wait, for the kernel behind this one, comes last.
    if (kShared)
        chain_release();
    else
        chain_wait();   // and the kernel that joins split rows may take its place
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2, t4 = lane & 3;
    const int groups = p.Hkv * groups_per_kv, G = p.Hq / p.Hkv;

    Share& share = *reinterpret_cast<Share*>(smem + S::kShare);
    if (!p.whole_rows) {
        make_share<S::kThreads, S::kTile, S::kChunk, kShared>(p, groups, blockIdx.x, reinterpret_cast<long long*>(smem + S::kScratch), &share);
    } else if (kShared) {
        if (tid == 0) share.fits = groups_fit(p);
        __syncthreads();
    }
    int split = 0;   // parts of the row that this CTA begins and others end
    Walk<S::kTile, S::kChunk, kShared> cw;
    bool live = cw.start(p, share, groups, blockIdx.x);
    bool fetching = live;

    char* const ring = smem + warp * (kStages * S::kSlot);
    const uint32_t ring32 = smem_u32(ring);
    char* const exps = smem + S::kExps + warp * (kStages * 64);
    uint32_t* const masks = reinterpret_cast<uint32_t*>(smem + S::kMasks) + warp * kStages;
    const int page_mask = (1 << p.page_shift) - 1;
    const bool one_page = (1 << p.page_shift) >= S::kChunk;   // a chunk lies in one page
    constexpr uint32_t kAllTokens = S::kChunk == 32 ? 0xffffffffu : (1u << (S::kChunk & 31)) - 1;

    // ---- copies ----
    Walk<S::kTile, S::kChunk, kShared> fw = cw;
    int id = -1;
    auto look_up = [&]() {   // page of this lane's token in the chunk to come
        const int t = fw.span.base + (fw.tile * S::kWarps + warp) * S::kChunk + (one_page ? 0 : lane);
        id = -1;
        if (t < fw.span.end && (one_page || lane < S::kChunk))
            id = p.table[static_cast<size_t>(fw.r) * p.max_pages + (t >> p.page_shift)];
    };
    // Queries of a row that begins: thread tid copies pieces tid % 8 + 8 i of head tid / 8 (and finds them there).
    auto q_src = [&](const Walk<S::kTile, S::kChunk, kShared>& w, int* heads) {
        const int hk = w.group / groups_per_kv, part = w.group - hk * groups_per_kv;
        *heads = min(per_group, G - part * per_group);
        return static_cast<const uint16_t*>(p.q) + w.r * p.q_row + (hk * G + part * per_group + (tid >> 3)) * p.q_head;
    };
    bool row_begins = true;
    auto fetch = [&](int stage) {
        if (row_begins && p.q_aligned) {
            int heads;
            const uint16_t* const src = q_src(fw, &heads);
            const bool in = (tid >> 3) < heads;
#pragma unroll
            for (int i = 0; i < D / 64; ++i)
                cp_async16(smem_u32(smem + S::kQ + stage * S::kQBytes + S::q_at(tid >> 3, i * 8 + (tid & 7))),
                           in ? src + (i * 8 + (tid & 7)) * 8 : p.q, in);
        }
        const int t0 = fw.span.base + (fw.tile * S::kWarps + warp) * S::kChunk, t = t0 + lane;
        const int hk = fw.group / groups_per_kv;
        const bool seen = lane < S::kChunk && t >= fw.span.begin && t < fw.span.end;
        const bool there = id >= 0 && id < p.n_pages;
        if (seen && !there) raise_status(p.status, QS_DEV_PAGES);
        const uint32_t mask = __ballot_sync(kFull, seen && there);
        if (lane == 0) masks[stage] = mask;
        if (mask == 0) return;
        const uint32_t dst = ring32 + stage * S::kSlot;
        const long long head_row = (static_cast<long long>(there ? id : 0) * p.Hkv + hk) << p.page_shift;
        if (one_page) {
            const long long row0 = head_row + (t0 & page_mask);
            const char* const k = static_cast<const char*>(p.k) + row0 * S::kRow;
            const char* const v = static_cast<const char*>(p.v) + row0 * S::kRow;
            if (mask == kAllTokens) {
#pragma unroll
                for (int i = 0; i < S::kChunk * S::kSeg / 32; ++i) {
                    const int e = i * 32 + lane, to = S::at(e / S::kSeg, e % S::kSeg);
                    cp_async16(dst + to, k + e * 16);
                    cp_async16(dst + S::kTensor + to, v + e * 16);
                }
            } else {
#pragma unroll 1
                for (int i = 0; i < S::kChunk * S::kSeg / 32; ++i) {
                    const int e = i * 32 + lane, row = e / S::kSeg, to = S::at(row, e % S::kSeg);
                    const bool on = (mask >> row) & 1;
                    cp_async16(dst + to, on ? k + e * 16 : static_cast<const char*>(p.k), on);
                    cp_async16(dst + S::kTensor + to, on ? v + e * 16 : static_cast<const char*>(p.v), on);
                }
            }
            if (kE4M3 && lane < 16) {
                // exponents of four tokens a lane, keys' then values'; groups of four lie within a page of 4 and more
                const int g = lane & 7;
                if ((mask >> (4 * g)) & 15)
                    cp_async4(smem_u32(exps + stage * 64 + lane * 4), (lane < 8 ? p.k_exp : p.v_exp) + row0 + 4 * g);
            }
        } else {
            const long long mine = head_row + (t & page_mask);   // row of the pool that this lane's token is
            const long long mine_at = mine * S::kRow;
#pragma unroll 4
            for (int i = 0; i < S::kChunk * S::kSeg / 32; ++i) {
                const int e = i * 32 + lane, row = e / S::kSeg, seg = e % S::kSeg, to = S::at(row, seg);
                const bool on = (mask >> row) & 1;
                const long long at = __shfl_sync(kFull, mine_at, row) + seg * 16;
                cp_async16(dst + to, static_cast<const char*>(p.k) + (on ? at : 0), on);
                cp_async16(dst + S::kTensor + to, static_cast<const char*>(p.v) + (on ? at : 0), on);
            }
            if (kE4M3 && p.page_shift >= 2) {
                const int g = lane & 7;
                const long long four = __shfl_sync(kFull, mine, 4 * g);   // in one page
                if (lane < 16 && ((mask >> (4 * g)) & 15))
                    cp_async4(smem_u32(exps + stage * 64 + lane * 4), (lane < 8 ? p.k_exp : p.v_exp) + four);
            } else if (kE4M3 && seen && there) {
                exps[stage * 64 + lane] = p.k_exp[mine];
                exps[stage * 64 + 32 + lane] = p.v_exp[mine];
            }
        }
    };
    if (fetching) look_up();
    auto fetch_next = [&](int stage) {
        if (fetching) {
            fetch(stage);
            row_begins = fw.ends(p);
            fetching = fw.next(p, share, groups);
            if (fetching) look_up();
        }
        cp_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) fetch_next(s);

    // ---- products ----
    uint32_t qf[kQInRegs ? kSteps : 1][4];
    float o[kOut][4], m[2], mo[2], l[2], zs[2], high[2];   // high: e4m3, the highest mo so far
    int stage = 0, heads = 0, h0 = 0, began = -1;
    const char* qs = smem + S::kQ;   // this row's queries

    auto q_frag = [&](uint32_t (&a)[4], int ks) {
        if (!kE4M3) {
            ldsm4(a, smem_u32(qs) + S::q_at((lane & 7) + ((lane >> 3) & 1) * 8, ks * 2 + (lane >> 4)));
        } else {
            // columns t4 16 + 4 (ks % 4) ... + 3 of 64-column block ks / 4: the order in which a lane finds its codes
            const int col = (ks >> 2) * 64 + t4 * 16 + (ks & 3) * 4;
            const uint2 x = *reinterpret_cast<const uint2*>(qs + S::q_at(quad, col >> 3) + (col & 7) * 2);
            const uint2 y = *reinterpret_cast<const uint2*>(qs + S::q_at(quad + 8, col >> 3) + (col & 7) * 2);
            a[0] = x.x, a[1] = y.x, a[2] = x.y, a[3] = y.y;
        }
    };

    while (live) {
        cp_wait<kStages - 1>();
        if (began < 0) {   // a row of work begins: its queries
            began = cw.tile;
            const uint16_t* const src = q_src(cw, &heads);
            h0 = cw.group / groups_per_kv * G + cw.group % groups_per_kv * per_group;
            const int row = tid >> 3, piece = tid & 7;
            char* const landed = smem + S::kQ + stage * S::kQBytes;
            char* const kept = kQInRegs ? landed : smem + S::kQRow;
            if (kE4M3 || !kQInRegs || !p.q_aligned) {
                uint4 x[D / 64];
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    if (p.q_aligned) {
                        x[i] = *reinterpret_cast<const uint4*>(landed + S::q_at(row, i * 8 + piece));
                    } else {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint16_t* const e = src + (i * 8 + piece) * 8 + 2 * j;
                            w[j] = row < heads ? e[0] | static_cast<uint32_t>(e[1]) << 16 : 0u;
                        }
                        x[i] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
                if (kE4M3) {
                    unsigned big = 0;   // |q| as integers order as the numbers do
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) {
                        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) big = max(big, max(w[j] << 16 & 0x7fffffffu, w[j] & 0x7fff0000u));
                    }
#pragma unroll
                    for (int s = 1; s < 8; s <<= 1) big = max(big, __shfl_xor_sync(kFull, big, s));
                    const int e = big == 0 ? 0 : min(max(static_cast<int>(big >> 23) - 127, -126), 126);
                    const float inv = __uint_as_float(static_cast<unsigned>(127 - e) << 23);
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) {
                        uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 y = unpack2<false>(w[j]);
                            w[j] = pack2<true>(y.x * inv, y.y * inv);
                        }
                        x[i] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if (piece == 0)
                        reinterpret_cast<float*>(smem + S::kQScale)[row] = __uint_as_float(static_cast<unsigned>(127 + e) << 23);
                }
#pragma unroll
                for (int i = 0; i < D / 64; ++i) *reinterpret_cast<uint4*>(kept + S::q_at(row, i * 8 + piece)) = x[i];
            }
            __syncthreads();
            qs = kept;
            if (kQInRegs) {
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks) q_frag(qf[ks], ks);
                __syncthreads();   // a warp ahead may have this buffer refilled
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                m[s] = mo[s] = high[s] = -INFINITY;
                l[s] = 0.0f;
                zs[s] = p.scale * kLog2e;
                if (kE4M3) zs[s] *= reinterpret_cast<const float*>(smem + S::kQScale)[quad + 8 * s];
            }
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
        }
        __syncwarp();
        const uint32_t mask = masks[stage];
        const uint32_t kt = ring32 + stage * S::kSlot, vt = kt + S::kTensor;
        const char* const kb = ring + stage * S::kSlot;
#pragma unroll
        for (int sb = 0; sb < S::kChunk / 16; ++sb) {
            const uint32_t on = (mask >> (16 * sb)) & 0xffffu;
            if (on == 0) continue;
            float z[2][4] = {};
            if (!kE4M3) {
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks) {
                    uint32_t a[4], b[4];
                    if (!kQInRegs) q_frag(a, ks);
                    ldsm4(b, kt + S::at((lane & 7) + (lane >> 4) * 8, ks * 2 + ((lane >> 3) & 1)));
                    mma<kProd16>(z[0], kQInRegs ? qf[ks] : a, b[0], b[1]);
                    mma<kProd16>(z[1], kQInRegs ? qf[ks] : a, b[2], b[3]);
                }
            } else {
#pragma unroll
                for (int blk = 0; blk < D / 64; ++blk) {
                    uint4 w[2];
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
                        w[nt] = *reinterpret_cast<const uint4*>(kb + S::at(sb * 16 + nt * 8 + quad, blk * 4 + t4));
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        uint32_t a[4];
                        if (!kQInRegs) q_frag(a, blk * 4 + s);
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            const uint32_t c = s == 0 ? w[nt].x : s == 1 ? w[nt].y : s == 2 ? w[nt].z : w[nt].w;
                            uint32_t b0, b1;
                            e4m3_cvt(c, b0, b1);
                            mma<true>(z[nt], kQInRegs ? qf[blk * 4 + s] : a, b0, b1);
                        }
                    }
                }
            }
            bool unit = false;   // values with the power 2^0
            // scores in base 2 less their reference; y also carries the values' powers, which have one of their own
            float y[2][4];
            constexpr int kRowSets = kHalf ? 1 : 2;
            float mz[2], my[2];
#pragma unroll
            for (int r = 0; r < kRowSets; ++r) {
                mz[r] = m[r] == -INFINITY ? 0.0f : m[r];
                my[r] = mo[r] == -INFINITY ? 0.0f : mo[r];
            }
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                float ke[2] = {1.0f, 1.0f}, ve[2] = {0.0f, 0.0f};
                if (kE4M3) {
                    const int tok = sb * 16 + nt * 8 + 2 * t4;
                    const uint32_t kx = *reinterpret_cast<const uint16_t*>(exps + stage * 64 + tok);
                    const uint32_t vx = *reinterpret_cast<const uint16_t*>(exps + stage * 64 + 32 + tok);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        // 2^(k - 127), and k - 127 as a number; 255, not finite, becomes NaN: its carry is a mantissa bit
                        const uint32_t kj = (kx >> (8 * j)) & 255, vj = (vx >> (8 * j)) & 255;
                        ke[j] = __uint_as_float(kj << 23 | (kj + 1) >> 8);
                        unit = unit || vj == 127;
                        ve[j] = vj == 255 ? __uint_as_float(0x7fffffffu) : __uint_as_float(0x4B000000u | vj) - 8388735.0f;
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int r = 0; r < kRowSets; ++r) {
                        float& x = z[nt][2 * r + j];
                        const float scale = kE4M3 ? zs[r] * ke[j] : zs[r];
                        if (kE4M3) y[nt][2 * r + j] = fmaf(x, scale, ve[j] - my[r]);
                        x = fmaf(x, scale, -mz[r]);
                    }
            }
            if (on != 0xffffu) {
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (!((on >> (nt * 8 + 2 * t4 + (j & 1))) & 1)) z[nt][j] = y[nt][j] = -INFINITY;
            }
            // The references follow only what has outgrown them, or, in f16, what they stand far above: a row of whose
            // four lanes none is near.  A lane with nothing near is rare enough to look closer.
            float top[2], topo[2];
            bool grown, apart;
            auto compare = [&]() {
                grown = apart = false;
#pragma unroll
                for (int r = 0; r < kRowSets; ++r) {
                    top[r] = fmaxf(fmaxf(z[0][2 * r], z[0][2 * r + 1]), fmaxf(z[1][2 * r], z[1][2 * r + 1]));
                    if (kE4M3) topo[r] = fmaxf(fmaxf(y[0][2 * r], y[0][2 * r + 1]), fmaxf(y[1][2 * r], y[1][2 * r + 1]));
                    if (kF16) topo[r] = top[r] + (mz[r] - my[r]);
                    if (!kF16) grown = grown || top[r] > (m[r] == -INFINITY ? -INFINITY : kLazy);
                    if (kProd16) {
                        grown = grown || topo[r] > (mo[r] == -INFINITY ? -INFINITY : kLift + kLazy);
                        apart = apart || topo[r] < kLift - kFar;
                    }
                }
            };
            compare();
            bool follow = __any_sync(kFull, grown || apart || unit);
            if (kProd16 && follow) {
                if (__any_sync(kFull, unit)) {
                    // Zeros have that power too, however small the values beside them are: it is no measure of them, and
                    // what they add is nothing.  (64 requests of 48 heads 150 us; 188 where every value has that power.)
                    uint32_t any = 0;
#pragma unroll 1
                    for (int seg = 0; seg < S::kSeg; ++seg) {
                        const uint4 w = *reinterpret_cast<const uint4*>(kb + S::kTensor + S::at(sb * 16 + (lane & 15), seg));
                        any |= w.x | w.y | w.z | w.w;
                    }
                    const uint32_t zeros = __ballot_sync(kFull, (any & 0x7f7f7f7fu) == 0);
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if ((zeros >> (nt * 8 + 2 * t4 + (j & 1))) & 1) y[nt][j] = -INFINITY;
                    compare();
                }
                follow = __any_sync(kFull, grown);
#pragma unroll
                for (int r = 0; r < kRowSets; ++r) {
                    const bool deep = kE4M3 ? mo[r] <= high[r] - kDeep : mz[r] - my[r] > kLift + kDeep - 0.5f;
                    uint32_t near = __ballot_sync(kFull, topo[r] >= kLift - kFar || deep);
                    near |= near >> 1;
                    follow = follow || (~(near | near >> 2) & 0x11111111u) != 0;
                }
            }
            if (follow) {
#pragma unroll
                for (int r = 0; r < kRowSets; ++r) {
                    const float now = fmaxf(m[r], mz[r] + max4(top[r]));
                    float nowo = now;
                    if (kProd16) {
                        const float t = max4(topo[r]);
                        const bool moves = t > kLift + kLazy || t < kLift - kFar || mo[r] == -INFINITY;
                        nowo = mo[r];
                        if (moves && t > -INFINITY) nowo = fmaxf(my[r] + t - kLift, kE4M3 ? high[r] - kDeep : now - kLift - kDeep);
                        high[r] = fmaxf(high[r], nowo);
                    }
                    l[r] *= part_weight(m[r], now);
                    const float c = part_weight(mo[r], nowo);
                    const float mzr = now == -INFINITY ? 0.0f : now, myr = nowo == -INFINITY ? 0.0f : nowo;
                    const float dz = mzr - mz[r], dy = myr - my[r];
                    m[r] = now;
                    mo[r] = nowo;
                    mz[r] = mzr;
                    my[r] = myr;
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            z[nt][2 * r + j] -= dz;
                            if (kE4M3) y[nt][2 * r + j] -= dy;
                        }
#pragma unroll
                    for (int i = 0; i < kOut; ++i) {
                        o[i][2 * r] *= c;
                        o[i][2 * r + 1] *= c;
                        if (kHalf) o[i][2] *= c, o[i][3] *= c;
                    }
                }
            }
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int s = 0; s < kRowSets; ++s) {
                const float lift = kF16 ? exp2_fast(mz[s] - my[s]) : 1.0f;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    const float p0 = exp2_fast(z[nt][2 * s]), p1 = exp2_fast(z[nt][2 * s + 1]);
                    l[s] += p0 + p1;
                    const float w0 = kE4M3 ? exp2_fast(y[nt][2 * s]) : p0 * lift, w1 = kE4M3 ? exp2_fast(y[nt][2 * s + 1]) : p1 * lift;
                    const uint32_t h = pack2<kProd16>(w0, w1);
                    hi[2 * nt + s] = h;
                    if (!kE4M3) {
                        const float2 r = unpack2<kProd16>(h);
                        (kHalf ? hi : lo)[2 * nt + (kHalf ? 1 : s)] = pack2<kProd16>(w0 - r.x, w1 - r.y);
                    } else if (kHalf) {
                        hi[2 * nt + 1] = 0;
                    }
                }
            }
#pragma unroll
            for (int np = 0; np < D / 16; ++np) {
                if (!kE4M3) {
                    uint32_t b[4];
                    ldsm4t(b, vt + S::at((lane & 7) + ((lane >> 3) & 1) * 8, np * 2 + (lane >> 4)));
                    mma<kProd16>(o[2 * np], hi, b[0], b[1]);
                    mma<kProd16>(o[2 * np + 1], hi, b[2], b[3]);
                    if (!kHalf) {
                        mma<kProd16>(o[2 * np], lo, b[0], b[1]);
                        mma<kProd16>(o[2 * np + 1], lo, b[2], b[3]);
                    }
                } else if ((np & 1) == 0) {
                    // two pieces of 16 columns; a register holds columns 2c, 2c + 1 of two tokens
                    uint32_t b[4];
                    ldsm4t(b, vt + S::at(sb * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, np + (lane >> 4)));
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        uint32_t even[2], odd[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            e4m3_cvt(__byte_perm(b[2 * s + j], 0, 0x3120), even[j], odd[j]);
                        }
                        mma<true>(o[2 * (np + s)], hi, even[0], even[1]);
                        mma<true>(o[2 * (np + s) + 1], hi, odd[0], odd[1]);
                    }
                }
            }
        }

        if (cw.ends(p)) {
            // ---- the warps' parts of this row ----
            float* const mine = reinterpret_cast<float*>(ring + stage * S::kSlot);
            float4* const ml = reinterpret_cast<float4*>(smem + S::kMl);
            __syncwarp();
#pragma unroll
            for (int s = 0; s < (kHalf ? 1 : 2); ++s) {
                const int row = quad + 8 * s;
                const float sum = sum4(l[s]);
                if (t4 == 0) ml[warp * kHeadRows + row] = make_float4(mo[s], m[s], sum, 0.0f);
                if (!kE4M3) {
#pragma unroll
                    for (int i = 0; i < kOut; ++i) {
                        float2 x = make_float2(o[i][2 * s], o[i][2 * s + 1]);
                        if (kHalf) x.x += o[i][2], x.y += o[i][3];
                        *reinterpret_cast<float2*>(mine + S::o_at(row, i * 8 + 2 * t4)) = x;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kOut; i += 2)   // columns 4 t4 ... + 3 of a 16-column piece
                        *reinterpret_cast<float4*>(mine + S::o_at(row, i * 8 + 4 * t4)) =
                            make_float4(o[i][2 * s], o[i + 1][2 * s], o[i][2 * s + 1], o[i + 1][2 * s + 1]);
                }
            }
            __syncthreads();
            const float* const all = reinterpret_cast<const float*>(smem + stage * S::kSlot);
            const size_t out_row = static_cast<size_t>(cw.r) * p.Hq + h0;
            const bool joined = kShared && share.fits && p.shared[cw.r].x > 0;   // with shared tokens' parts
            auto finish = [&](int row, int col, float4 acc, float4 sums) {
                if (joined) {
                    reinterpret_cast<float4*>(p.store)[((out_row + row) * D + col) / 4] = acc;
                    if (col == 0) p.store_ml[out_row + row] = sums;
                    return;
                }
                // sums: references of values and weights, sum of weights
                const float inv = sums.z == 0.0f ? 0.0f : 1.0f / sums.z;
                const float c = kProd16 && sums.x != sums.y ? inv * exp2_fast(sums.x - sums.y) : inv;
                uint2 w;
                w.x = pack2<kF16>(acc.x * c, acc.y * c);
                w.y = pack2<kF16>(acc.z * c, acc.w * c);
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o) + (out_row + row) * D + col) = w;
                if (col == 0 && p.lse)
                    p.lse[out_row + row] = sums.z == 0.0f ? -INFINITY : (sums.y + log2f(sums.z)) * 0.6931471805599453f;
            };
            const bool whole = began == 0 && cw.tile == cw.span.tiles - 1;
            const int slot = part_slot(blockIdx.x, began == 0);
            for (int idx = tid; idx < heads * (D / 4); idx += S::kThreads) {
                const int row = idx / (D / 4), col = (idx - row * (D / 4)) * 4;
                float4 x[S::kWarps];
                float Mo = -INFINITY, M = -INFINITY, L = 0.0f;
#pragma unroll
                for (int w = 0; w < S::kWarps; ++w) {
                    x[w] = ml[w * kHeadRows + row];
                    Mo = fmaxf(Mo, x[w].x);
                    M = fmaxf(M, x[w].y);
                }
                float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int w = 0; w < S::kWarps; ++w) {
                    L += x[w].z * part_weight(x[w].y, M);
                    const float c = part_weight(x[w].x, Mo);
                    const float4 v = *reinterpret_cast<const float4*>(all + w * (kStages * S::kSlot / 4) + S::o_at(row, col));
                    acc.x += c * v.x;
                    acc.y += c * v.y;
                    acc.z += c * v.z;
                    acc.w += c * v.w;
                }
                const float4 sums = make_float4(Mo, M, L, L);
                if (whole) {
                    finish(row, col, acc, sums);
                } else {
                    reinterpret_cast<float4*>(p.part)[static_cast<size_t>(slot) * (kHeadRows * D / 4) + idx] = acc;
                    if (col == 0) reinterpret_cast<float4*>(p.part_ml)[slot * kHeadRows + row] = sums;
                }
            }
            if (kShared && tid == 0 && began == 0)
                p.dir[static_cast<size_t>(cw.r) * groups + cw.group] =
                    whole ? make_int2(joined ? -1 : -2, joined ? 1 : 0)   // -2: done
                          : make_int2(blockIdx.x, row_parts(p, share, blockIdx.x, cw.left, cw.tile, cw.span.tiles));
            if (!kShared && tid == 0 && !whole && began == 0) {
                split = row_parts(p, share, blockIdx.x, cw.left, cw.tile, cw.span.tiles);
                p.split[kKvWorkers + blockIdx.x] = cw.r * groups + cw.group;
            }
            began = -1;
            __syncthreads();   // parts and queries of the row are read
        }
        __syncwarp();
        fetch_next(stage);
        stage = stage + 1 == kStages ? 0 : stage + 1;
        live = cw.next(p, share, groups);
    }
    for (int r = blockIdx.x; r < p.R; r += p.workers)   // requests without tokens
        if (clamped_len(p, r, true) == 0 && !kShared) {
            uint4* out = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.o) + static_cast<size_t>(r) * p.Hq * D);
            for (int i = tid; i < p.Hq * (D / 8); i += S::kThreads) out[i] = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = tid; i < p.Hq; i += S::kThreads) p.lse[static_cast<size_t>(r) * p.Hq + i] = -INFINITY;
        }
    if (!kShared && !p.whole_rows && tid == 0) p.split[blockIdx.x] = split;
    cp_wait<0>();
    if (kShared) chain_enter();
}

template <int D, bool kF16, bool kE4M3, bool kHalf, int kStages, int kCtas, bool kShared>
cudaError_t launch_heads(KvAttendParams p, int per_group, int groups_per_kv, cudaStream_t stream) {
    using S = HeadsShape<D, kE4M3, kStages>;
    auto* kernel = kv_heads_kernel<D, kF16, kE4M3, kHalf, kStages, kCtas, kShared>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
    if (e != cudaSuccess) return e;
    const int ctas = device_sm_count() * kCtas;
    p.workers = ctas < kKvWorkers ? ctas : kKvWorkers;
    p.whole_rows = (static_cast<long long>(p.max_pages) << p.page_shift) <= kWholeTiles * S::kTile;
    if (p.whole_rows) {
        const long long rows = static_cast<long long>(p.R) * p.Hkv * groups_per_kv;
        if (rows < p.workers) p.workers = static_cast<int>(rows);
    }
    e = launch_chained(kernel, p.workers, S::kThreads, S::kBytes, stream, true, p, per_group, groups_per_kv);
    if (e != cudaSuccess || (p.whole_rows && !kShared)) return e;
    const JoinGeo geo{1, kHeadRows, per_group, p.Hq / p.Hkv, groups_per_kv};
    if constexpr (kShared) return launch_join_shared<D, kF16>(p, geo, stream);
    return launch_join<D, kF16>(p, geo, stream);
}

// Heads of a group: G / ceil(G / 16), rounded up; up to 8 of them leave half of the products' rows free.
template <int D, bool kF16, bool kE4M3, int kStages, int kCtas>
cudaError_t launch_heads_of(const KvAttendParams& p, cudaStream_t stream) {
    const int G = p.Hq / p.Hkv, n = (G + kHeadRows - 1) / kHeadRows, per = (G + n - 1) / n;
    if (p.shared)
        return per <= 8 ? launch_heads<D, kF16, kE4M3, true, kStages, kCtas, true>(p, per, n, stream)
                        : launch_heads<D, kF16, kE4M3, false, kStages, kCtas, true>(p, per, n, stream);
    return per <= 8 ? launch_heads<D, kF16, kE4M3, true, kStages, kCtas, false>(p, per, n, stream)
                    : launch_heads<D, kF16, kE4M3, false, kStages, kCtas, false>(p, per, n, stream);
}

}  // namespace kv
}  // namespace qs
