// qs_kv_latent.cuh -- one new token of each request against one latent vector a token, shared by all heads.
//
// z_t = scale q_h.c_t over the dk entries of c_t, o_h = sum_t e^{z_t} c_t[:dv] / sum_t e^{z_t}.  A token's
// 2 dk bytes meet 2 H (dk + dv) operations: 121 a byte at 64 heads of 512 + 64, more than the
// register-fed matrix products sustain beside the loads, so both products run on the tensor cores
// with their sums in tensor memory, and the cache's bytes stay the floor.
//
// A tile is 64 tokens, stored once in shared memory (rows of 128 bytes in blocks of 64 entries, 128-byte
// swizzle) and read in both directions:
//     S^T [64 tokens x heads] = C [64 x dk] Q^T        C with dk contiguous (K-major)
//     O^T [dv x heads]       += C^T [dv x 64] P        the same bytes with dv contiguous (M-major)
// Tokens and dv are the products' rows, so up to 64 heads are their columns and few heads waste nothing;
// more heads go to further CTAs that walk the same tiles at the same time and find them in L2.
//   warps 0-7   softmax: 16 tokens and half of the heads each from S^T, p to shared memory in 16 bits; at
//               a row's end o
//   warp 8      issues the products
//   warp 9      copies tiles that lie in one page, a box of the tensor map for each 64 entries; in parts, so that S need
//               not wait for the whole of a tile
//   warps 9-12  (10-12 where warp 9 copies boxes) copy a row's queries, and, 16 bytes at a time, tiles of shorter pages
// As in the kernel for heads, the softmax reference follows the maximum only when that has outgrown it by
// 2^8; all tokens of a row share one reference, so the eight warps vote.  In f16, which ends at 2^-24, a weight of the
// reference is 2^7, and the reference also goes down, to a tile whose largest weight is under 2^-16 of it: what
// lies far under one large weight would otherwise be lost beside it, and where that one's value is zero it is all
// there is (f16, 64 heads: 512 + 64 93 us with it, 91 without; 128 + 0 143 and 127, 256 + 64 95 and 93).  p has 16 bits in the second product
// and o is divided by the sum of the rounded p, so that the weights in use add up to one; lse comes from
// the sum before rounding.  That leaves o with 1.04 to 1.14 times the error of the same in 32 bits, rounded once
// (measured over the cases).  Carrying the remainder of p in a second product would cost a second pass over the tile: at 64 heads of 512 + 64, S
// reads 147 KB of operands from shared memory for each tile, at 128 bytes a cycle, O 98 KB and the remainder 98 KB
// more (105 us against 102 when it was tried, before the steps that made it 92).
// What bounds it: with 64 heads of 512 + 64, room for two tiles, whose copies, S, softmax and O follow one another (0.31 GB
// in 93 us, 49 % of the copy rate; 16 heads 72); with latents of 128 or 256, where three and four tiles fit, the softmax's
// chain (64 heads of 128 + 0: 127 us for 0.3 GB; 16 heads of 128 + 64 57, 77 %).
#pragma once

#include <cuda.h>   // CUtensorMap

#include "qs_kv_tiles.cuh"
#include "qs_tc.cuh"

namespace qs {
namespace kv {

constexpr int kLatTile = 64;
constexpr int kLatSoftmax = 8, kLatIssuer = kLatSoftmax, kLatCopiers = 4;   // warps
constexpr int kLatThreads = (kLatSoftmax + 1 + kLatCopiers) * 32;
constexpr int kBlockBytes = kLatTile * 128;   // 64 tokens x 64 entries
constexpr int kMaxStages = 4;
constexpr int kLatSmem = 227 * 1024;   // shared memory of an SM's only CTA
constexpr int kPartBlocks = 3, kMaxParts = 3;   // a tile is waited for in parts, so that S follows the copies
constexpr float kLazyLatent = 8.0f;
// f16: a weight of the reference is 2^kLiftLatent; the reference goes down where a tile's largest weight is under
// 2^-kFarLatent of it, but not under 2^-kDeepLatent of the highest it was.
constexpr float kLiftLatent = 7.0f, kFarLatent = 16.0f, kDeepLatent = 48.0f;

struct LatentGeo {
    int blocks;        // of 64 entries, the last may be half
    int stages, smem, groups, per_group, columns, workers;
    bool boxes;        // a tile lies in one page and is copied by the tensor map
};

// CTAs an SM that the kernel's registers are held to: two where shared memory has room for two with two tiles each.  (64 heads of
// 128 + 0, 0.3 GB: 166 us with one, 127 with two.)
__host__ __device__ constexpr int latent_ctas(int dv, int columns) { return dv == 128 || (dv == 256 && columns < 64) ? 2 : 1; }

// Shared memory behind the tiles, the queries and p.
struct LatentMisc {
    uint64_t full[kMaxStages][kMaxParts], free[kMaxStages], sready[2], qfull, qfree, pready, drain;
    uint64_t mask[kMaxStages];
    uint32_t flags[kMaxStages];   // of the tile: 1 its row begins here, 2 it ends here, 4 it is the last
    float top[4][64];
    float topr[4][64];   // f16, within a row: in the first the highest references so far
    alignas(16) uint32_t near[2][kLatSoftmax];   // f16: of a tile, heads with a weight of some size, a bit each
    float corr[64];   // what O's sums are multiplied by; warps read it at their own pace until the next vote
    float inv[64];    // at a row's end its references, then what o is multiplied by
    Share share;
    uint32_t tmem;
    int abort;
};
// two tiles of the widest latents stand beside 64 heads' queries and p
static_assert(2 * 9 * kBlockBytes + 9 * 64 * 128 + 64 * 128 + sizeof(LatentMisc) <= kLatSmem, "shared memory of an SM");

// Products of 16-bit types, FP32 sums: M x N, A optionally M-major.
__host__ __device__ constexpr uint32_t idesc_f16(bool f16, int M, int N, bool a_m_major) {
    return (1u << 4) | ((f16 ? 0u : 1u) << 7) | ((f16 ? 0u : 1u) << 10) | ((a_m_major ? 1u : 0u) << 15) |
           (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
// Operands in 128-byte rows with the 128-byte swizzle.  K-major: 1024 bytes (sbo) between groups of 8 rows.  M-major:
// lbo between blocks of 64 entries, 1024 (sbo) between groups of 8 of K.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return (addr >> 4) | (lbo >> 4) << 16; }
// Executed by a whole warp in step, issued by the lane whose `lead` is not 0: descriptors then stay in uniform
// registers (issued from a branch that one lane takes, each product took 85 cycles).
// Descriptors differ in their low words only (start address and lbo; all of shared memory fits in them).
template <uint32_t kHi>
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, bool accumulate, uint32_t lead) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 a, b;\nmov.b64 a, {%1, %6};\nmov.b64 b, {%2, %6};\nsetp.ne.b32 p, %4, 0;\n"
        "setp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate ? 1u : 0u), "r"(lead), "n"(kHi)
        : "memory");
}
__device__ __forceinline__ void commit_by(uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_u32(bar)),
        "r"(lead)
        : "memory");
}
__device__ __forceinline__ uint32_t elect_lane() {
    uint32_t lead;
    asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xffffffff;\nselp.u32 %0, 1, 0, q;\n}\n" : "=r"(lead));
    return lead;
}
// 16 lanes x 8 N columns: register 4 j + i of lane t is row t / 4 + 8 (i / 2), column 8 j + 2 (t % 4) + i % 2.
template <int N>
__device__ __forceinline__ void tmem_ld_rows(uint32_t at, float (&v)[4 * N]) {
    static_assert(N == 1 || N == 2 || N == 4, "columns in eights");
    uint32_t r[4 * N];
    if constexpr (N == 1)
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];\ntcgen05.wait::ld.sync.aligned;\n"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
    else if constexpr (N == 2)
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\ntcgen05.wait::ld.sync.aligned;\n"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(at) : "memory");
    else
        asm volatile(
            "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
            "tcgen05.wait::ld.sync.aligned;\n"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
              "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
            : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) v[i] = __uint_as_float(r[i]);
}
// A box of the pool, 64 entries wide, to shared memory; its bytes count towards the barrier's phase.  Executed by a
// warp in step and issued by its leading lane, as the products are (lanes with boxes of their own take turns of
// some 200 cycles).
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int col, int row, uint32_t bar, uint32_t lead) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.b32 q, %5, 0;\n"
        "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n}\n" ::"r"(dst),
        "l"(map), "r"(col), "r"(row), "r"(bar), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];\n" ::"l"(map) : "memory"); }
__device__ __forceinline__ void mbar_arrive_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void stmatrix4t(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
__device__ __forceinline__ void stmatrix2t(uint32_t at, uint32_t a, uint32_t b) {
    asm volatile("stmatrix.sync.aligned.m8n8.x2.trans.shared.b16 [%0], {%1,%2};" ::"r"(at), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
// An arrival (of those that the barrier was told to expect) when this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
// Whether a phase of a barrier is complete, for the whole warp alike; one lane looks for all.  (With this and phases that
// are kept, not divided out of the tile's number, 64 requests of 64 heads of 128 + 0, up to 36000 tokens, took 166 us for
// 191.)
__device__ __forceinline__ bool warp_look(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.eq.u32 q, %3, 0;\nsetp.ne.u32 p, %3, %3;\n"
        "@q mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(threadIdx.x & 31) : "memory");
    const bool done = __any_sync(kFull, ok != 0);
    __syncwarp();   // what the phase's arrivals made visible to one lane is there for all
    return done;
}
// The same without waiting a while in hardware.
__device__ __forceinline__ bool warp_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.eq.u32 q, %3, 0;\nsetp.ne.u32 p, %3, %3;\n"
        "@q mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(threadIdx.x & 31) : "memory");
    const bool done = __any_sync(kFull, ok != 0);
    __syncwarp();   // what the phase's arrivals made visible to one lane is there for all
    return done;
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;\n" ::: "memory"); }
__device__ __forceinline__ bool softmax_any(bool x) {
    int any;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %1, 0;\nbar.red.or.pred q, 1, 256, p;\nselp.s32 %0, 1, 0, q;\n}\n"
                 : "=r"(any) : "r"(static_cast<int>(x)) : "memory");
    return any != 0;
}

// Waits for a phase of a barrier; gives up after the limit, or at once where another role has.  Every role
// runs to its end all the same (so that no one waits for a warp that left), without starting copies or
// products any more.
// Whole warps wait, and a warp's lanes agree on the answer.
__device__ __forceinline__ bool role_wait(uint64_t* bar, uint32_t parity, volatile int* abort, const KvAttendParams& p) {
    for (int it = 0; it < p.wait_polls; ++it) {
        if (warp_look(bar, parity)) return true;
        if (__any_sync(kFull, *abort)) break;
    }
    if (!*abort) raise_status(p.status, QS_DEV_TIMEOUT);
    *abort = 1;
    return false;
}

template <int DV, int kN, bool kF16>
__global__ void __launch_bounds__(kLatThreads, latent_ctas(DV, kN)) kv_latent_kernel(const KvAttendParams p, const LatentGeo g,
                                                                const __grid_constant__ CUtensorMap map) {
    using W = Walk<kLatTile, kLatTile>;   // tiles start at multiples of a tile: a copy lies in one page
    constexpr int kOCols = DV / 128 * kN, kCols = kOCols + 2 * kN;
    constexpr int kAlloc = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    constexpr int kPer = kN / 8;   // heads a lane holds: 2 of each 8 of its warp's half
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(1024) char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    char* const tiles = smem;
    char* const queries_at = tiles + g.stages * g.blocks * kBlockBytes;
    char* const probs = queries_at + g.blocks * kN * 128;
    LatentMisc& x = *reinterpret_cast<LatentMisc*>(probs + kN * 128);
    const int worker = blockIdx.x / g.groups, group = blockIdx.x - worker * g.groups;
    const int h0 = group * g.per_group, heads = min(g.per_group, p.Hq - h0);
    const int askers = g.boxes ? kLatCopiers - 1 : kLatCopiers;   // warps that copy queries
    chain_enter();

    if (g.boxes && warp == kLatIssuer + 1) prefetch_map(&map);
    if (warp == kLatIssuer) {
        tc::tmem_alloc(&x.tmem, kAlloc);
        tc::tmem_relinquish();
        chain_release();   // the kernel that joins split rows may take its place; one with tensor memory no sooner
    }
    if (tid == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            for (int k = 0; k < kMaxParts; ++k) tc::mbar_init(&x.full[s][k], g.boxes ? 1 : kLatCopiers * 33);
            tc::mbar_init(&x.free[s], 1);
        }
        tc::mbar_init(&x.sready[0], 1);
        tc::mbar_init(&x.sready[1], 1);
        tc::mbar_init(&x.qfull, askers * 33);
        tc::mbar_init(&x.qfree, 1);
        tc::mbar_init(&x.pready, kLatSoftmax);
        tc::mbar_init(&x.drain, 1);
        tc::mbar_fence_init();
        x.abort = 0;
    }
    if (!p.whole_rows) make_share<kLatThreads, kLatTile, kLatTile>(p, 1, worker, reinterpret_cast<long long*>(x.top), &x.share);
    const Share& share = x.share;
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = x.tmem;
    volatile int* const abort = &x.abort;
    W w;
    bool live = w.start(p, share, 1, worker);
    int split = 0;   // parts of the row that this CTA begins and others end
    int copied = 0;  // tiles whose copies have been started
    constexpr int kParts = (DV / 64 + kPartBlocks) / kPartBlocks;   // with or without a block behind the values

    if (live && warp > kLatIssuer) {
        // ---- copies ----
        const int pw = warp - kLatIssuer - 1, page_mask = (1 << p.page_shift) - 1;
        const bool asks = !g.boxes || pw > 0, copier = !g.boxes || pw == 0;
        // of a tile's tokens, the one whose page a lane looks up, and those that are with it
        const int from = g.boxes ? 0 : pw * 16 + lane, tokens = g.boxes ? kLatTile : 1;
        const bool looks = copier && (g.boxes || lane < 16);
        auto look_up = [&](const W& at) {
            const int t = at.span.base + at.tile * kLatTile + from;
            return looks && t < at.span.end ? p.table[static_cast<size_t>(at.r) * p.max_pages + (t >> p.page_shift)] : -1;
        };
        const uint32_t lead = elect_lane();
        // a thread copies one of eight pieces of every block of its heads
        auto queries = [&](int r) {
            const int sg = lane & 7;
            for (int h = (warp - kLatIssuer - 1 - kLatCopiers + askers) * 4 + (lane >> 3); h < kN; h += askers * 4) {
                const uint16_t* const q = static_cast<const uint16_t*>(p.q) + r * p.q_row + (h0 + h) * p.q_head + sg * 8;
                uint32_t to = smem_u32(queries_at + h * 128 + ((sg ^ (h & 7)) << 4));
                for (int b = 0; b < g.blocks; ++b, to += kN * 128) {
                    const bool in = h < heads && b * 64 + sg * 8 < p.dk;
                    if (p.q_aligned) {
                        cp_async16(to, in ? q + b * 64 : p.q, in);
                    } else {
                        uint16_t v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = in ? q[b * 64 + k] : 0;
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v[0] | v[1] << 16),
                                     "r"(v[2] | v[3] << 16), "r"(v[4] | v[5] << 16), "r"(v[6] | v[7] << 16) : "memory");
                    }
                }
            }
        };
        auto queries_done = [&]() {
            cp_async_arrive(&x.qfull);
            __syncwarp();
            if (lane == 0) mbar_arrive(&x.qfull);
        };
        int id = look_up(w), s = 0, phase = 0, rows = 0;   // rows: that have waited for the queries of the one before
        if (asks) {
            queries(w.r);
            queries_done();
        }
        bool begins = true, ok = true;   // ok: no wait has been given up
        for (int i = 0; live; ++i) {
            const int r = w.r, t = w.span.base + w.tile * kLatTile + from;
            // pages that hold nothing in the window are not looked at (a program with tables of its own may have taken
            // them back)
            const bool wanted = looks && t < w.span.end && t + tokens > w.span.begin;
            const bool there = wanted && id >= 0 && id < p.n_pages;
            if (wanted && !there) raise_status(p.status, QS_DEV_PAGES);
            const long long row = there ? (static_cast<long long>(id) << p.page_shift) + (t & page_mask) : 0;
            const uint32_t tile = smem_u32(tiles + s * g.blocks * kBlockBytes);
            const bool first = begins;
            begins = w.ends(p);
            W after = w;
            const bool more = after.next(p, share, 1);
            uint64_t mask = 0;   // tokens that are seen: lanes take two each
            if (g.boxes) {
                const int begin = w.span.begin - w.span.base - w.tile * kLatTile, end = w.span.end - w.span.base - w.tile * kLatTile;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int u = lane + 32 * k;
                    mask |= static_cast<uint64_t>(__ballot_sync(kFull, u >= begin && u < end && there)) << (32 * k);
                }
            }
            if (copier && i >= g.stages) ok = ok && role_wait(&x.free[s], phase ^ 1, abort, p);
            if (pw == 0 && lane == 0 && ok)
                *reinterpret_cast<volatile uint32_t*>(&x.flags[s]) = (first ? 1u : 0u) | (begins ? 2u : 0u) | (more ? 0u : 4u);
            if (g.boxes) {
                if (copier && ok) {
                    copied = i + 1;
                    if (lane == 0) *reinterpret_cast<volatile uint64_t*>(&x.mask[s]) = mask;
                    for (int k = 0; k < kParts; ++k) {
                        const int b0 = k * kPartBlocks, many = min(kPartBlocks, g.blocks - b0);
                        if (lane == 0) mbar_arrive_expect(&x.full[s][k], there ? many * kBlockBytes : 0);
                        __syncwarp();
                        const uint32_t bar = smem_u32(&x.full[s][k]);
#pragma unroll
                        for (int b = 0; b < kPartBlocks; ++b)
                            if (there && b < many)
                                tma_box(tile + (b0 + b) * kBlockBytes, &map, (b0 + b) * 64, static_cast<int>(row), bar, lead);
                    }
                }
            } else {
                const uint32_t on = __ballot_sync(kFull, there);
                if (lane == 0) reinterpret_cast<volatile uint16_t*>(&x.mask[s])[pw] = static_cast<uint16_t>(on);
                const char* src[4];
                const int seg = lane & 7, row0 = lane >> 3;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    src[k] = static_cast<const char*>(p.k) + __shfl_sync(kFull, row, k * 4 + row0) * (2 * p.dk) + seg * 16;
                const uint32_t to = tile + (pw * 16 + row0) * 128;
                for (int part = 0; part < kParts; ++part) {
                    for (int b = part * kPartBlocks; ok && b < min(g.blocks, (part + 1) * kPartBlocks); ++b)
                        if (b * 64 + seg * 8 < p.dk) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int u = k * 4 + row0;
                                cp_async16(to + b * kBlockBytes + k * 512 + ((seg ^ (u & 7)) << 4), src[k] + b * 128, (on >> u) & 1);
                            }
                        }
                    cp_async_arrive(&x.full[s][part]);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&x.full[s][part]);
                }
            }
            w = after;
            live = more;
            if (live) id = look_up(w);
            if (first && i > 0 && asks) {
                // S of the row before is done with its queries
                ok = ok && role_wait(&x.qfree, rows++ & 1, abort, p);
                if (ok) queries(r);
                queries_done();
            }
            if (++s == g.stages) s = 0, phase ^= 1;
        }
        cp_commit();
        cp_wait<0>();
    } else if (live && warp == kLatIssuer) {
        // ---- products ----
        constexpr uint32_t idS = idesc_f16(kF16, 64, kN, false), idO = idesc_f16(kF16, 128, kN, true);
        constexpr int kMain = DV / 64;   // blocks of values; behind them a block, or half of one, or none
        const uint32_t lead = elect_lane(), tile_bytes = g.blocks * kBlockBytes;
        const uint32_t t32 = smem_u32(tiles), dq = desc_lo(smem_u32(queries_at), 16), dp = desc_lo(smem_u32(probs), 16);
        const int rope = (p.dk - DV) / 16;
        int ss = 0, so = 0;   // stages of the tiles whose S and whose O come next
        auto block = [&](int b, uint32_t a0, uint32_t d, int steps) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < steps)
                    mma_f16_ss<kDescHi>(d, a0 + (b * kBlockBytes + k * 32) / 16, dq + (b * kN * 128 + k * 32) / 16, idS, b > 0 || k > 0, lead);
        };
        auto scores = [&](int i, int part) {
            tc::fence_async_smem();   // the copies' writes, for the tensor core's reads
            tc::fence_after_sync();
            const uint32_t d = tmem + kOCols + (i & 1) * kN, a0 = desc_lo(t32 + ss * tile_bytes, 16);
#pragma unroll
            for (int k = 0; k < kParts; ++k)
                if (k == part)
#pragma unroll
                    for (int b = k * kPartBlocks; b < (k + 1) * kPartBlocks && b < kMain; ++b) block(b, a0, d, 4);
            if (part == kParts - 1 && rope) block(kMain, a0, d, rope);
        };
        auto values = [&](bool begins) {
            tc::fence_after_sync();
            const uint32_t a0 = desc_lo(t32 + so * tile_bytes, kBlockBytes);
#pragma unroll
            for (int c = 0; c < DV / 128; ++c)
#pragma unroll
                for (int k = 0; k < kLatTile / 16; ++k)
                    mma_f16_ss<kDescHi>(tmem + c * kN, a0 + (2 * c * kBlockBytes + k * 2048) / 16, dp + k * 2, idO, !begins || k > 0, lead);
            commit_by(&x.free[so], lead);
            so = so + 1 == g.stages ? 0 : so + 1;
        };
        // S runs one tile ahead of O, a part at a time as the parts come, and never makes O wait for it: with two
        // tiles in flight the copy of the next one waits for O
        int is = 0, part = 0, io = 0, full_phase = 0, q_phase = 0;   // tiles whose S and whose O have been issued
        uint32_t now = 0, before = 0;   // flags of the tiles is and is - 1
        bool more = true;
        while (more || io < is) {
            // Whichever can go first.  The loop that waits is a small one of its own: with the products' code inside it
            // each look took 450 cycles (64 requests of 64 heads of 512 + 64: 101 us so, 95 now).
            bool o_next = false, s_next = false;
            const bool o_open = io < is, s_open = more && is <= io + 1;
            int idle = 0;
#pragma unroll 1
            for (;; ++idle) {
                o_next = o_open && warp_test(&x.pready, io & 1);
                if (o_next) break;
                s_next = s_open && warp_test(&x.full[ss][part], full_phase);
                if (s_next && part == 0)
                    s_next = !(*reinterpret_cast<volatile uint32_t*>(&x.flags[ss]) & 1) || warp_test(&x.qfull, q_phase);
                if (s_next) break;
                if (__any_sync(kFull, idle > p.wait_polls || *abort)) break;
            }
            if (o_next) {
                // the tile before the one whose S is under way, or has just been issued
                values((io + 1 == is && part == 0 ? now : before) & 1);
                ++io;
            } else if (s_next) {
                if (part == 0) {
                    before = now;
                    now = *reinterpret_cast<volatile uint32_t*>(&x.flags[ss]);
                    q_phase ^= now & 1;
                }
                scores(is, part);
                if (++part == kParts) {
                    commit_by(&x.sready[is & 1], lead);
                    if (now & 2) commit_by(&x.qfree, lead);
                    more = !(now & 4);
                    ++is;
                    part = 0;
                    if (++ss == g.stages) ss = 0, full_phase ^= 1;
                }
            } else {
                if (!*abort) raise_status(p.status, QS_DEV_TIMEOUT);
                *abort = 1;
                break;
            }
        }
    } else if (live && warp < kLatIssuer) {
        // ---- softmax ----
        const int quad = lane >> 2, t4 = lane & 3, sub = warp & 3, c0 = (warp >> 2) * (kN / 2);   // token quarter, first head
        const uint32_t tlane = tmem + (static_cast<uint32_t>(32 * sub) << 16);
        const uint32_t p32 = smem_u32(probs);
        const float zs = p.scale * kLog2e;
        // sums of p before and after its rounding
        float m[kPer], l[kPer], lr[kPer];
        int prev = 0, prev_phase = 0, s = 0, phase = 0, began = 0;   // prev: stage of the tile before
        constexpr uint32_t kHeads = 0xffffffffu >> (32 - 4 * kPer);   // bits of a warp's heads
        constexpr float kAbove = kF16 ? kLazyLatent + kLiftLatent : kLazyLatent, kBelow = kLiftLatent - kFarLatent;
        bool begins = true;
        // k: head c0 + 8 (k / 2) + 2 t4 + k % 2, at tokens quad and quad + 8 of the quarter
        auto head = [&](int k) { return c0 + 8 * (k >> 1) + 2 * t4 + (k & 1); };
        for (int i = 0; live; ++i) {
            const bool ends = w.ends(p);
            if (begins) {
                began = w.tile;
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    m[k] = -INFINITY, l[k] = lr[k] = 0.0f;
                    if (kF16 && sub == 0 && quad == 0) x.topr[0][head(k)] = -INFINITY;
                }
            }
            role_wait(&x.full[s][0], phase, abort, p);
            role_wait(&x.sready[i & 1], (i >> 1) & 1, abort, p);
            tc::fence_after_sync();
            float z[2 * kPer];
            tmem_ld_rows<kN / 16>(tlane + kOCols + (i & 1) * kN + c0, z);
            const uint64_t seen = *reinterpret_cast<volatile uint64_t*>(&x.mask[s]);
            const uint32_t on = static_cast<uint32_t>(seen >> (16 * sub)) & 0xffffu;
            if (g.boxes && seen != ~0ull) {
                // what a box brought beside the tokens that are seen, or left as it was, must not meet p = 0 as NaN
                for (int u = warp; u < kLatTile; u += kLatSoftmax)
                    if (!((seen >> u) & 1))
                        for (int e = lane; e < DV / 8; e += 32)
                            *reinterpret_cast<uint4*>(tiles + (s * g.blocks + (e >> 3)) * kBlockBytes + u * 128 + (e & 7) * 16) =
                                make_uint4(0, 0, 0, 0);
            }
            bool grown = false;
            uint32_t near = 0;   // f16: heads with a weight of some size among this lane's tokens
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                float& a = z[4 * (k >> 1) + (k & 1)];
                float& b = z[4 * (k >> 1) + (k & 1) + 2];
                a = (on >> quad) & 1 ? a * zs : -INFINITY;
                b = (on >> (quad + 8)) & 1 ? b * zs : -INFINITY;
                grown = grown || fmaxf(a, b) > m[k] + kAbove;
                if (kF16 && fmaxf(a, b) >= m[k] + kBelow) near |= 1u << k;
            }
            if (kF16) {   // or among this warp's, for the other warps
                const uint32_t all = __reduce_or_sync(kFull, near << (kPer * t4));
                if (lane == 0) x.near[i & 1][warp] = all;
            }
            bool follow = softmax_any(grown);
            if (kF16) {   // heads without one in the tile
                const uint4 a = *reinterpret_cast<const uint4*>(x.near[i & 1]), b = *reinterpret_cast<const uint4*>(x.near[i & 1] + 4);
                follow = follow || (a.x | a.y | a.z | a.w) != kHeads || (b.x | b.y | b.z | b.w) != kHeads;
            }
            if (follow) {
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    float top = fmaxf(z[4 * (k >> 1) + (k & 1)], z[4 * (k >> 1) + (k & 1) + 2]);
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
                    if (quad == 0) x.top[sub][head(k)] = top;
                }
                softmax_sync();
                bool moved = false;
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int h = head(k);
                    const float top = fmaxf(fmaxf(x.top[0][h], x.top[1][h]), fmaxf(x.top[2][h], x.top[3][h]));
                    float now = fmaxf(top, m[k]);
                    if (kF16) {
                        now = fmaxf(m[k], top - kLiftLatent);
                        if (top < m[k] + kBelow && top > -INFINITY) now = fmaxf(top - kLiftLatent, x.topr[0][h] - kDeepLatent);
                    }
                    moved = moved || now != m[k];
                    const float c = part_weight(m[k], now);
                    l[k] *= c;
                    lr[k] *= c;
                    m[k] = now;
                    if (sub == 0 && quad == 0) x.corr[h] = c;
                }
                moved = softmax_any(moved);
                if (kF16 && sub == 0 && quad == 0)
#pragma unroll
                    for (int k = 0; k < kPer; ++k) x.topr[0][head(k)] = fmaxf(x.topr[0][head(k)], m[k]);
                if (moved && !begins) {
                    role_wait(&x.free[prev], prev_phase, abort, p);   // the products so far are in
                    tc::fence_after_sync();
#pragma unroll 1
                    for (int c = (warp >> 2) * 16; c < kOCols; c += 32) {
                        float v[16];
                        tc::tmem_ld16(tlane + c, v);
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] *= x.corr[(c + k) % kN];
                        tc::tmem_st16(tlane + c, v);
                    }
                    tc::wait_st();
                }
            }
            uint32_t pk[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const float mz = m[k] == -INFINITY ? 0.0f : m[k];
                float& a = z[4 * (k >> 1) + (k & 1)];
                float& b = z[4 * (k >> 1) + (k & 1) + 2];
                a = exp2_fast(a - mz);
                b = exp2_fast(b - mz);
                l[k] += a + b;
            }
#pragma unroll
            for (int j = 0; j < kPer; ++j) {   // j: heads of k = j & ~1 and the next, tokens quad + 8 (j % 2)
                pk[j] = pack2<kF16>(z[2 * j], z[2 * j + 1]);
                const float2 r = unpack2<kF16>(pk[j]);
                lr[j & ~1] += r.x;
                lr[j | 1] += r.y;
            }
            if (i > 0) role_wait(&x.free[prev], prev_phase, abort, p);   // p of the tile before has been read
            if constexpr (kN == 16) {
                const int h = c0 + (lane & 7), chunk = sub * 2 + ((lane >> 3) & 1);
                stmatrix2t(p32 + h * 128 + ((chunk ^ (h & 7)) << 4), pk[0], pk[1]);
            } else {
#pragma unroll
                for (int j = 0; j < kN / 16; j += 2) {
                    const int mat = lane >> 3, h = c0 + (j + (mat >> 1)) * 8 + (lane & 7), chunk = sub * 2 + (mat & 1);
                    stmatrix4t(p32 + h * 128 + ((chunk ^ (h & 7)) << 4), pk[2 * j], pk[2 * j + 1], pk[2 * j + 2], pk[2 * j + 3]);
                }
            }
            tc::fence_async_smem();
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&x.pready);

            if (ends) {
                // ---- the row's end ----
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int h = head(k);
                    float sum = l[k], sumr = lr[k];
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) {
                        sum += __shfl_xor_sync(kFull, sum, o);
                        sumr += __shfl_xor_sync(kFull, sumr, o);
                    }
                    if (quad == 0) {
                        x.top[sub][h] = sum;
                        x.topr[sub][h] = sumr;
                        if (sub == 0) x.inv[h] = m[k];
                    }
                }
                softmax_sync();
                const bool whole = began == 0 && w.tile == w.span.tiles - 1;
                const int slot = part_slot(worker, began == 0);
                const size_t row = static_cast<size_t>(w.r) * p.Hq + h0;
                const size_t prow = (static_cast<size_t>(slot) * g.groups + group) * kN;
                if (tid < kN) {
                    const float sum = x.top[0][tid] + x.top[1][tid] + x.top[2][tid] + x.top[3][tid], ref = x.inv[tid];
                    const float sumr = x.topr[0][tid] + x.topr[1][tid] + x.topr[2][tid] + x.topr[3][tid];
                    x.inv[tid] = sumr == 0.0f ? 0.0f : 1.0f / sumr;
                    if (!whole)
                        reinterpret_cast<float4*>(p.part_ml)[prow + tid] = make_float4(ref, ref, sum, sumr);
                    else if (p.lse && tid < heads)
                        p.lse[row + tid] = log_sum(ref, sum);
                }
                softmax_sync();
                role_wait(&x.free[s], phase, abort, p);
                tc::fence_after_sync();
#pragma unroll 1
                for (int c = (warp >> 2) * 16; c < kOCols; c += 32) {
                    float v[16];
                    tc::tmem_ld16(tlane + c, v);
                    const int dim = (c / kN) * 128 + sub * 32 + lane, hb = c % kN;
                    if (whole) {
                        uint16_t* const o = static_cast<uint16_t*>(p.o) + (row + hb) * DV + dim;
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (hb + k < heads) o[k * DV] = static_cast<uint16_t>(pack2<kF16>(v[k] * x.inv[hb + k], 0.0f));
                    } else {
                        float* const o = p.part + (prow + hb) * DV + dim;
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (hb + k < heads) o[k * DV] = v[k];
                    }
                }
                if (tid == 0 && !whole && began == 0) {
                    split = row_parts(p, share, worker, w.left, w.tile, w.span.tiles);
                    if (group == 0) p.split[kKvWorkers + worker] = w.r * g.groups;
                }
            }
            prev = s;
            prev_phase = phase;
            if (++s == g.stages) s = 0, phase ^= 1;
            begins = ends;
            live = w.next(p, share, 1);
        }
    }
    if (!p.whole_rows && group == 0 && tid == 0) p.split[worker] = split;
    // requests without tokens, by the warps that are done first
    const int ctid = tid - (kLatIssuer + 1) * 32;
    for (int r = worker; ctid >= 0 && r < p.R; r += p.workers)
        if (clamped_len(p, r, true) == 0) {
            uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.o) + (static_cast<size_t>(r) * p.Hq + h0) * DV);
            for (int i = ctid; i < heads * (DV / 8); i += kLatCopiers * 32) o[i] = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = ctid; i < heads; i += kLatCopiers * 32) p.lse[static_cast<size_t>(r) * p.Hq + h0 + i] = -INFINITY;
        }

    tc::fence_before_sync();
    __syncthreads();
    if (*abort && warp == kLatIssuer + 1)   // copies by the tensor map may be under way: none may land in a CTA that has gone
        for (int i = max(0, copied - g.stages); i < copied; ++i)
            for (int k = 0; k < kParts; ++k) tc::mbar_wait(&x.full[i % g.stages][k], (i / g.stages) & 1, kDefaultWaitPolls);
    if (warp == kLatIssuer) {
        if (*abort) {   // products may be under way: wait for them before tensor memory goes back
            const uint32_t lead = elect_lane();
            commit_by(&x.drain, lead);
            if (lead && !tc::mbar_wait(&x.drain, 0, kDefaultWaitPolls)) raise_status(p.status, QS_DEV_TEARDOWN);
        }
        __syncwarp();
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, kAlloc);
    }
}

// Map of the pool as rows of dk 16-bit entries, for boxes of 64 entries x box_rows; false if the driver has no such
// call or refuses (qs_kv_attend.cu).
bool pool_map(CUtensorMap* map, const void* pool, int dk, long long rows, int box_rows);

// Groups of at most 64 heads, products of 16, 32 or 64 columns; as many tiles in flight as fit beside the
// queries, and two CTAs on an SM where the kernel is made for it.
inline LatentGeo latent_geo(int Hq, int dk, int dv, int sms) {
    if (sms > kKvSms) sms = kKvSms;
    LatentGeo g;
    g.groups = (Hq + 63) / 64;
    g.per_group = (Hq + g.groups - 1) / g.groups;
    const int N = g.per_group <= 16 ? 16 : g.per_group <= 32 ? 32 : 64;
    g.columns = N;
    g.blocks = (dk + 63) / 64;
    const int fixed = g.blocks * N * 128 + N * 128 + static_cast<int>(sizeof(LatentMisc)), tile = g.blocks * kBlockBytes;
    constexpr int kHalf = 113 * 1024;
    const int limit = latent_ctas(dv, N) == 2 && fixed + 2 * tile <= kHalf ? kHalf : kLatSmem;
    g.stages = (limit - fixed) / tile;
    if (g.stages > kMaxStages) g.stages = kMaxStages;
    g.smem = fixed + g.stages * tile;
    g.workers = sms * (limit == kHalf ? 2 : 1) / g.groups;
    if (g.workers < 1) g.workers = 1;
    if (g.workers > kKvWorkers) g.workers = kKvWorkers;
    return g;
}

template <int DV, int kN, bool kF16>
cudaError_t launch_latent(KvAttendParams p, const LatentGeo& g, const CUtensorMap& map, cudaStream_t stream) {
    auto* kernel = kv_latent_kernel<DV, kN, kF16>;
    // The limit is the kernel's, and layers of other widths share the kernel: all of an SM for every call, so that none
    // takes it away from another thread's between its two steps.
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLatSmem);
    if (e != cudaSuccess) return e;
    p.workers = g.workers;
    p.whole_rows = (static_cast<long long>(p.max_pages) << p.page_shift) <= kWholeTiles * kLatTile;
    if (p.whole_rows && p.R < p.workers) p.workers = p.R;
    e = launch_chained(kernel, p.workers * g.groups, kLatThreads, g.smem, stream, true, p, g, map);
    if (e != cudaSuccess || p.whole_rows) return e;
    return launch_join<DV, kF16>(p, JoinGeo{g.groups, kN, g.per_group, p.Hq, g.groups}, stream);
}

template <int DV>
cudaError_t launch_latent_of(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    LatentGeo g = latent_geo(p.Hq, p.dk, DV, device_sm_count());
    // Boxes where a page holds a whole tile: nine of them for 512 + 64.  One lane issues them, some 100 cycles each, so that with
    // shorter pages the copies of 16 bytes, which cost four warps' instructions but nothing a page, are the faster ones
    // or near (64 requests, heads and latents: pages of 32 tokens by boxes and by 16 bytes, then pages of 64: 64 of 512 + 64
    // 95.8, 92.3, then 91.9 and 92.0 us; 64 of 256 + 64 68.4, 59.8, then 58.0 and 59.7; 16 of 128 + 64 87.2, 89.0, then 75.5
    // and 89.0; at pages of 8 the first took 191 by boxes, 107 by 16 bytes).
    CUtensorMap map = {};
    g.boxes = c.page >= kLatTile && pool_map(&map, p.k, p.dk, static_cast<long long>(c.n_pages) * c.page, kLatTile);
    const bool f16 = c.dtype == QSTATE_KV_F16;
    if (g.columns == 16) return f16 ? launch_latent<DV, 16, true>(p, g, map, stream) : launch_latent<DV, 16, false>(p, g, map, stream);
    if (g.columns == 32) return f16 ? launch_latent<DV, 32, true>(p, g, map, stream) : launch_latent<DV, 32, false>(p, g, map, stream);
    return f16 ? launch_latent<DV, 64, true>(p, g, map, stream) : launch_latent<DV, 64, false>(p, g, map, stream);
}

}  // namespace kv
}  // namespace qs
