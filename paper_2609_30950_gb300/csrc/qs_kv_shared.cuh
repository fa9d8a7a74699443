// qs_kv_shared.cuh -- the tokens that a group of requests has in common, read once for all of its requests.
//
// With n tokens in common, rows i = (request, query head) of one key head, z_it = scale q_i.k_t:
//     part_i = (m_i, l_i = sum_t 2^{z_it - m_i}, sum_t 2^{z_it - m_i} v_t),   z in base 2, m_i near the largest z_it.
// The requests' own tokens give such parts too (qs_kv_heads.cuh), and the parts of a row are joined at the end:
//     o_i = sum_parts 2^{m - M} sums / sum_parts 2^{m - M} l.
// A block of up to 256 rows (128 at 256 entries) meets a tile of 128 (64) tokens: 4 d operations a row and token against
// the tile's 4 d bytes a token, so that from some 300 rows on it is the tensor cores and the softmax, not
// the cache's bytes, that bound it, and below that one pass over the bytes.  Both products run on the tensor cores:
//     S [128 rows x tokens] = Q K^T     Q and K in shared memory, entries contiguous (K-major)
//     O [128 rows x d]     += P V       P in tensor memory over S itself, V in shared memory, entries contiguous (N-major)
//   warps 0-3, 4-7  softmax: a row each, of the block's first and second 128 rows (at 256 entries only the first, whose S has two
//                   buffers instead)
//   warp 8          issues the products
//   warps 9-12      copy queries, keys and values, 16 bytes at a time (e4m3: eight warps, which turn codes into bf16 on the way,
//                   exactly: a code has 4 bits and its power of two is one of the type's)
// The units of all blocks (a tile; kSharedRowUnits more for the block itself) are dealt out evenly, as the rows' are in
// qs_kv_tiles.cuh: a block that several CTAs share leaves a part from each.
// The reference m follows the maximum only when that has outgrown it by 2^8.  In f16, which ends at 2^-24, a weight of the
// reference is 2^7, and the reference also goes down, to a tile whose largest weight is under 2^-16 of it (see
// qs_kv_latent.cuh).  p has 16 bits in the second product, and o is divided by the sum of the rounded p, so that the weights in
// use add up to one; lse comes from the sum before rounding.
#pragma once

#include "qs_kv_latent.cuh"

namespace qs {
namespace kv {

constexpr int kMaxRing = 8, kMaskRing = 8;

template <int D, bool kE4M3>
struct SharedShape {
    static constexpr int kTile = kv_shared_tile(D), kRows = kv_shared_rows(D), kM = kRows / 128;
    static constexpr int kBuffers = kM == 1 ? 2 : 1;                  // of S
    static constexpr int kBlocks = D / 64;                            // of 64 entries
    static constexpr int kTensor = kTile * D * 2;                     // bytes of a tile's keys
    static constexpr int kBlock = kTile * 128;                        // and of a block of them
    static constexpr int kQBlock = 128 * 128, kQTile = kBlocks * kQBlock;
    static constexpr int kStages = D == 64 ? 8 : 5;
    static constexpr int kRing = kM * kQTile, kMisc = kRing + kStages * kTensor;
    static constexpr int kSoftmax = 4 * kM, kIssuer = kSoftmax, kCopiers = kE4M3 ? 8 : 4;
    static constexpr int kThreads = (kSoftmax + 1 + kCopiers) * 32;
    static constexpr int kOCol = kM * kBuffers * kTile;               // columns of tensor memory in front of O
    static_assert(kStages <= kMaxRing && kOCol + kM * D <= 512, "tensor memory");
    static constexpr int kWarpTokens = kTile / kCopiers;
};

struct SharedMisc {
    uint64_t full[kMaxRing], free[kMaxRing], seen[kMaskRing], sready[2], pready[2], odone[2], qfull, qfree, drain;
    uint32_t mask[kMaskRing][4];
    uint32_t tmem;
    int abort;
};

// Walks a worker's units.
struct SharedWalk {
    int e, hb, tile, tiles;      // group, key head and block of rows in one, tile
    int left;
    KvGroup g;

    __device__ __forceinline__ void load(const KvGroup* groups, int index, int kTile) {
        e = index;
        const int4* const src = reinterpret_cast<const int4*>(groups + index);
        int4 a = __ldcg(src), b = __ldcg(src + 1);
        g.first = a.x, g.rows = a.y, g.owner = a.z, g.tokens = a.w;
        g.blocks = b.x, g.block0 = b.y;
        g.unit0 = static_cast<long long>(static_cast<unsigned>(b.z)) | static_cast<long long>(b.w) << 32;
        tiles = (g.tokens + kTile - 1) / kTile;
    }
    __device__ __forceinline__ bool start(const KvGroupHead& head, const KvGroup* groups, int worker, int workers, int kTile) {
        const long long u0 = share_start(head.units, worker, workers), u1 = share_start(head.units, worker + 1, workers);
        left = static_cast<int>(u1 - u0);
        if (left <= 0) return false;
        int lo = 0, n = head.groups;   // last group that begins at u0 or before
        while (n > 1) {
            const int half = n >> 1;
            if (__ldcg(&groups[lo + half].unit0) <= u0) {
                lo += half;
                n -= half;
            } else {
                n = half;
            }
        }
        load(groups, lo, kTile);
        const int per = tiles + kSharedRowUnits;
        const long long at = u0 - g.unit0;
        hb = static_cast<int>(at / per);
        tile = static_cast<int>(at - static_cast<long long>(hb) * per) - kSharedRowUnits;
        if (tile < 0) {
            left += tile;
            tile = 0;
        }
        return left > 0;
    }
    __device__ __forceinline__ bool next(const KvGroup* groups, int Hkv, int kTile) {
        if (--left <= 0) return false;
        if (++tile < tiles) return true;
        tile = 0;
        left -= kSharedRowUnits;
        if (left <= 0) return false;
        if (++hb < g.blocks * Hkv) return true;
        hb = 0;
        load(groups, e + 1, kTile);
        return true;
    }
    __device__ __forceinline__ bool ends() const { return tile == tiles - 1 || left == 1; }
    __device__ __forceinline__ int kv() const { return hb / g.blocks; }
    __device__ __forceinline__ int block() const { return hb % g.blocks; }
};

// D [128 x N] (+)= A [128 x 16] B, A in tensor memory (two entries a column).  As mma_f16_ss: a whole warp in step.
template <uint32_t kHi>
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, bool accumulate, uint32_t lead) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 b;\nmov.b64 b, {%2, %6};\nsetp.ne.b32 p, %4, 0;\n"
        "setp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n" ::"r"(d),
        "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate ? 1u : 0u), "r"(lead), "n"(kHi)
        : "memory");
}
// 32 columns of a lane's row.
__device__ __forceinline__ void tmem_ld32(uint32_t at, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16u(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

template <int D, bool kF16, bool kE4M3>
__global__ void __launch_bounds__(SharedShape<D, kE4M3>::kThreads, 1) kv_shared_kernel(const KvAttendParams p) {
    using S = SharedShape<D, kE4M3>;
    constexpr int kTile = S::kTile, kM = S::kM, kAlloc = 512;
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(1024) char smem[];
    SharedMisc& x = *reinterpret_cast<SharedMisc*>(smem + S::kMisc);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, worker = blockIdx.x;
    const KvGroupHead* const head_at = reinterpret_cast<const KvGroupHead*>(p.groups);
    const KvGroup* const groups = reinterpret_cast<const KvGroup*>(reinterpret_cast<const char*>(p.groups) + kKvGroupHeadBytes);
    chain_enter();
    if (warp == S::kIssuer) {
        tc::tmem_alloc(&x.tmem, kAlloc);
        tc::tmem_relinquish();
        chain_release();   // the next kernel may take its place; one with tensor memory no sooner
    }
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            tc::mbar_init(&x.full[s], S::kCopiers * (kE4M3 ? 1 : 33));
            tc::mbar_init(&x.free[s], 1);
        }
        for (int s = 0; s < kMaskRing; ++s) tc::mbar_init(&x.seen[s], S::kCopiers);
        for (int m = 0; m < 2; ++m) {
            tc::mbar_init(&x.sready[m], 1);
            tc::mbar_init(&x.pready[m], 4);
            tc::mbar_init(&x.odone[m], 1);
        }
        tc::mbar_init(&x.qfull, S::kCopiers * 33);
        tc::mbar_init(&x.qfree, 1);
        tc::mbar_init(&x.drain, 1);
        tc::mbar_fence_init();
        x.abort = 0;
    }
    KvGroupHead head;
    head.groups = __ldcg(&head_at->groups);
    head.R = __ldcg(&head_at->R);
    head.Hq = __ldcg(&head_at->Hq);
    head.Hkv = __ldcg(&head_at->Hkv);
    head.tile = __ldcg(&head_at->tile);
    head.units = __ldcg(&head_at->units);
    // groups that were made for other requests or another kind of layer are none
    const bool fits = head.groups == 0 || (head.R == p.R && head.Hq == p.Hq && head.Hkv == p.Hkv && head.tile == kTile);
    if (!fits && tid == 0) raise_status(p.status, QS_DEV_PAGES);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = x.tmem;
    volatile int* const abort = &x.abort;
    const int G = p.Hq / p.Hkv;
    SharedWalk w;
    bool live = fits && head.groups > 0 && w.start(head, groups, worker, p.workers, kTile);

    if (live && warp > S::kIssuer) {
        // ---- copies ----
        const int pw = warp - S::kIssuer - 1, page_mask = (1 << p.page_shift) - 1;
        auto look_up = [&](const SharedWalk& at) {
            const int t = at.tile * kTile + pw * S::kWarpTokens + lane;
            return lane < S::kWarpTokens && t < at.g.tokens ? __ldcg(p.table + static_cast<size_t>(at.g.owner) * p.max_pages + (t >> p.page_shift)) : -1;
        };
        // a thread copies one of eight pieces of every block of its rows
        auto queries = [&](const SharedWalk& at) {
            const int sg = lane & 7, h0 = at.kv() * G, i0 = at.block() * S::kRows;
            const int rows = min(S::kRows, at.g.rows - i0);
            for (int i = pw * 4 + (lane >> 3); i < S::kRows; i += S::kCopiers * 4) {
                const bool in = i < rows;
                const int at_row = i0 + i, member = in ? at_row / G : 0;
                const uint16_t* const q = static_cast<const uint16_t*>(p.q) + (at.g.first + member) * p.q_row +
                                          (in ? h0 + at_row - member * G : 0) * p.q_head + sg * 8;
                uint32_t to = smem_u32(smem + (i >> 7) * S::kQTile + (i & 127) * 128 + ((sg ^ (i & 7)) << 4));
                for (int b = 0; b < S::kBlocks; ++b, to += S::kQBlock) {
                    if (p.q_aligned) {
                        cp_async16(to, in ? q + b * 64 : p.q, in);
                    } else {
                        uint16_t v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = in ? q[b * 64 + k] : 0;
                        st_shared16(to, v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
                    }
                }
            }
            cp_async_arrive(&x.qfull);
            __syncwarp();
            if (lane == 0) mbar_arrive(&x.qfull);
        };
        int id = look_up(w), s = 0, phase = 0, blocks = 0, used = 0;   // blocks: of rows, whose queries have been asked for
        bool begins = true, ok = true;                                 // ok: no wait has been given up
        for (int i = 0; live; ++i) {
            if (begins) {
                if (blocks > 0) ok = ok && role_wait(&x.qfree, (blocks - 1) & 1, abort, p);   // S of the block before is done
                if (ok)
                    queries(w);
                else {
                    cp_async_arrive(&x.qfull);
                    if (lane == 0) mbar_arrive(&x.qfull);
                }
                ++blocks;
            }
            begins = w.ends();
            const int t = w.tile * kTile + pw * S::kWarpTokens + lane;
            const bool wanted = lane < S::kWarpTokens && t < w.g.tokens, there = wanted && id >= 0 && id < p.n_pages;
            if (wanted && !there) raise_status(p.status, QS_DEV_PAGES);
            const uint32_t on = __ballot_sync(kFull, there);
            if (lane == 0) {
                if (S::kWarpTokens == 32)
                    *reinterpret_cast<volatile uint32_t*>(&x.mask[i % kMaskRing][pw]) = on;
                else if (S::kWarpTokens == 16)
                    reinterpret_cast<volatile uint16_t*>(x.mask[i % kMaskRing])[pw] = static_cast<uint16_t>(on);
                else
                    reinterpret_cast<volatile uint8_t*>(x.mask[i % kMaskRing])[pw] = static_cast<uint8_t>(on);
                mbar_arrive(&x.seen[i % kMaskRing]);
            }
            const long long row = there ? ((static_cast<long long>(id) * p.Hkv + w.kv()) << p.page_shift) + (t & page_mask) : 0;
            live = w.next(groups, p.Hkv, kTile);
            if (live) id = look_up(w);
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
                const char* const pool = static_cast<const char*>(kv ? p.v : p.k);
                const uint32_t stage = smem_u32(smem + S::kRing + s * S::kTensor);
                if constexpr (!kE4M3) {
                    if (used >= S::kStages) ok = ok && role_wait(&x.free[s], phase ^ 1, abort, p);
                    const int sg = lane & 7, row0 = lane >> 3;
                    if (ok)
#pragma unroll
                        for (int k = 0; k < S::kWarpTokens / 4; ++k) {
                            const int u = k * 4 + row0;
                            const char* const src = pool + __shfl_sync(kFull, row, u) * (2 * D) + sg * 16;
                            const bool seen = (on >> u) & 1;
                            const uint32_t to = stage + (pw * S::kWarpTokens + u) * 128 + ((sg ^ (u & 7)) << 4);
#pragma unroll
                            for (int b = 0; b < S::kBlocks; ++b) cp_async16(to + b * S::kBlock, src + b * 128, seen);
                        }
                    cp_async_arrive(&x.full[s]);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&x.full[s]);
                } else {
                    // 16 codes a lane and load, all of a tile's in flight; D / 16 lanes take a token
                    constexpr int kLanes = D / 16, kLoads = S::kWarpTokens * kLanes / 32;
                    const uint8_t* const exps = kv ? p.v_exp : p.k_exp;
                    const int sg = lane % kLanes, row0 = lane / kLanes;
                    uint4 codes[kLoads];
                    const int power = there ? __ldcg(exps + row) : 127;
#pragma unroll
                    for (int k = 0; k < kLoads; ++k) {
                        const int u = k * (32 / kLanes) + row0;
                        const char* const src = pool + __shfl_sync(kFull, row, u) * D + sg * 16;
                        codes[k] = (on >> u) & 1 ? __ldcg(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0);
                    }
                    if (used >= S::kStages) ok = ok && role_wait(&x.free[s], phase ^ 1, abort, p);
#pragma unroll
                    for (int k = 0; k < kLoads; ++k) {
                        const int u = k * (32 / kLanes) + row0;
                        const unsigned e = __shfl_sync(kFull, power, u);
                        // 2^(e - 127); 0 is the type's lowest power (2^-127, not a normal number), 255 NaN
                        const float two = e == 255 ? __uint_as_float(0x7fffffffu) : e ? __uint_as_float(e << 23) : 0x1p-127f;
                        const uint32_t c[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t lo, hi;
                            asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}"
                                : "=r"(lo), "=r"(hi) : "r"(c[j]));
                            const float2 a = unpack2<true>(lo), b = unpack2<true>(hi);
                            y[2 * j] = pack2<false>(a.x * two, a.y * two);
                            y[2 * j + 1] = pack2<false>(b.x * two, b.y * two);
                        }
                        // entries 16 sg ...: pieces 2 (sg % 4) and the next of block sg / 4
                        const int token = pw * S::kWarpTokens + u, piece = (sg & 3) * 2;
                        const uint32_t to = stage + (sg >> 2) * S::kBlock + token * 128;
                        if (ok) {
                            st_shared16(to + ((piece ^ (token & 7)) << 4), y[0], y[1], y[2], y[3]);
                            st_shared16(to + (((piece + 1) ^ (token & 7)) << 4), y[4], y[5], y[6], y[7]);
                        }
                    }
                    tc::fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&x.full[s]);
                }
                ++used;
                if (++s == S::kStages) s = 0, phase ^= 1;
            }
        }
        cp_commit();
        cp_wait<0>();
    } else if (live && warp == S::kIssuer) {
        // ---- products ----
        constexpr uint32_t idS = idesc_f16(kF16, 128, kTile, false), idO = idesc_f16(kF16, 128, D, false) | 1u << 16;
        const uint32_t lead = elect_lane();
        const uint32_t dq = desc_lo(smem_u32(smem), 16), ring = smem_u32(smem + S::kRing);
        int s = 0, phase = 0;           // ring
        int done[2] = {0, 0};           // tiles of either half whose S has been issued
        int blocks = 0;
        bool ok = true, begins = true;
        auto advance = [&]() {
            if (++s == S::kStages) s = 0, phase ^= 1;
        };
        auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && role_wait(bar, parity, abort, p); };
        auto scores = [&](int m, uint32_t k_at) {   // of the half's next tile
            const int n = done[m]++, buffer = kM == 2 ? m : n & 1;
            const int before = n - S::kBuffers;     // its tile that had this buffer: p has been read
            if (before >= 0) wait(&x.odone[m], before & 1);
            if (!ok) return;
            tc::fence_after_sync();
            const uint32_t b0 = desc_lo(k_at, 16), a0 = dq + m * (S::kQTile / 16);
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_f16_ss<kDescHi>(tmem + buffer * kTile, a0 + (b * S::kQBlock + k * 32) / 16, b0 + (b * S::kBlock + k * 32) / 16, idS,
                                        b > 0 || k > 0, lead);
            commit_by(&x.sready[buffer], lead);
        };
        auto values = [&](int m, int n, uint32_t v_at, bool first) {   // of the half's tile n
            const int buffer = kM == 2 ? m : n & 1;
            wait(&x.pready[buffer], (S::kBuffers == 2 ? n >> 1 : n) & 1);
            if (!ok) return;
            tc::fence_after_sync();
            const uint32_t b0 = desc_lo(v_at, S::kBlock);
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
                mma_f16_ts<kDescHi>(tmem + S::kOCol + m * D, tmem + buffer * kTile + k * 8, b0 + k * 128, idO, !first || k > 0, lead);
            commit_by(&x.odone[m], lead);
        };
        // keys of the walk's tile: S of both halves
        auto keys = [&]() {
            const bool two = kM == 2 && w.g.rows - w.block() * S::kRows > 128;
            if (begins) wait(&x.qfull, blocks++ & 1);
            wait(&x.full[s], phase);
            if (ok) tc::fence_async_smem();   // the copies' writes, for the tensor core's reads
            const uint32_t at = ring + s * S::kTensor;
            scores(0, at);
            if (two) scores(1, at);
            if (ok) {
                commit_by(&x.free[s], lead);
                if (w.ends()) commit_by(&x.qfree, lead);
            }
            advance();
            return two;
        };
        bool two = keys();
        while (live && ok) {
            // keys of the next tile go in front of this one's values in the ring's order, behind them where S has one buffer
            const bool first = begins, ends = w.ends(), now = two;
            const int n0 = done[0] - 1, n1 = done[1] - 1;
            const int sv = s, pv = phase;
            auto products = [&]() {
                wait(&x.full[sv], pv);
                if (ok) tc::fence_async_smem();
                const uint32_t at = ring + sv * S::kTensor;
                values(0, n0, at, first);
                if (now) values(1, n1, at, first);
                if (ok) commit_by(&x.free[sv], lead);
            };
            advance();
            if (S::kBuffers == 1) products();
            begins = ends;
            live = w.next(groups, p.Hkv, kTile);
            if (live) two = keys();
            if (S::kBuffers == 2) products();
        }
    } else if (live && warp < S::kSoftmax) {
        // ---- softmax ----
        const int m_half = warp >> 2, row = (warp & 3) * 32 + lane;   // of the half
        const uint32_t tlane = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
        const uint32_t o_at = tlane + S::kOCol + m_half * D;
        const float zs = p.scale * kLog2e;
        constexpr float kAbove = kF16 ? kLazyLatent + kLiftLatent : kLazyLatent, kBelow = kLiftLatent - kFarLatent;
        float m = -INFINITY, high = -INFINITY, l = 0.0f, lr = 0.0f;   // reference, the highest so far, sums of p and of rounded p
        bool begins = true;
        int began = 0, n = 0;   // n: tiles of this half
        for (int i = 0; live; ++i) {
            const int i0 = w.block() * S::kRows, rows = min(S::kRows, w.g.rows - i0) - m_half * 128;
            const bool ends = w.ends();
            if (begins) {
                began = w.tile;
                m = high = -INFINITY;
                l = lr = 0.0f;
            }
            if (rows > 0) {
                const int buffer = kM == 2 ? m_half : n & 1;
                const uint32_t s_at = tlane + buffer * kTile;
                role_wait(&x.sready[buffer], (S::kBuffers == 2 ? n >> 1 : n) & 1, abort, p);
                // behind the scores: a half that stepped over blocks may be rounds ahead of the masks
                role_wait(&x.seen[i % kMaskRing], (i / kMaskRing) & 1, abort, p);
                uint32_t on[kTile / 32];
                bool all = true;
#pragma unroll
                for (int k = 0; k < kTile / 32; ++k) {
                    on[k] = *reinterpret_cast<volatile uint32_t*>(&x.mask[i % kMaskRing][k]);
                    all = all && on[k] == kFull;
                }
                tc::fence_after_sync();
                // the largest score
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < kTile / 32; ++k) {
                    float z[32];
                    tmem_ld32(s_at + k * 32, z);
                    if (!all)
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = (on[k] >> j) & 1 ? z[j] * zs : -INFINITY;
                    float a = -INFINITY, b = -INFINITY;
                    if (all && zs < 0.0f) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) a = fmaxf(a, -z[j]), b = fmaxf(b, -z[j + 1]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) a = fmaxf(a, z[j]), b = fmaxf(b, z[j + 1]);
                    }
                    a = fmaxf(a, b);
                    top = fmaxf(top, all ? a * fabsf(zs) : a);
                }
                float now = m;
                if (kF16) {
                    if (top > m + kAbove || m == -INFINITY) now = fmaxf(m, top - kLiftLatent);
                    if (top < m + kBelow && top > -INFINITY) now = fmaxf(top - kLiftLatent, high - kDeepLatent);
                    high = fmaxf(high, now);
                } else if (top > m + kAbove || m == -INFINITY) {
                    now = fmaxf(m, top);
                }
                if (__any_sync(kFull, now != m)) {
                    const float c = part_weight(m, now);
                    l *= c;
                    lr *= c;
                    m = now;
                    if (!begins) {
                        role_wait(&x.odone[m_half], (n - 1) & 1, abort, p);   // the products so far are in
                        tc::fence_after_sync();
#pragma unroll 1
                        for (int k = 0; k < D; k += 16) {
                            float v[16];
                            tc::tmem_ld16(o_at + k, v);
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] *= c;
                            tc::tmem_st16(o_at + k, v);
                        }
                    }
                }
                const float mz = m == -INFINITY ? 0.0f : m;
                const float2 zs2 = make_float2(zs, zs), mz2 = make_float2(-mz, -mz);
                float2 ls = make_float2(0.0f, 0.0f), lrs = ls;
#pragma unroll
                for (int k = 0; k < kTile / 32; ++k) {
                    float z[32];
                    tmem_ld32(s_at + k * 32, z);
                    uint32_t w16[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float2 y = __ffma2_rn(make_float2(z[2 * j], z[2 * j + 1]), zs2, mz2);
                        if (!all) {
                            y.x = (on[k] >> (2 * j)) & 1 ? y.x : -INFINITY;
                            y.y = (on[k] >> (2 * j + 1)) & 1 ? y.y : -INFINITY;
                        }
                        y.x = exp2_fast(y.x);
                        y.y = exp2_fast(y.y);
                        ls = __fadd2_rn(ls, y);
                        w16[j] = pack2<kF16>(y.x, y.y);
                        lrs = __fadd2_rn(lrs, unpack2<kF16>(w16[j]));
                    }
                    tmem_st16u(s_at + k * 16, w16);   // over scores that have been read
                }
                l += ls.x + ls.y;
                lr += lrs.x + lrs.y;
                tc::wait_st();
                // With two buffers the products of the tile before may be under way still: its phase is waited for while this
                // tile's cannot be over, for the wait below tells neighbouring phases apart only.
                if (S::kBuffers == 2 && ends && n > 0) role_wait(&x.odone[m_half], (n - 1) & 1, abort, p);
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&x.pready[buffer]);
                if (ends) {
                    // ---- the part's end ----
                    role_wait(&x.odone[m_half], n & 1, abort, p);
                    tc::fence_after_sync();
                    const bool whole = began == 0 && w.tile == w.tiles - 1;
                    const size_t slot_row = static_cast<size_t>(part_slot(worker, began == 0)) * S::kRows + m_half * 128 + row;
                    const int at_row = i0 + m_half * 128 + row, member = at_row / G;
                    const size_t out_row = static_cast<size_t>(w.g.first + member) * p.Hq + w.kv() * G + at_row - member * G;
                    float* const to = whole ? p.pre_store + out_row * D : p.pre_part + slot_row * D;
                    if (row < rows) (whole ? p.pre_store_ml[out_row] : p.pre_ml[slot_row]) = make_float4(m, m, l, lr);
#pragma unroll 1
                    for (int k = 0; k < D; k += 16) {
                        float v[16];
                        tc::tmem_ld16(o_at + k, v);
                        if (row < rows)
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<float4*>(to + k + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    }
                    if (tid == 0 && began == 0) {
                        const long long last = w.g.unit0 + static_cast<long long>(w.hb + 1) * (w.tiles + kSharedRowUnits) - 1;
                        p.pre_dir[w.g.block0 + w.hb] =
                            whole ? make_int2(-1, 1) : make_int2(worker, share_owner(head.units, last, p.workers) - worker + 1);
                    }
                    tc::fence_before_sync();
                }
                ++n;
            }
            begins = ends;
            live = w.next(groups, p.Hkv, kTile);
        }
    }

    tc::fence_before_sync();
    __syncthreads();
    if (warp == S::kIssuer) {
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

template <int D, bool kF16, bool kE4M3>
cudaError_t launch_shared(KvAttendParams p, cudaStream_t stream) {
    using S = SharedShape<D, kE4M3>;
    constexpr int kBytes = S::kMisc + sizeof(SharedMisc);
    static_assert(kBytes <= kLatSmem, "shared memory of an SM");
    const cudaError_t e = cudaFuncSetAttribute(kv_shared_kernel<D, kF16, kE4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    const int sms = device_sm_count();
    p.workers = sms < kKvSms ? sms : kKvSms;
    return launch_chained(kv_shared_kernel<D, kF16, kE4M3>, p.workers, S::kThreads, kBytes, stream, true, p);
}

template <int D>
cudaError_t launch_shared_of(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    if (c.store == QSTATE_KV_E4M3) return launch_shared<D, false, true>(p, stream);
    return c.dtype == QSTATE_KV_F16 ? launch_shared<D, true, false>(p, stream) : launch_shared<D, false, false>(p, stream);
}

}  // namespace kv
}  // namespace qs
