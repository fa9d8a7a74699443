// qs_kv_shared.cuh -- the tokens that a group of requests has in common, read once for all of its requests.
//
// With n tokens in common, rows i = (request, query head) of one key head, z_it = scale q_i.k_t:
//     part_i = (m_i, l_i = sum_t 2^{z_it - m_i}, sum_t 2^{z_it - m_i} v_t),   z in base 2, m_i near the largest z_it.
// The requests' own tokens give such parts too (qs_kv_heads.cuh), and the parts of a row are joined at the end:
//     o_i = sum_parts 2^{m - M} sums / sum_parts 2^{m - M} l.
// A block of up to 256 rows (128 at 256 entries) meets a tile of 64 tokens: 4 d operations a row and token against the tile's
// 4 d bytes a token, so that from some 300 rows on the operations, not the cache's bytes, are the floor.  Both products run on
// the tensor cores:
//     S [128 rows x tokens] = Q K^T     Q and K in shared memory, entries contiguous (K-major)
//     O [128 rows x d]     += P V       P in tensor memory over S itself, V in shared memory, entries contiguous (N-major)
// What bounds it is the softmax: 8 key heads of 1024 rows by 8192 tokens in 36 us, some 1900 clocks for a tile of two halves, in which the
// tensor pipe works 42 % and instructions issue 46 % of the time; the loads of S, the exponentials, the rounding and the store
// of P follow one another, and two rows' worth of warps to a scheduler do not hide it.  Two S buffers a stream let the next
// scores come in meanwhile (one buffer and tiles of 128 tokens: 4800 clocks for 128 tokens of two halves, against 3800).
// Measured and left out: a row's tile in the hands of two warps (40 -> 45 us at 128 entries, 42 -> 60 in e4m3); weights
// against the old reference without a look at the maximum first (36 us either way, 256 entries 10 % slower).
//   warps 0-3, 4-7  copy queries, softmax: a row to a lane, of the block's first and second 128 rows; of a block with no second
//                   half, of its even and odd tiles, which make a part each (256 entries have room for one O: warps 0-3 only)
//   warps 8-11      issue S and O of either stream: each waits for nothing but what its next product needs (in fewer warps, the
//                   instructions between products, at some ten clocks each, were what everyone waited for)
//   warps 12-15     copy keys and values: by the tensor map's boxes where pages have 8 tokens or more, 16 bytes at a time else
//                   (e4m3: they turn codes into bf16 on the way, exactly where bf16 has the product of a code, of 4 bits, and
//                   its power: what is under 2^-126 has steps of 2^-133, half of one lost at most, and 2^128, to which the largest
//                   bf16 is rounded in e4m3, becomes that bf16 again, 2^-8 less).  256 entries have 10 warps: 0-3, two that
//                   issue, four that copy
// The units of all blocks (some for a tile; those of kSharedRowUnits tiles more for the block itself) are dealt out evenly, as the rows' are in
// qs_kv_tiles.cuh: a block that several CTAs share leaves a part from each.
// The reference m follows the maximum only when that has outgrown it by 2^8.  In f16, which ends at 2^-24, a weight of the
// reference is 2^7, and the reference also goes down, to a tile whose largest weight is under 2^-16 of it (see
// qs_kv_latent.cuh).  p has 16 bits in the second product, and o is divided by the sum of the rounded p, so that the weights in
// use add up to one; lse comes from the sum before rounding.
#pragma once

#include "qs_kv_latent.cuh"

namespace qs {
namespace kv {

constexpr int kMaxRing = 16, kMaskRing = 16;

template <int D>
struct SharedShape {
    static constexpr int kTile = kSharedTile, kRows = kv_shared_rows(D), kM = kRows / 128;
    static constexpr int kBuffers = 2;                                // of S, for each stream
    static constexpr int kBlocks = D / 64;                            // of 64 entries
    static constexpr int kTensor = kTile * D * 2;                     // bytes of a tile's keys
    static constexpr int kBlock = kTile * 128;                        // and of a block of them
    static constexpr int kQBlock = 128 * 128, kQTile = kBlocks * kQBlock;
    // of the ring, keys' and values' tensors in turn; a multiple of the copying warps, so that a slot is always one warp's
    static constexpr int kStages = D == 64 ? 16 : D == 128 ? 8 : 4;
    static constexpr int kRing = kM * kQTile, kMisc = kRing + kStages * kTensor;
    static constexpr int kSoftmax = 4 * kM, kIssuer = kSoftmax, kIssuers = 2 * kM, kCopier = kIssuer + kIssuers, kCopiers = 4;   // warps
    static constexpr int kThreads = (kCopier + kCopiers) * 32;
    // S, P and O of a stream's job n are waited for at barriers of its buffer, whose next phase needs all who wait for this one:
    // a parity tells neighbouring phases apart only.
    static __device__ __forceinline__ int buffer(int stream, int n) { return stream * kBuffers + (n & 1); }
    static __device__ __forceinline__ int phase(int n) { return (n >> 1) & 1; }
    static constexpr int kOCol = kM * kBuffers * kTile;               // columns of tensor memory in front of O
    static_assert(kStages <= kMaxRing && kOCol + kM * D <= 512, "barriers, tensor memory");
    static_assert(kTile == 64 && kCopiers == 4 && kStages % kCopiers == 0, "a lane's two tokens, a copying warp's tensors");
};

struct SharedMisc {
    uint64_t full[kMaxRing], free[kMaxRing], sready[4], pready[4], odone[4], qfull, qfree, drain;
    alignas(8) uint32_t mask[kMaskRing][2];   // tokens of a tile that are there
    uint32_t tmem;
    int abort;
};

// A worker's units, part after part: a part is the worker's tiles of one block of rows, those whose first unit is in its share.
// kHalves: a tile of a block with one half weighs two units, others three (1270 and 1900 clocks): 304 rows of four key heads by 100000
// tokens 99.1 -> 90.6 us; 1024 rows of eight by 8192, all blocks alike, 80.6 -> 81.7.  In e4m3, where the copying warps set the pace,
// all are the same.
template <int kRows, bool kHalves>
struct SharedPart {
    KvGroup g;
    int e, hb, tile, count, tiles;   // group; key head and block of rows in one; first tile and how many; the block's
    int left;                        // units from the first tile to the share's end

    __device__ __forceinline__ int weight_of(int block) const {
        return kHalves && g.rows - block * kRows <= 128 ? kSharedHalfWeight : kSharedWeight;
    }
    __device__ __forceinline__ int weight() const { return weight_of(hb % g.blocks); }
    // Shares are no smaller than a tile weighs, so that every one between a block's first and last has a tile of it.
    static __device__ __forceinline__ int sharing(long long units, int workers) {
        return units < static_cast<long long>(workers) * kSharedWeight ? static_cast<int>(units) / kSharedWeight : workers;
    }
    // Of a key head's blocks; only the last may have one half.
    __device__ __forceinline__ long long head_units() const {
        return static_cast<long long>(tiles + kSharedRowUnits) * ((g.blocks - 1) * kSharedWeight + weight_of(g.blocks - 1));
    }
    // The first unit of this block's last tile.
    __device__ __forceinline__ long long last_tile() const {
        const int kv = hb / g.blocks, b = hb - kv * g.blocks;
        return g.unit0 + kv * head_units() + static_cast<long long>(tiles + kSharedRowUnits) * (b * kSharedWeight) +
               static_cast<long long>(tiles + kSharedRowUnits - 1) * weight_of(b);
    }
    // The block's tiles from this one on, as far as the share goes.
    __device__ __forceinline__ void from(int first, int weight) {
        tile = first;
        count = min(tiles - first, static_cast<int>(static_cast<unsigned>(left + weight - 1) / static_cast<unsigned>(weight)));
    }

    __device__ __forceinline__ void take(const int4& a, const int4& b, int kTile) {
        g.first = a.x, g.rows = a.y, g.owner = a.z, g.tokens = a.w;
        g.blocks = b.x, g.block0 = b.y;
        g.unit0 = static_cast<long long>(static_cast<unsigned>(b.z)) | static_cast<long long>(b.w) << 32;
        tiles = (g.tokens + kTile - 1) / kTile;
    }
    __device__ __forceinline__ void load(const KvGroup* groups, int index, int kTile) {
        e = index;
        const int4* const src = reinterpret_cast<const int4*>(groups + index);
        const int4 a = __ldcg(src), b = __ldcg(src + 1);
        take(a, b, kTile);
    }
    // a and b: this lane's group, of the first 32, as they lie in memory (anything behind the last group); a whole warp.
    __device__ __forceinline__ bool start(const KvGroupHead& head, const KvGroup* groups, const int4& a, const int4& b, int worker,
                                          int workers, int Hkv, int kTile) {
        const int n = sharing(head.units, workers);
        if (worker >= n) return false;
        const long long u0 = share_start(head.units, worker, n), u1 = share_start(head.units, worker + 1, n);
        left = static_cast<int>(u1 - u0);
        if (left <= 0) return false;
        const long long mine = static_cast<long long>(static_cast<unsigned>(b.z)) | static_cast<long long>(b.w) << 32;
        const int lane = threadIdx.x & 31;
        // the last group that begins at u0 or before
        const unsigned before = __ballot_sync(kFull, lane < head.groups && mine <= u0);
        if (before != kFull || head.groups == 32) {
            const int l = 31 - __clz(before);
            e = l;
            auto from = [&](int v) { return __shfl_sync(kFull, v, l); };
            take(make_int4(from(a.x), from(a.y), from(a.z), from(a.w)), make_int4(from(b.x), from(b.y), from(b.z), from(b.w)), kTile);
        } else {
            int lo = 31, many = head.groups - 31;
            while (many > 1) {
                const int half = many >> 1;
                if (__ldcg(&groups[lo + half].unit0) <= u0) {
                    lo += half;
                    many -= half;
                } else {
                    many = half;
                }
            }
            load(groups, lo, kTile);
        }
        const int per = (tiles + kSharedRowUnits) * kSharedWeight;   // of a block
        const long long at = u0 - g.unit0, all = head_units();
        const long long kv = all >> 31 ? at / all : divided(at, static_cast<int>(all)), in_kv = at - kv * all;
        const int block = min(static_cast<int>(divided(in_kv, per)), g.blocks - 1);
        hb = static_cast<int>(kv) * g.blocks + block;
        const int weight = weight_of(block);
        const int in_block = static_cast<int>(in_kv - static_cast<long long>(block) * per);
        const int first = max((in_block + weight - 1) / weight - kSharedRowUnits, 0);
        left -= (first + kSharedRowUnits) * weight - in_block;   // to the first tile that begins in the share
        if (first == tiles) return behind(groups, Hkv, kTile);
        from(first, weight);
        return left > 0;
    }
    // What is left begins behind this block.
    __device__ __forceinline__ bool behind(const KvGroup* groups, int Hkv, int kTile) {
        if (left <= 0) return false;
        if (++hb == g.blocks * Hkv) {
            hb = 0;
            load(groups, e + 1, kTile);
        }
        const int to = weight();
        left -= kSharedRowUnits * to;
        from(0, to);
        return left > 0;
    }
    __device__ __forceinline__ bool next(const KvGroup* groups, int Hkv, int kTile) {
        left -= count * weight();
        return behind(groups, Hkv, kTile);
    }
    __device__ __forceinline__ int kv() const { return hb / g.blocks; }
    __device__ __forceinline__ int row0() const { return hb % g.blocks * kRows; }
    __device__ __forceinline__ bool whole() const { return count == tiles; }
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
// Columns of a lane's row.
__device__ __forceinline__ void tmem_ld64(uint32_t at, float (&v)[64]) {
    uint32_t r[64];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
        "%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,"
        "%57,%58,%59,%60,%61,%62,%63"
        "}, [%64];\ntcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]),
          "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]),
          "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]),
          "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]),
          "=r"(r[63])
        : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16u(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Two bf16; what is above the largest becomes that, NaN stays.
__device__ __forceinline__ uint32_t pack2_finite(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A role's wait has given up, or another role's has: every role ends, without starting copies or products any more.
static __device__ __noinline__ void give_up(volatile int* abort, int* status) {
    if (!*abort) raise_status(status, QS_DEV_TIMEOUT);
    *abort = 1;
}
// Waits for a phase of a barrier, all lanes of a warp alike, until the limit or until a role has given up.  Few instructions
// where the phase is over: the roles' loops take turns in the instruction cache, and what they take is what they wait for
// (80 clocks against 400 of role_wait's, in the issuing warps).
__device__ __forceinline__ bool phase_wait(uint64_t* bar, uint32_t parity, volatile int* abort, const KvAttendParams& p) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .u32 n, a;\nmov.u32 %0, 1;\nmov.u32 n, 0;\nWAIT:\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n@p bra DONE;\n"
        "ld.volatile.shared.u32 a, [%3];\nadd.u32 n, n, 1;\nsetp.ge.u32 q, n, %4;\nsetp.ne.or.u32 q, a, 0, q;\n@!q bra WAIT;\n"
        "mov.u32 %0, 0;\nDONE:\n}\n"
        : "=&r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(smem_u32(const_cast<int*>(abort))), "r"(p.wait_polls) : "memory");
    if (__all_sync(kFull, ok != 0)) return true;
    give_up(abort, p.status);
    return false;
}

template <int D, bool kF16, bool kE4M3>
__global__ void __launch_bounds__(SharedShape<D>::kThreads, 1) kv_shared_kernel(const KvAttendParams p, const int box_rows, const int most_groups,
                                                                                const __grid_constant__ CUtensorMap k_map,
                                                                                const __grid_constant__ CUtensorMap v_map) {
    using S = SharedShape<D>;
    constexpr int kTile = S::kTile, kM = S::kM, kAlloc = 512;
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(1024) char smem[];
    SharedMisc& x = *reinterpret_cast<SharedMisc*>(smem + S::kMisc);
    const int tid = threadIdx.x, lane = tid & 31, worker = blockIdx.x;
    const int warp = __shfl_sync(kFull, tid >> 5, 0);   // the same for a warp, as the compiler can see
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
            tc::mbar_init(&x.full[s], kE4M3 || box_rows ? 1 : 33);
            tc::mbar_init(&x.free[s], kM);
        }
        for (int m = 0; m < 4; ++m) {
            tc::mbar_init(&x.sready[m], 2);   // the product, and its tile's mask
            tc::mbar_init(&x.pready[m], 4);
            tc::mbar_init(&x.odone[m], 1);
        }
        tc::mbar_init(&x.qfull, S::kSoftmax * 33);
        tc::mbar_init(&x.qfree, kM);
        tc::mbar_init(&x.drain, S::kIssuers);
        tc::mbar_fence_init();
        x.abort = 0;
    }
    if (!kE4M3 && box_rows && warp == S::kCopier) {
        prefetch_map(&k_map);
        prefetch_map(&v_map);
    }
    // the head, and a lane's group of the first 32 (there is room for most_groups)
    KvGroupHead head;
    int4 g0 = make_int4(0, 0, 0, 0), g1 = g0;
    bool fits;   // and the wait limit is not 0
    {
        const int4* const src = reinterpret_cast<const int4*>(head_at);
        const int4 h0 = __ldcg(src), h1 = __ldcg(src + 1);
        const long long units = __ldcg(&head_at->units);
        if (lane < most_groups) {
            g0 = __ldcg(reinterpret_cast<const int4*>(groups + lane));
            g1 = __ldcg(reinterpret_cast<const int4*>(groups + lane) + 1);
        }
        head.groups = h0.x;
        head.units = units;
        fits = groups_fit(p, h0, h1);
        // a limit of no polls gives up at the first wait
        if (head.groups != 0 && !fits && tid == 0)
            raise_status(p.status, groups_made_for(p, h0, h1) ? QS_DEV_TIMEOUT : QS_DEV_PAGES);
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(kFull, x.tmem, 0);
    volatile int* const abort = &x.abort;
    const int G = p.Hq / p.Hkv;
    using Part = SharedPart<S::kRows, S::kM == 2 && !kE4M3>;
    Part w;
    int copied = 0;   // tensors that this warp has begun to copy
    const bool live = fits && w.start(head, groups, g0, g1, worker, p.workers, p.Hkv, kTile);
    // Streams have their own S, P, O and softmax warps.  They are a block's halves (`two`), or, where it has one half, the part's
    // even and odd tiles.
    const bool fences = !kE4M3 && !box_rows;   // copies by cp.async, whose writes the product's issuer makes visible to the tensor core
    auto two_halves = [&](int rows) { return kM == 2 && rows > 128; };
    auto stream_of = [&](int t) { return kM == 2 ? t & 1 : 0; };   // of a part's tile where there is one half

    if (live && warp >= S::kCopier) {
        // ---- copies ----
        // A warp copies the keys or the values of every other tile; lanes look up two tokens each.
        const int pw = warp - S::kCopier, page_mask = (1 << p.page_shift) - 1;
        const bool values = pw & 1;
        const char* const pool = static_cast<const char*>(values ? p.v : p.k);
        const uint8_t* const exps = values ? p.v_exp : p.k_exp;
        const uint32_t lead = elect_lane();
        int s = pw, phase = 0, i = 0;   // i: tiles of the worker
        bool ok = true, more = true;    // ok: no wait has been given up
        while (more && ok) {
            const int kv_head = w.kv();
            const int32_t* const pages = p.table + static_cast<size_t>(w.g.owner) * p.max_pages;
            int id[2];
            auto look_up = [&](int tile) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int t = tile * kTile + k * 32 + lane;
                    id[k] = t < w.g.tokens ? __ldcg(pages + (t >> p.page_shift)) : -1;
                }
            };
            uint32_t on[2];     // tokens that are there
            long long row[2];   // of the pool
            int power[2];       // e4m3
            auto prepare = [&](int c) {   // the tile's rows; the pages of the warp's next one are looked up meanwhile
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int t = (w.tile + c) * kTile + k * 32 + lane;
                    const bool wanted = t < w.g.tokens, there = wanted && id[k] >= 0 && id[k] < p.n_pages;
                    if (wanted && !there) raise_status(p.status, QS_DEV_PAGES);
                    on[k] = __ballot_sync(kFull, there);
                    row[k] = there ? ((static_cast<long long>(id[k]) * p.Hkv + kv_head) << p.page_shift) + (t & page_mask) : 0;
                    if (kE4M3) power[k] = there ? __ldcg(exps + row[k]) : 127;
                }
                if (c + 2 < w.count) look_up(w.tile + c + 2);
            };
            // e4m3: 16 codes a lane and load, some tokens' in flight while those before are converted; D / 16 lanes take a token
            constexpr int kLanes = D / 16, kTokens = 32 / kLanes, kLoads = D == 64 ? 4 : 8, kSteps = kTile / (kTokens * kLoads);
            const int code_sg = lane % kLanes, code_row = lane / kLanes;
            uint4 codes[kE4M3 ? kLoads : 1], ahead[kE4M3 ? kLoads : 1];
            auto load = [&](int step) {
#pragma unroll
                for (int k = 0; k < (kE4M3 ? kLoads : 0); ++k) {
                    const int u = (step * kLoads + k) * kTokens + code_row;
                    const long long a = __shfl_sync(kFull, row[0], u & 31), b = __shfl_sync(kFull, row[1], u & 31);
                    const bool seen = ((u < 32 ? on[0] : on[1]) >> (u & 31)) & 1;
                    const char* const src = pool + (u < 32 ? a : b) * D + code_sg * 16;
                    ahead[kE4M3 ? k : 0] = seen ? __ldcg(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0);
                }
            };
            int c = (i & 1) == pw >> 1 ? 0 : 1;   // the first tile that is this warp's
            if (c < w.count) {
                look_up(w.tile + c);
                if (kE4M3) {
                    prepare(c);
                    load(0);
                }
            }
            for (; c < w.count && ok; c += 2) {
                if (!kE4M3) prepare(c);
                if (!values && lane == 0) {
                    volatile uint32_t* const mask = x.mask[(i + c) % kMaskRing];
                    mask[0] = on[0];
                    mask[1] = on[1];
                }
                const uint32_t stage = smem_u32(smem + S::kRing + s * S::kTensor);
                const bool whole = (on[0] & on[1]) == kFull;
                if constexpr (!kE4M3) {
                    if (copied * S::kCopiers >= S::kStages) ok = phase_wait(&x.free[s], phase ^ 1, abort, p);
                    if (!ok) break;
                    if (box_rows && whole) {
                        if (lane == 0) mbar_arrive_expect(&x.full[s], S::kTensor);
                        __syncwarp();
                        const uint32_t bar = smem_u32(&x.full[s]);
                        const CUtensorMap* const map = values ? &v_map : &k_map;
#pragma unroll 1
                        for (int u = 0; u < kTile; u += box_rows) {
                            const int at = __shfl_sync(kFull, static_cast<int>(u < 32 ? row[0] : row[1]), u & 31);
#pragma unroll 1
                            for (int b = 0; b < S::kBlocks; ++b) tma_box(stage + b * S::kBlock + u * 128, map, b * 64, at, bar, lead);
                        }
                    } else {
                        // 16 bytes a lane; zeros in place of what is not there
                        const int sg = lane & 7, row0 = lane >> 3;
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll 4
                            for (int k = 0; k < 8; ++k) {
                                const int u = k * 4 + row0;
                                const char* const src = pool + __shfl_sync(kFull, row[half], u) * (2 * D) + sg * 16;
                                const bool seen = (on[half] >> u) & 1;
                                const uint32_t to = stage + (half * 32 + u) * 128 + ((sg ^ (u & 7)) << 4);
#pragma unroll
                                for (int b = 0; b < S::kBlocks; ++b) cp_async16(to + b * S::kBlock, src + b * 128, seen);
                            }
                        if (box_rows) {   // the ends of what is shared only
                            cp_commit();
                            cp_wait<0>();
                            tc::fence_async_smem();
                        } else {
                            cp_async_arrive(&x.full[s]);
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&x.full[s]);
                    }
                } else {
                    const int powers[2] = {power[0], power[1]};
                    if (copied * S::kCopiers >= S::kStages) ok = phase_wait(&x.free[s], phase ^ 1, abort, p);
                    if (!ok) break;
#pragma unroll 1
                    for (int step = 0; step < kSteps; ++step) {
#pragma unroll
                        for (int k = 0; k < kLoads; ++k) codes[k] = ahead[k];
                        if (step + 1 < kSteps) {
                            load(step + 1);
                        } else if (c + 2 < w.count) {   // the warp's next tile
                            prepare(c + 2);
                            load(0);
                        }
#pragma unroll
                        for (int k = 0; k < kLoads; ++k) {
                            const int u = (step * kLoads + k) * kTokens + code_row;
                            const unsigned e0 = __shfl_sync(kFull, powers[0], u & 31), e1 = __shfl_sync(kFull, powers[1], u & 31), e = u < 32 ? e0 : e1;
                            // 2^(e - 127); 0 is the type's lowest power (2^-127, not a normal number), 255 NaN
                            const float two = e == 255 ? __uint_as_float(0x7fffffffu) : e ? __uint_as_float(e << 23) : 0x1p-127f;
                            const uint32_t w4[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
                            uint32_t y[8];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t lo, hi;
                                asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}"
                                    : "=r"(lo), "=r"(hi) : "r"(w4[j]));
                                const float2 a = __fmul2_rn(unpack2<true>(lo), make_float2(two, two));
                                const float2 b = __fmul2_rn(unpack2<true>(hi), make_float2(two, two));
                                y[2 * j] = pack2_finite(a.x, a.y);
                                y[2 * j + 1] = pack2_finite(b.x, b.y);
                            }
                            // entries 16 sg ...: pieces 2 (sg % 4) and the next of block sg / 4
                            const int piece = (code_sg & 3) * 2;
                            const uint32_t to = stage + (code_sg >> 2) * S::kBlock + u * 128;
                            st_shared16(to + ((piece ^ (u & 7)) << 4), y[0], y[1], y[2], y[3]);
                            st_shared16(to + (((piece + 1) ^ (u & 7)) << 4), y[4], y[5], y[6], y[7]);
                        }
                    }
                    tc::fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&x.full[s]);
                }
                ++copied;
                s += S::kCopiers;
                if (s >= S::kStages) s -= S::kStages, phase ^= 1;
            }
            i += w.count;
            more = w.next(groups, p.Hkv, kTile);
        }
        cp_commit();
        cp_wait<0>();
    } else if (live && warp >= S::kIssuer) {
        // ---- products ----
        const int stream = (warp - S::kIssuer) % kM;
        const bool scores = warp < S::kIssuer + kM;
        // S = Q K^T; a scale below zero is taken as -Q K^T (bit 13: A negated).  O += P V, B N-major.
        const uint32_t idS = idesc_f16(kF16, 128, kTile, false) | (p.scale < 0.0f ? 1u << 13 : 0u);
        constexpr uint32_t idO = idesc_f16(kF16, 128, D, false) | 1u << 16;
        const uint32_t lead = elect_lane(), base = smem_u32(smem);
        const uint32_t ring = desc_lo(base + S::kRing, scores ? 16 : S::kBlock), s_at = tmem + stream * S::kBuffers * kTile;
        int s = scores ? 0 : 1, phase = 0, parts = 0, n = 0;   // n: jobs that have been issued
        bool ok = true, more = true;
        while (more && ok) {
            const bool two = two_halves(min(S::kRows, w.g.rows - w.row0()));
            const uint32_t dq = desc_lo(base + (two ? stream * S::kQTile : 0), 16);
            if (scores) {
                ok = phase_wait(&x.qfull, parts++ & 1, abort, p);
                tc::fence_async_smem();   // the copies' writes, for the tensor core's reads
            }
            bool first = true;
#pragma unroll 1
            for (int c = 0; c < w.count && ok; ++c) {
                ok = phase_wait(&x.full[s], phase, abort, p);
                if (!ok) break;
                if (fences) tc::fence_async_smem();
                if (!two && stream_of(c) != stream) {   // the other stream's tile
                    if (lane == 0) mbar_arrive(&x.free[s]);
                } else {
                    const int buffer = S::buffer(stream, n);
                    const uint32_t buffer_at = s_at + (n & 1) * kTile, b0 = ring + s * (S::kTensor / 16);
                    if (scores) {
                        if (n >= S::kBuffers) ok = phase_wait(&x.odone[buffer], S::phase(n - S::kBuffers), abort, p);   // p before has been read
                        if (!ok) break;
                        if (lane == 0) mbar_arrive(&x.sready[buffer]);   // the tile's mask is there
                        tc::fence_after_sync();
#pragma unroll
                        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mma_f16_ss<kDescHi>(buffer_at, dq + (b * S::kQBlock + k * 32) / 16, b0 + (b * S::kBlock + k * 32) / 16, idS,
                                                    b > 0 || k > 0, lead);
                        commit_by(&x.sready[buffer], lead);
                    } else {
                        ok = phase_wait(&x.pready[buffer], S::phase(n), abort, p);
                        if (!ok) break;
                        tc::fence_after_sync();
#pragma unroll
                        for (int k = 0; k < kTile / 16; ++k)
                            mma_f16_ts<kDescHi>(tmem + S::kOCol + stream * D, buffer_at + k * 8, b0 + k * 128, idO, !first || k > 0, lead);
                        commit_by(&x.odone[buffer], lead);
                        first = false;
                    }
                    commit_by(&x.free[s], lead);
                    ++n;
                }
                s += 2;
                if (s >= S::kStages) s -= S::kStages, phase ^= 1;
            }
            if (scores && ok) commit_by(&x.qfree, lead);
            more = w.next(groups, p.Hkv, kTile);
        }
    } else if (live && warp < S::kSoftmax) {
        // ---- softmax ----
        const int stream = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t tlane = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
        const uint32_t o_at = tlane + S::kOCol + stream * D;
        // S carries the scale's sign; a scale of zero as next to nothing, so that the -inf of tokens that are not seen stays
        const float zs = fmaxf(fabsf(p.scale) * kLog2e, 0x1p-126f);
        constexpr float kAbove = kF16 ? kLazyLatent + kLiftLatent : kLazyLatent, kBelow = kLiftLatent - kFarLatent;
        float m = -INFINITY, high = -INFINITY, l = 0.0f, lr = 0.0f;   // reference, the highest so far, sums of p and of rounded p
        // Queries of w's block, this warp's 32 rows: a lane looks up a row, eight lanes copy it.
        auto queries = [&]() {
            const int i0 = w.row0(), rows = min(S::kRows, w.g.rows - i0), first = stream * 128 + (warp & 3) * 32, sg = lane & 7;
            const bool in = first + lane < rows;
            const int at_row = i0 + first + lane, member = in ? at_row / G : 0;
            const uint16_t* const mine = static_cast<const uint16_t*>(p.q) + (w.g.first + member) * p.q_row +
                                         (in ? w.kv() * G + at_row - member * G : 0) * p.q_head;
            const uint32_t to = smem_u32(smem + stream * S::kQTile);
            if (first < rows)
#pragma unroll 2
                for (int k = 0; k < 8; ++k) {
                    const int u = k * 4 + (lane >> 3), at = (warp & 3) * 32 + u;
                    const uint16_t* const q =
                        reinterpret_cast<const uint16_t*>(__shfl_sync(kFull, reinterpret_cast<unsigned long long>(mine), u)) + sg * 8;
                    const bool on = first + u < rows;
#pragma unroll
                    for (int b = 0; b < S::kBlocks; ++b) {
                        const uint32_t piece = to + b * S::kQBlock + at * 128 + ((sg ^ (at & 7)) << 4);
                        if (p.q_aligned) {
                            cp_async16(piece, on ? q + b * 64 : p.q, on);
                        } else {
                            uint16_t v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = on ? q[b * 64 + e] : 0;
                            st_shared16(piece, v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
                        }
                    }
                }
            cp_async_arrive(&x.qfull);
            __syncwarp();
            if (lane == 0) mbar_arrive(&x.qfull);
        };
        queries();
        int n = 0, i = 0, parts = 0;   // the stream's jobs, all tiles
        for (bool more = true; more;) {
            const int i0 = w.row0(), rows = min(S::kRows, w.g.rows - i0);
            const bool two = two_halves(rows);
            bool any = false;   // the stream has had a tile of this part
            m = high = -INFINITY;
            l = lr = 0.0f;
            for (int c = 0; c < w.count; ++c, ++i) {
                if (!two && stream_of(c) != stream) continue;
                const int buffer = S::buffer(stream, n);
                const uint32_t s_at = tlane + buffer * kTile;
                phase_wait(&x.sready[buffer], S::phase(n), abort, p);
                tc::fence_after_sync();
                const uint2 seen = *reinterpret_cast<const uint2*>(x.mask[i % kMaskRing]);
                if ((seen.x & seen.y) != kFull)
#pragma unroll 1
                for (int k = 0; k < kTile / 32; ++k) {   // scores of tokens that are not there
                    const uint32_t on = x.mask[i % kMaskRing][k];
                    if (on == kFull) continue;
#pragma unroll 1
                    for (int j = 0; j < 32; j += 16) {
                        float z[16];
                        tc::tmem_ld16(s_at + k * 32 + j, z);
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[e] = (on >> (j + e)) & 1 ? z[e] : -INFINITY;
                        tc::tmem_st16(s_at + k * 32 + j, z);
                    }
                    tc::wait_st();
                }
                float z[64], a = -INFINITY, b = -INFINITY;
                tmem_ld64(s_at, z);
#pragma unroll
                for (int j = 0; j < 64; j += 4) {
                    a = fmaxf(fmaxf(a, z[j]), z[j + 1]);
                    b = fmaxf(fmaxf(b, z[j + 2]), z[j + 3]);
                }
                const float top = fmaxf(a, b) * zs;
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
                    if (any) {
                        phase_wait(&x.odone[S::buffer(stream, n - 1)], S::phase(n - 1), abort, p);   // the products so far are in
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
                for (int k = 0; k < 64; k += 32) {
                    uint32_t w16[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float2 y = __ffma2_rn(make_float2(z[k + 2 * j], z[k + 2 * j + 1]), zs2, mz2);
                        y.x = exp2_fast(y.x);
                        y.y = exp2_fast(y.y);
                        ls = __fadd2_rn(ls, y);
                        w16[j] = pack2<kF16>(y.x, y.y);
                        lrs = __fadd2_rn(lrs, unpack2<kF16>(w16[j]));
                    }
                    tmem_st16u(s_at + k / 2, w16);   // over scores that are in registers
                }
                l += ls.x + ls.y;
                lr += lrs.x + lrs.y;
                tc::wait_st();
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&x.pready[buffer]);
                any = true;
                ++n;
            }
            // ---- the part's end ----
            const Part was = w;
            const bool whole = was.whole();
            int many = 1;   // workers that have a part of the block
            if (tid == 0 && was.tile == 0 && !whole) many = share_owner(head.units, was.last_tile(), Part::sharing(head.units, p.workers)) - worker + 1;
            more = w.next(groups, p.Hkv, kTile);
            if (more) {
                phase_wait(&x.qfree, parts++ & 1, abort, p);   // S of this part is done with its queries
                queries();
            }
            if (any) phase_wait(&x.odone[S::buffer(stream, n - 1)], S::phase(n - 1), abort, p);
            tc::fence_after_sync();
            const int at = two ? stream * 128 + row : row, at_row = i0 + at, member = at_row / G;   // of the block, of the group
            const size_t slot = part_slot(worker, was.tile == 0);
            const size_t out_row = (two ? 0 : static_cast<size_t>(stream) * p.R * p.Hq) +
                                   static_cast<size_t>(was.g.first + member) * p.Hq + was.kv() * G + at_row - member * G;
            if (at < rows) {
                if (whole)
                    p.pre_store_ml[out_row] = make_float4(m, m, l, lr);
                else
                    p.pre_ml[slot * S::kRows + stream * 128 + row] = make_float4(m, m, l, lr);
            }
            if (any) {
                // a part's sums lie column by column: 32 lanes' rows side by side
                float4* const to = whole ? reinterpret_cast<float4*>(p.pre_store) + out_row * (D / 4)
                                         : reinterpret_cast<float4*>(p.pre_part) + slot * (S::kRows * (D / 4)) + stream * 128 + row;
                const int column = whole ? 1 : S::kRows;
#pragma unroll 1
                for (int k = 0; k < D; k += 16) {
                    float v[16];
                    tc::tmem_ld16(o_at + k, v);
                    if (at < rows)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            to[(k / 4 + j) * column] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
            }
            if (tid == 0 && was.tile == 0) {
                p.pre_dir[was.g.block0 + was.hb] = make_int2(whole ? -1 : worker, kM == 2 && !two ? -many : many);
            }
            tc::fence_before_sync();
        }
        cp_commit();
        cp_wait<0>();
    }

    tc::fence_before_sync();
    __syncthreads();
    if (!kE4M3 && box_rows && *abort && warp >= S::kCopier && lane == 0) {
        // boxes may be under way: none may land in a CTA that has gone
        constexpr int kOwn = S::kStages / S::kCopiers;
        for (int k = max(0, copied - kOwn); k < copied; ++k)
            tc::mbar_wait(&x.full[warp - S::kCopier + k % kOwn * S::kCopiers], (k / kOwn) & 1, kDefaultWaitPolls);
    }
    __syncwarp();
    if (*abort && warp >= S::kIssuer && warp < S::kCopier) commit_by(&x.drain, elect_lane());   // of the products that it issued
    if (warp == S::kIssuer) {
        // products may be under way: wait for them before tensor memory goes back
        if (*abort && lane == 0 && !tc::mbar_wait(&x.drain, 0, kDefaultWaitPolls)) raise_status(p.status, QS_DEV_TEARDOWN);
        __syncwarp();
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, kAlloc);
    }
}

template <int D, bool kF16, bool kE4M3>
cudaError_t launch_shared(const qstate_kv_cfg& c, KvAttendParams p, cudaStream_t stream) {
    using S = SharedShape<D>;
    constexpr int kBytes = S::kMisc + sizeof(SharedMisc);
    static_assert(kBytes <= kLatSmem, "shared memory of an SM");
    const cudaError_t e = cudaFuncSetAttribute(kv_shared_kernel<D, kF16, kE4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    const int sms = device_sm_count();
    p.workers = sms < kKvSms ? sms : kKvSms;
    // Boxes of a page's tokens, a tile's at most: whole groups of eight rows of the swizzle, and rows of the pool
    // that 31 bits number.
    CUtensorMap k_map = {}, v_map = {};
    int box_rows = 0;
    const long long rows = static_cast<long long>(c.n_pages) * c.Hkv * c.page;
    if (!kE4M3 && c.page >= 8 && rows <= 0x7fffffffLL) {
        box_rows = c.page < S::kTile ? c.page : S::kTile;
        if (!pool_map(&k_map, p.k, D, rows, box_rows) || !pool_map(&v_map, p.v, D, rows, box_rows)) box_rows = 0;
    }
    return launch_chained(kv_shared_kernel<D, kF16, kE4M3>, p.workers, S::kThreads, kBytes, stream, true, p, box_rows, kv_most_groups(p.R),
                          k_map, v_map);
}

template <int D>
cudaError_t launch_shared_of(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    if (c.store == QSTATE_KV_E4M3) return launch_shared<D, false, true>(c, p, stream);
    return c.dtype == QSTATE_KV_F16 ? launch_shared<D, true, false>(c, p, stream) : launch_shared<D, false, false>(c, p, stream);
}

}  // namespace kv
}  // namespace qs
