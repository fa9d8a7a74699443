// qs_kv_latent.cuh -- one new token of each request against one latent vector a token, shared by all heads.
//
// z_t = scale q_h.c_t over the dk entries of c_t, o_h = sum_t e^{z_t} c_t[:dv] / sum_t e^{z_t}.  A token's
// 2 dk bytes meet 2 H (dk + dv) operations: 121 a byte at 64 heads of 512 + 64, more than the
// register-fed matrix products sustain beside the loads, so both products run on the tensor cores
// with their sums in tensor memory, and the cache's bytes stay the bound.
//
// A tile is 64 tokens, stored once in shared memory (rows of 128 bytes in blocks of 64 entries, 128-byte
// swizzle) and read in both directions:
//     S^T [64 tokens x heads] = C [64 x dk] Q^T        C with dk contiguous (K-major)
//     O^T [dv x heads]       += C^T [dv x 64] P        the same bytes with dv contiguous (M-major)
// Tokens and dv are the products' rows, so up to 64 heads are their columns and few heads waste nothing;
// more heads go to further CTAs that walk the same tiles at the same time and find them in L2.
//   warps 0-3   softmax: 16 tokens each from S^T, p to shared memory in 16 bits; at a row's end o
//   warp 4      issues the products; S of the next tile goes ahead of O of this one
//   warps 5-8   copy tiles (and, where a row begins, its queries) with cp.async, zeros for what is not seen
// As in the kernel for heads, the softmax reference follows the maximum only when that has outgrown it by
// 2^8; all tokens of a row share one reference, so the four warps vote.  p goes into the second product
// as hi + lo of two 16-bit values, since one alone would add as much error as the rounding of o; lo lies
// in the tile's last block where that holds no values and has been read by then.
#pragma once

#include "qs_kv_tiles.cuh"
#include "qs_tc.cuh"

namespace qs {
namespace kv {

constexpr int kLatTile = 64;
constexpr int kLatThreads = 9 * 32;
constexpr int kBlockBytes = kLatTile * 128;   // 64 tokens x 64 entries
constexpr int kMaxStages = 4;
constexpr float kLazyLatent = 8.0f;

struct LatentGeo {
    int blocks;        // of 64 entries, the last may be half
    int stages, smem, groups, per_group, workers;
};

// Shared memory behind the tiles, the queries and p.
struct LatentMisc {
    uint64_t full[kMaxStages], free[kMaxStages], sready[2], pready, drain;
    uint64_t mask[kMaxStages];
    float top[4][64], corr[64], ref[64], sum[64];
    long long scratch[16];
    uint32_t tmem;
    int abort;
};

// Products of 16-bit types, FP32 sums: M x N, A optionally M-major.
__host__ __device__ constexpr uint32_t idesc_f16(bool f16, int M, int N, bool a_m_major) {
    return (1u << 4) | ((f16 ? 0u : 1u) << 7) | ((f16 ? 0u : 1u) << 10) | ((a_m_major ? 1u : 0u) << 15) |
           (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
// Operand in 128-byte rows with the 128-byte swizzle.  K-major: sbo between groups of 8 rows.  M-major: lbo
// between blocks of 64 entries, sbo between groups of 8 of K.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return tc::smem_desc(addr, lbo, sbo) | (static_cast<uint64_t>(2u) << 61);
}
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
}
// 16 lanes x 8 N columns: register 4 j + i of lane t is row t / 4 + 8 (i / 2), column 8 j + 2 (t % 4) + i % 2.
template <int N>
__device__ __forceinline__ void tmem_ld_rows(uint32_t at, float (&v)[4 * N]) {
    static_assert(N == 2 || N == 4 || N == 8, "columns in eights");
    uint32_t r[4 * N];
    if constexpr (N == 2)
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\ntcgen05.wait::ld.sync.aligned;\n"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(at) : "memory");
    else if constexpr (N == 4)
        asm volatile(
            "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
            "tcgen05.wait::ld.sync.aligned;\n"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
              "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
            : "r"(at) : "memory");
    else
        asm volatile(
            "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
            "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\ntcgen05.wait::ld.sync.aligned;\n"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
              "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
              "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
              "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
            : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void stmatrix4t(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
// An arrival (of those that the barrier was told to expect) when this thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 128;\n" ::: "memory"); }
__device__ __forceinline__ bool softmax_any(bool x) {
    int any;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %1, 0;\nbar.red.or.pred q, 1, 128, p;\nselp.s32 %0, 1, 0, q;\n}\n"
                 : "=r"(any) : "r"(static_cast<int>(x)) : "memory");
    return any != 0;
}

// Waits for a phase of a barrier; gives up after the limit, or at once where another role has.  Every role
// runs to its end all the same (so that no one waits for a warp that left), without starting copies or
// products any more.
__device__ __forceinline__ bool role_wait(uint64_t* bar, uint32_t parity, volatile int* abort, const KvAttendParams& p) {
    for (int it = 0; it < p.wait_polls; ++it) {
        if (tc::mbar_try_wait(bar, parity)) return true;
        if (*abort) return false;
    }
    *abort = 1;
    raise_status(p.status, QS_DEV_TIMEOUT);
    return false;
}

template <int DV, int kN, bool kF16>
__global__ void __launch_bounds__(kLatThreads) kv_latent_kernel(const KvAttendParams p, const LatentGeo g) {
    using W = Walk<kLatTile, 1>;
    constexpr int kOCols = DV / 128 * kN, kCols = kOCols + 2 * kN;
    constexpr int kAlloc = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    constexpr int kPer = kN / 4;   // heads a lane holds
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(1024) char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    char* const tiles = smem;
    char* const queries = tiles + g.stages * g.blocks * kBlockBytes;
    char* const probs = queries + g.blocks * kN * 128;
    const bool lo_in_tile = p.dk > DV;
    LatentMisc& x = *reinterpret_cast<LatentMisc*>(probs + (lo_in_tile ? 1 : 2) * kN * 128);
    const int worker = blockIdx.x / g.groups, group = blockIdx.x - worker * g.groups;
    const int h0 = group * g.per_group, heads = min(g.per_group, p.Hq - h0);
    chain_release();   // the kernel that joins split rows may take its place

    // requests without tokens
    for (int r = worker; r < p.R; r += g.workers)
        if (clamped_len(p, r, false) == 0) {
            uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.o) + (static_cast<size_t>(r) * p.Hq + h0) * DV);
            for (int i = tid; i < heads * (DV / 8); i += kLatThreads) o[i] = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = tid; i < heads; i += kLatThreads) p.lse[static_cast<size_t>(r) * p.Hq + h0 + i] = -INFINITY;
        }

    if (warp == 4) {
        tc::tmem_alloc(&x.tmem, kAlloc);
        tc::tmem_relinquish();
    }
    if (tid == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            tc::mbar_init(&x.full[s], 128 + 4);
            tc::mbar_init(&x.free[s], 1);
        }
        tc::mbar_init(&x.sready[0], 1);
        tc::mbar_init(&x.sready[1], 1);
        tc::mbar_init(&x.pready, 4);
        tc::mbar_init(&x.drain, 1);
        tc::mbar_fence_init();
        x.abort = 0;
    }
    const Share share = make_share<kLatThreads, kLatTile, 1>(p, 1, worker, g.workers, x.scratch);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = x.tmem;
    const int n = static_cast<int>(share.u1 - share.u0);
    volatile int* const abort = &x.abort;
    if (group == 0 && tid == 0 && n <= 0) p.split[worker] = 0;

    if (n > 0 && warp >= 5) {
        // ---- copies ----
        const int pw = warp - 5, page_mask = (1 << p.page_shift) - 1;
        W w;
        w.start(p, share);
        auto look_up = [&]() {
            const int t = w.span.base + w.tile * kLatTile + pw * 16 + lane;
            return lane < 16 && t < w.span.end ? __ldg(p.table + static_cast<size_t>(w.r) * p.max_pages + (t >> p.page_shift)) : -1;
        };
        int id = look_up(), s = 0;
        for (int i = 0; i < n; ++i) {
            bool ok = i < g.stages || role_wait(&x.free[s], (i / g.stages - 1) & 1, abort, p);
            const int r = w.r, t = w.span.base + w.tile * kLatTile + pw * 16 + lane;
            const bool begins = i == 0 || w.tile == 0;
            const bool seen = lane < 16 && t < w.span.end, there = id >= 0 && id < p.n_pages;
            if (seen && !there) raise_status(p.status, QS_DEV_PAGES);
            const uint32_t on = __ballot_sync(kFull, seen && there) & 0xffffu;
            if (lane == 0) reinterpret_cast<volatile uint16_t*>(&x.mask[s])[pw] = static_cast<uint16_t>(on);
            const long long mine = there && seen ? ((static_cast<long long>(id) << p.page_shift) + (t & page_mask)) : 0;
            const char* src[4];
            const int seg = lane & 7, row0 = lane >> 3;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                src[k] = static_cast<const char*>(p.k) + __shfl_sync(kFull, mine, k * 4 + row0) * (2 * p.dk) + seg * 16;
            if (i + 1 < n) {
                w.next(p, 1);
                id = look_up();
            }
            // the queries of the row before are no longer read once S of its last tile is there
            if (begins && i > 0) ok = ok && role_wait(&x.sready[(i - 1) & 1], ((i - 1) >> 1) & 1, abort, p);
            if (ok) {
                if (begins) {
                    const uint16_t* const q = static_cast<const uint16_t*>(p.q) + r * p.q_row + h0 * p.q_head;
                    for (int b = 0; b < g.blocks; ++b)
                        for (int e = tid - 160; e < kN * 8; e += 128) {
                            const int h = e >> 3, sg = e & 7, col = b * 64 + sg * 8;
                            const uint32_t to = smem_u32(queries + (b * kN + h) * 128 + ((sg ^ (h & 7)) << 4));
                            if (p.q_aligned) {
                                const bool in = h < heads && col < p.dk;
                                cp_async16(to, in ? q + h * p.q_head + col : p.q, in);
                            } else {
                                uint16_t v[8];
#pragma unroll
                                for (int k = 0; k < 8; ++k) v[k] = h < heads && col < p.dk ? q[h * p.q_head + col + k] : 0;
                                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v[0] | v[1] << 16),
                                             "r"(v[2] | v[3] << 16), "r"(v[4] | v[5] << 16), "r"(v[6] | v[7] << 16) : "memory");
                            }
                        }
                }
                const uint32_t to = smem_u32(tiles + s * g.blocks * kBlockBytes) + (pw * 16 + row0) * 128;
                for (int b = 0; b < g.blocks; ++b)
                    if (b * 64 + seg * 8 < p.dk) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int row = k * 4 + row0;
                            cp_async16(to + b * kBlockBytes + k * 512 + ((seg ^ (row & 7)) << 4), src[k] + b * 128, (on >> row) & 1);
                        }
                    }
            }
            cp_async_arrive(&x.full[s]);
            __syncwarp();
            if (lane == 0) mbar_arrive(&x.full[s]);
            s = s + 1 == g.stages ? 0 : s + 1;
        }
        cp_commit();
        cp_wait<0>();
    } else if (n > 0 && warp == 4) {
        // ---- products ----
        if (lane == 0) {
            constexpr uint32_t idS = idesc_f16(kF16, 64, kN, false), idO = idesc_f16(kF16, 128, kN, true);
            const uint32_t q32 = smem_u32(queries), p32 = smem_u32(probs), t32 = smem_u32(tiles);
            W w;
            w.start(p, share);
            auto scores = [&](int i) {
                const int s = i % g.stages;
                if (!role_wait(&x.full[s], (i / g.stages) & 1, abort, p)) return;
                tc::fence_async_smem();   // the copies' writes, for the tensor core's reads
                tc::fence_after_sync();
                const uint32_t tile = t32 + s * g.blocks * kBlockBytes, d = tmem + kOCols + (i & 1) * kN;
                for (int k = 0; k < p.dk / 16; ++k)
                    mma_f16_ss(d, desc_sw128(tile + (k >> 2) * kBlockBytes + (k & 3) * 32, 16, 1024),
                               desc_sw128(q32 + (k >> 2) * (kN * 128) + (k & 3) * 32, 16, 1024), idS, k > 0);
                tc::mma_commit(&x.sready[i & 1]);
            };
            scores(0);
            for (int i = 0; i < n; ++i) {
                if (i + 1 < n) scores(i + 1);
                const bool begins = i == 0 || w.tile == 0;
                if (role_wait(&x.pready, i & 1, abort, p)) {
                    tc::fence_after_sync();
                    const int s = i % g.stages;
                    const uint32_t tile = t32 + s * g.blocks * kBlockBytes;
                    const uint32_t lo32 = lo_in_tile ? tile + DV / 64 * kBlockBytes : p32 + kN * 128;
#pragma unroll
                    for (int c = 0; c < DV / 128; ++c)
#pragma unroll
                        for (int k = 0; k < kLatTile / 16; ++k) {
                            const uint64_t a = desc_sw128(tile + 2 * c * kBlockBytes + k * 2048, kBlockBytes, 1024);
                            mma_f16_ss(tmem + c * kN, a, desc_sw128(p32 + k * 32, 16, 1024), idO, !begins || k > 0);
                            mma_f16_ss(tmem + c * kN, a, desc_sw128(lo32 + k * 32, 16, 1024), idO, true);
                        }
                    tc::mma_commit(&x.free[s]);
                }
                if (i + 1 < n) w.next(p, 1);
            }
        }
    } else if (n > 0) {
        // ---- softmax ----
        const int quad = lane >> 2, t4 = lane & 3;
        const uint32_t tlane = tmem + (static_cast<uint32_t>(32 * warp) << 16);
        const uint32_t p32 = smem_u32(probs);
        const float zs = p.scale * kLog2e;
        float m[kPer], l[kPer];
        int prev = 0, s = 0, began = 0, split = 0;   // prev: stage of the tile before
        W w;
        w.start(p, share);
        for (int i = 0; i < n; ++i) {
            const bool begins = i == 0 || w.tile == 0, row_ends = w.tile == w.span.tiles - 1, ends = row_ends || i + 1 == n;
            if (begins) {
                began = w.tile;
#pragma unroll
                for (int k = 0; k < kPer; ++k) m[k] = -INFINITY, l[k] = 0.0f;
            }
            role_wait(&x.full[s], (i / g.stages) & 1, abort, p);
            role_wait(&x.sready[i & 1], (i >> 1) & 1, abort, p);
            tc::fence_after_sync();
            float z[2 * kPer];
            tmem_ld_rows<kN / 8>(tlane + kOCols + (i & 1) * kN, z);
            const uint32_t on = reinterpret_cast<volatile uint16_t*>(&x.mask[s])[warp];
            bool grown = false;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {   // k: head 8 (k / 2) + 2 t4 + k % 2, tokens quad and quad + 8
                float& a = z[4 * (k >> 1) + (k & 1)];
                float& b = z[4 * (k >> 1) + (k & 1) + 2];
                a = (on >> quad) & 1 ? a * zs : -INFINITY;
                b = (on >> (quad + 8)) & 1 ? b * zs : -INFINITY;
                grown = grown || fmaxf(a, b) > m[k] + kLazyLatent;
            }
            const uint32_t prev_parity = i > 0 ? ((i - 1) / g.stages) & 1 : 0;
            if (softmax_any(grown)) {
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    float top = fmaxf(z[4 * (k >> 1) + (k & 1)], z[4 * (k >> 1) + (k & 1) + 2]);
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
                    if (quad == 0) x.top[warp][8 * (k >> 1) + 2 * t4 + (k & 1)] = top;
                }
                softmax_sync();
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int h = 8 * (k >> 1) + 2 * t4 + (k & 1);
                    const float now = fmaxf(fmaxf(fmaxf(x.top[0][h], x.top[1][h]), fmaxf(x.top[2][h], x.top[3][h])), m[k]);
                    const float c = part_weight(m[k], now);
                    l[k] *= c;
                    m[k] = now;
                    if (warp == 0 && quad == 0) x.corr[h] = c;
                }
                softmax_sync();
                if (!begins) {
                    role_wait(&x.free[prev], prev_parity, abort, p);   // the products so far are in
                    tc::fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < kOCols; c += 16) {
                        float v[16];
                        tc::tmem_ld16(tlane + c, v);
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] *= x.corr[(c + k) % kN];
                        tc::tmem_st16(tlane + c, v);
                    }
                    tc::wait_st();
                }
            }
            uint32_t hi[kPer], lo[kPer];
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
            for (int j = 0; j < kPer; ++j) {
                hi[j] = pack2<kF16>(z[2 * j], z[2 * j + 1]);
                const float2 r = unpack2<kF16>(hi[j]);
                lo[j] = pack2<kF16>(z[2 * j] - r.x, z[2 * j + 1] - r.y);
            }
            const uint32_t lo32 = lo_in_tile ? smem_u32(tiles + (s * g.blocks + DV / 64) * kBlockBytes) : p32 + kN * 128;
            if (i > 0) role_wait(&x.free[prev], prev_parity, abort, p);   // p of the tile before has been read
#pragma unroll
            for (int j = 0; j < kN / 8; j += 2) {
                const int mat = lane >> 3, h = (j + (mat >> 1)) * 8 + (lane & 7), chunk = warp * 2 + (mat & 1);
                const int to = h * 128 + ((chunk ^ (h & 7)) << 4);
                stmatrix4t(p32 + to, hi[2 * j], hi[2 * j + 1], hi[2 * j + 2], hi[2 * j + 3]);
                stmatrix4t(lo32 + to, lo[2 * j], lo[2 * j + 1], lo[2 * j + 2], lo[2 * j + 3]);
            }
            tc::fence_async_smem();
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&x.pready);

            if (ends) {
                // ---- the row's end ----
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int h = 8 * (k >> 1) + 2 * t4 + (k & 1);
                    float sum = l[k];
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(kFull, sum, o);
                    if (quad == 0) {
                        x.top[warp][h] = sum;
                        if (warp == 0) x.ref[h] = m[k];
                    }
                }
                softmax_sync();
                const bool whole = began == 0 && row_ends;
                int slot = 0, parts = 0;
                if (!whole) {
                    const Joint jt = joint_of(share.total, share.u0 + i - w.tile, w.span.tiles, g.workers);
                    slot = part_slot(worker, jt.first == worker);
                    if (jt.first == worker) parts = jt.n;
                }
                const size_t row = static_cast<size_t>(w.r) * p.Hq + h0;
                const size_t prow = (static_cast<size_t>(slot) * g.groups + group) * kN;
                if (tid < kN) {
                    const float sum = x.top[0][tid] + x.top[1][tid] + x.top[2][tid] + x.top[3][tid], ref = x.ref[tid];
                    x.sum[tid] = sum == 0.0f ? 0.0f : 1.0f / sum;
                    if (!whole)
                        reinterpret_cast<float2*>(p.part_ml)[prow + tid] = make_float2(ref, sum);
                    else if (p.lse && tid < heads)
                        p.lse[row + tid] = sum == 0.0f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
                }
                if (parts) {   // the row that this CTA begins and others end
                    split = parts;
                    if (group == 0 && tid == 0) p.split[kKvWorkers + worker] = w.r;
                }
                softmax_sync();
                role_wait(&x.free[s], (i / g.stages) & 1, abort, p);
                tc::fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < kOCols; c += 16) {
                    float v[16];
                    tc::tmem_ld16(tlane + c, v);
                    const int dim = (c / kN) * 128 + warp * 32 + lane, hb = c % kN;
                    if (whole) {
                        uint16_t* const o = static_cast<uint16_t*>(p.o) + (row + hb) * DV + dim;
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (hb + k < heads) o[k * DV] = static_cast<uint16_t>(pack2<kF16>(v[k] * x.sum[hb + k], 0.0f));
                    } else {
                        float* const o = p.part + (prow + hb) * DV + dim;
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (hb + k < heads) o[k * DV] = v[k];
                    }
                }
            }
            prev = s;
            s = s + 1 == g.stages ? 0 : s + 1;
            if (i + 1 < n) w.next(p, 1);
        }
        if (group == 0 && tid == 0) p.split[worker] = split;
    }
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 4) {
        if (lane == 0 && *abort) {   // products may be under way: wait for them before tensor memory goes back
            tc::mma_commit(&x.drain);
            if (!tc::mbar_wait(&x.drain, 0, kDefaultWaitPolls)) raise_status(p.status, QS_DEV_TEARDOWN);
        }
        __syncwarp();
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, kAlloc);
    }
}

// Joins the rows that several CTAs share: a warp for each of a split row's heads.  The CTA that begins a row
// has left its request and the number of parts.
template <int DV, bool kF16>
__global__ void __launch_bounds__(128) kv_latent_join_kernel(const KvAttendParams p, const LatentGeo g, const int kN) {
    chain_wait();
    const int per = (g.per_group + 3) / 4;
    const int quad = blockIdx.x % per, rest = blockIdx.x / per, group = rest % g.groups, worker = rest / g.groups;
    const int n = __ldcg(p.split + worker);
    const int h = quad * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (n < 2 || h >= g.per_group || group * g.per_group + h >= p.Hq) return;
    const int r = __ldcg(p.split + kKvWorkers + worker);
    auto at = [&](int i) { return (static_cast<size_t>(part_slot(worker + i, i == 0)) * g.groups + group) * kN + h; };
    const float2* const ml = reinterpret_cast<const float2*>(p.part_ml);
    float M = -INFINITY, L = 0.0f;
    for (int i = lane; i < n; i += 32) M = fmaxf(M, __ldcg(ml + at(i)).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(kFull, M, o));
    float4 acc[DV / 128] = {};
    for (int i0 = 0; i0 < n; i0 += 32) {
        float2 mine = make_float2(-INFINITY, 0.0f);
        if (i0 + lane < n) mine = __ldcg(ml + at(i0 + lane));
        const float weight = part_weight(mine.x, M);
        L += mine.y * weight;
        const int many = min(32, n - i0);
#pragma unroll 4
        for (int i = 0; i < many; ++i) {
            const float c = __shfl_sync(kFull, weight, i);
            const float4* const src = reinterpret_cast<const float4*>(p.part + at(i0 + i) * DV) + lane;
#pragma unroll
            for (int k = 0; k < DV / 128; ++k) {
                const float4 v = __ldcg(src + k * 32);
                acc[k].x += c * v.x;
                acc[k].y += c * v.y;
                acc[k].z += c * v.z;
                acc[k].w += c * v.w;
            }
        }
    }
    L = warp_sum(L);
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const size_t row = static_cast<size_t>(r) * p.Hq + group * g.per_group + h;
#pragma unroll
    for (int k = 0; k < DV / 128; ++k) {
        uint2 w;
        w.x = pack2<kF16>(acc[k].x * inv, acc[k].y * inv);
        w.y = pack2<kF16>(acc[k].z * inv, acc[k].w * inv);
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o) + row * DV + k * 128 + lane * 4) = w;
    }
    if (lane == 0 && p.lse) p.lse[row] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// Groups of at most 64 heads, products of 16, 32 or 64 columns; as many tiles in flight as fit beside the
// queries, and two CTAs on an SM where each gets two.
inline LatentGeo latent_geo(int Hq, int dk, int dv, int sms, int* cols) {
    if (sms > kKvSms) sms = kKvSms;
    LatentGeo g;
    g.groups = (Hq + 63) / 64;
    g.per_group = (Hq + g.groups - 1) / g.groups;
    const int N = g.per_group <= 16 ? 16 : g.per_group <= 32 ? 32 : 64;
    *cols = N;
    g.blocks = (dk + 63) / 64;
    const int fixed = g.blocks * N * 128 + (dk > dv ? 1 : 2) * N * 128 + static_cast<int>(sizeof(LatentMisc)), tile = g.blocks * kBlockBytes;
    constexpr int kMost = 227 * 1024, kHalf = 113 * 1024;
    const int limit = fixed + 2 * tile <= kHalf ? kHalf : kMost;
    g.stages = (limit - fixed) / tile;
    if (g.stages > kMaxStages) g.stages = kMaxStages;
    g.smem = fixed + g.stages * tile;
    g.workers = sms * (limit == kHalf ? 2 : 1) / g.groups;
    if (g.workers < 1) g.workers = 1;
    if (g.workers > kKvWorkers) g.workers = kKvWorkers;
    return g;
}

template <int DV, int kN, bool kF16>
cudaError_t launch_latent(const KvAttendParams& p, const LatentGeo& g, cudaStream_t stream) {
    auto* kernel = kv_latent_kernel<DV, kN, kF16>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, g.smem);
    if (e != cudaSuccess) return e;
    kernel<<<g.workers * g.groups, kLatThreads, g.smem, stream>>>(p, g);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const int grid = g.workers * g.groups * ((g.per_group + 3) / 4);
    return launch_chained(kv_latent_join_kernel<DV, kF16>, grid, 128, 0, stream, true, p, g, kN);
}

template <int DV>
cudaError_t launch_latent_of(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    int N = 0;
    const LatentGeo g = latent_geo(p.Hq, p.dk, DV, device_sm_count(), &N);
    const bool f16 = c.dtype == QSTATE_KV_F16;
    if (N == 16) return f16 ? launch_latent<DV, 16, true>(p, g, stream) : launch_latent<DV, 16, false>(p, g, stream);
    if (N == 32) return f16 ? launch_latent<DV, 32, true>(p, g, stream) : launch_latent<DV, 32, false>(p, g, stream);
    return f16 ? launch_latent<DV, 64, true>(p, g, stream) : launch_latent<DV, 64, false>(p, g, stream);
}

}  // namespace kv
}  // namespace qs
