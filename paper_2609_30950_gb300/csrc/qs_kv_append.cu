// qs_kv_append.cu -- new tokens' keys and values into their slots of the paged cache.
//
// Rows of the step are T x Hkv x d with strides of their own (views of a fused projection), the cache
// is (page, head, place in the page, entry).  In 16 bits this is a copy; in e4m3 each vector of d
// entries is first scaled by the power of two 2^-k, k the smallest with max|x| <= 448 * 2^k, which is
// exact, and its entries are then rounded to codes (nearest, ties to even): the codes' rounding is
// the only one.  Memory bounds both (16384 tokens of 8 heads of 128 in 16 bits: 134 MB in 21.3 us, 93 % of the copy rate;
// 20011 in e4m3: 124 MB in 21.4, 85 %); a step of some dozen tokens is a launch (1.5 us).
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kThreads = 256;

// Entry 0 of head h in a slot.
__device__ __forceinline__ size_t place(int slot, int h, int Hkv, int d, int sh) {
    const size_t page = static_cast<size_t>(slot >> sh);
    return (((page * Hkv + h) << sh) + (slot & ((1 << sh) - 1))) * static_cast<size_t>(d);
}

// kLanes lanes take a token's rows, both tensors at once: every load of up to four steps is in flight before the
// slot, loaded beside them, says where they go.
template <int kLanes>
struct TokenLanes {
    static constexpr int kTokens = kThreads / kLanes;
};

// 16 bits: kEntries entries a lane and step (8: 16 bytes; 1 where rows are not 16-byte aligned).
template <int kEntries, int kLanes>
__global__ void __launch_bounds__(kThreads) kv_copy_kernel(const KvAppendParams p, const int head_shift) {
    using Vec = typename std::conditional<kEntries == 8, uint4, uint16_t>::type;
    constexpr int kSteps = 4;
    chain_wait();
    const long long t = static_cast<long long>(blockIdx.x) * TokenLanes<kLanes>::kTokens + threadIdx.x / kLanes;
    const int part = threadIdx.x % kLanes;
    if (t >= p.T) return;
    int slot = p.slot[t];
    const int per_row = p.Hkv * p.d[0] / kEntries;
    for (int c0 = part; c0 < per_row; c0 += kSteps * kLanes) {
        Vec x[2][kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = c0 + i * kLanes, h = c >> head_shift, e = (c & ((1 << head_shift) - 1)) * kEntries;
#pragma unroll
            for (int y = 0; y < 2; ++y)
                if (c < per_row && y < p.tensors)
                    x[y][i] = *reinterpret_cast<const Vec*>(static_cast<const uint16_t*>(p.src[y]) + t * p.row[y] + h * p.head[y] + e);
        }
        if (slot >= p.n_slots) {
            raise_status(p.status, QS_DEV_PAGES);
            slot = -1;
        }
        if (slot < 0) return;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = c0 + i * kLanes, h = c >> head_shift, e = (c & ((1 << head_shift) - 1)) * kEntries;
#pragma unroll
            for (int y = 0; y < 2; ++y)
                if (c < per_row && y < p.tensors)
                    *reinterpret_cast<Vec*>(static_cast<uint16_t*>(p.dst[y]) + place(slot, h, p.Hkv, p.d[0], p.page_shift) + e) = x[y][i];
        }
    }
}

// e4m3: D / 16 lanes take a vector, 16 entries each.
template <int D, bool kAligned, int kLanes>
__global__ void __launch_bounds__(kThreads) kv_quant_kernel(const KvAppendParams p) {
    constexpr int kVec = D / 16;
    chain_wait();
    const long long t = static_cast<long long>(blockIdx.x) * TokenLanes<kLanes>::kTokens + threadIdx.x / kLanes;
    const int part = threadIdx.x % kLanes;
    int slot = t < p.T ? p.slot[t] : -1;
    const int per_row = p.Hkv * kVec;
    if (part == 0 && slot >= p.n_slots) raise_status(p.status, QS_DEV_PAGES);
    // every lane of a warp stays for the shuffles
    for (int c0 = 0; c0 < per_row; c0 += kLanes) {
        const int c = c0 + part, h = c / kVec, e = c % kVec * 16;
        const bool in = t < p.T && c < per_row;
        uint32_t w[2][8] = {};
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const uint16_t* const src = static_cast<const uint16_t*>(p.src[y]) + t * p.row[y] + h * p.head[y] + e;
            if (in && kAligned) {
                const uint4 u = *reinterpret_cast<const uint4*>(src), v = *reinterpret_cast<const uint4*>(src + 8);
                w[y][0] = u.x, w[y][1] = u.y, w[y][2] = u.z, w[y][3] = u.w;
                w[y][4] = v.x, w[y][5] = v.y, w[y][6] = v.z, w[y][7] = v.w;
            } else if (in) {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[y][j] = src[2 * j] | static_cast<uint32_t>(src[2 * j + 1]) << 16;
            }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            // |x| as integers order as the numbers do, NaN and infinity on top
            unsigned top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, max(w[y][j] << 16 & 0x7fffffffu, w[y][j] & 0x7fff0000u));
#pragma unroll
            for (int o = kVec / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
            // max|x| = m 2^e, 1 <= m < 2: k = e - 8 where m <= 1.75 = 448 / 2^8, else e - 7
            const bool fine = top < 0x7f800000u;
            int k = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
            k = top == 0 ? 0 : max(k, -126);
            const float inv = __uint_as_float(static_cast<unsigned>(127 - k) << 23);
            uint32_t out[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t code = 0;
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint32_t u = w[y][2 * j + m];
                    const float2 v = make_float2(__uint_as_float(u << 16) * inv, __uint_as_float(u & 0xffff0000u) * inv);
                    code |= static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3)) << (16 * m);
                }
                out[j] = fine ? code : 0u;
            }
            if (in && slot >= 0 && slot < p.n_slots) {
                const size_t at = place(slot, h, p.Hkv, 1, p.page_shift);
                *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.dst[y]) + at * D + e) = make_uint4(out[0], out[1], out[2], out[3]);
                if (e == 0) p.exps[y][at] = fine ? static_cast<uint8_t>(k + 127) : 255;
            }
        }
    }
}

// Blocks of tokens, so that the hardware deals them out as SMs come free.
template <int kLanes>
unsigned token_blocks(int T) { return (static_cast<unsigned>(T) + TokenLanes<kLanes>::kTokens - 1) / TokenLanes<kLanes>::kTokens; }

template <int D>
cudaError_t launch_quant(bool aligned, const KvAppendParams& p, cudaStream_t stream) {
    constexpr int kFew = D / 16 > 8 ? D / 16 : 8;   // lanes of a token of one or two heads
    const bool few = p.Hkv * (D / 16) <= kFew;
    if (few && aligned) return launch_chained(kv_quant_kernel<D, true, kFew>, token_blocks<kFew>(p.T), kThreads, 0, stream, true, p);
    if (few) return launch_chained(kv_quant_kernel<D, false, kFew>, token_blocks<kFew>(p.T), kThreads, 0, stream, true, p);
    if (aligned) return launch_chained(kv_quant_kernel<D, true, 32>, token_blocks<32>(p.T), kThreads, 0, stream, true, p);
    return launch_chained(kv_quant_kernel<D, false, 32>, token_blocks<32>(p.T), kThreads, 0, stream, true, p);
}

template <int kEntries>
cudaError_t launch_copy(const KvAppendParams& p, cudaStream_t stream) {
    // entries of a head as a power of two of steps; one head needs none
    int shift = 30;
    if (p.Hkv > 1)
        for (shift = 0; (kEntries << shift) < p.d[0];) ++shift;
    if (p.Hkv * p.d[0] / kEntries <= 8)
        return launch_chained(kv_copy_kernel<kEntries, 8>, token_blocks<8>(p.T), kThreads, 0, stream, true, p, shift);
    return launch_chained(kv_copy_kernel<kEntries, 32>, token_blocks<32>(p.T), kThreads, 0, stream, true, p, shift);
}

}  // namespace

cudaError_t launch_kv_append(const qstate_kv_cfg& c, const KvAppendParams& p, cudaStream_t stream) {
    bool aligned = true;   // every vector of 8 entries starts on 16 bytes
    for (int x = 0; x < p.tensors; ++x)
        aligned = aligned && reinterpret_cast<uintptr_t>(p.src[x]) % 16 == 0 && p.row[x] % 8 == 0 &&
                  (p.head[x] % 8 == 0 || p.Hkv == 1);
    if (c.store == QSTATE_KV_E4M3) {
        if (p.d[0] == 64) return launch_quant<64>(aligned, p, stream);
        return p.d[0] == 128 ? launch_quant<128>(aligned, p, stream) : launch_quant<256>(aligned, p, stream);
    }
    return aligned ? launch_copy<8>(p, stream) : launch_copy<1>(p, stream);
}

}  // namespace qs
