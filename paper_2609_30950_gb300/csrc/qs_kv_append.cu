// qs_kv_append.cu -- new tokens' keys and values into their slots of the paged cache.
//
// Rows of the step are T x Hkv x d with strides of their own (views of a fused projection), the cache
// is (page, head, place in the page, entry).  In 16 bits this is a copy; in e4m3 each vector of d
// entries is first scaled by the power of two 2^-k, k the smallest with max|x| <= 448 * 2^k, which is
// exact, and its entries are then rounded to codes (nearest, ties to even): the codes' rounding is
// the only one.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "qs_common.cuh"

namespace qs {
namespace {

constexpr int kThreads = 256;

// Entry 0 of head h in a slot.
__device__ __forceinline__ size_t place(int slot, int h, int Hkv, int d, int sh) {
    const size_t page = static_cast<size_t>(slot >> sh);
    return (((page * Hkv + h) << sh) + (slot & ((1 << sh) - 1))) * static_cast<size_t>(d);
}

// 16 bits: V entries a thread and step (8: 16 bytes; 1 where rows are not 16-byte aligned).
template <int V>
__global__ void __launch_bounds__(kThreads) kv_copy_kernel(const KvAppendParams p) {
    using Vec = typename std::conditional<V == 8, uint4, uint16_t>::type;
    for (int x = 0; x < p.tensors; ++x) {
        const int per_head = p.d[x] / V, per_row = p.Hkv * per_head;
        const long long n = static_cast<long long>(p.T) * per_row;
        const uint16_t* src = static_cast<const uint16_t*>(p.src[x]);
        uint16_t* dst = static_cast<uint16_t*>(p.dst[x]);
        for (long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x; i < n;
             i += static_cast<long long>(gridDim.x) * kThreads) {
            const int t = static_cast<int>(i / per_row), c = static_cast<int>(i - static_cast<long long>(t) * per_row);
            const int h = c / per_head, e = (c - h * per_head) * V, slot = p.slot[t];
            if (slot < 0) continue;
            if (slot >= p.n_slots) {
                raise_status(p.status, QS_DEV_PAGES);
                continue;
            }
            *reinterpret_cast<Vec*>(dst + place(slot, h, p.Hkv, p.d[x], p.page_shift) + e) =
                *reinterpret_cast<const Vec*>(src + t * p.row[x] + h * p.head[x] + e);
        }
    }
}

// e4m3: d / 8 lanes take a vector, 8 entries each.
template <int D, bool kAligned>
__global__ void __launch_bounds__(kThreads) kv_quant_kernel(const KvAppendParams p) {
    constexpr int kLanes = D / 8, kVecs = kThreads / kLanes;
    const int part = threadIdx.x % kLanes;
    const long long n = static_cast<long long>(p.T) * p.Hkv, per_pass = static_cast<long long>(gridDim.x) * kVecs;
    for (int x = 0; x < 2; ++x) {
        for (long long i0 = static_cast<long long>(blockIdx.x) * kVecs; i0 < n; i0 += per_pass) {
            // every lane of the warp stays for the shuffles
            const long long i = i0 + threadIdx.x / kLanes;
            int slot = -1, h = 0;
            float v[8] = {};
            if (i < n) {
                const int t = static_cast<int>(i / p.Hkv);
                h = static_cast<int>(i - static_cast<long long>(t) * p.Hkv);
                slot = p.slot[t];
                if (slot >= p.n_slots) {
                    raise_status(p.status, QS_DEV_PAGES);
                    slot = -1;
                }
                if (slot >= 0) {
                    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.src[x]) + t * p.row[x] +
                                               h * p.head[x] + part * 8;
                    if (kAligned) {
                        const uint4 u = *reinterpret_cast<const uint4*>(src);
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            v[2 * j] = __uint_as_float(w[j] << 16);
                            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = __bfloat162float(src[j]);
                    }
                }
            }
            // |x| as integers order as the numbers do, NaN and infinity on top
            unsigned top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
            // max|x| = m 2^e, 1 <= m < 2: k = e - 8 where m <= 1.75 = 448 / 2^8, else e - 7
            const bool fine = top < 0x7f800000u;
            int k = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
            k = top == 0 ? 0 : max(k, -126);
            const float inv = __uint_as_float(static_cast<unsigned>(127 - k) << 23);
            if (slot < 0) continue;
            uint32_t out[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t w = 0;
#pragma unroll
                for (int m = 0; m < 4; m += 2) {
                    const float2 y = make_float2(v[4 * j + m] * inv, v[4 * j + m + 1] * inv);
                    w |= static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3)) << (8 * m);
                }
                out[j] = fine ? w : 0u;
            }
            const size_t at = place(slot, h, p.Hkv, 1, p.page_shift);
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.dst[x]) + at * D + part * 8) = make_uint2(out[0], out[1]);
            if (part == 0) p.exps[x][at] = fine ? static_cast<uint8_t>(k + 127) : 255;
        }
    }
}

template <int D>
void launch_quant(bool aligned, int grid, const KvAppendParams& p, cudaStream_t stream) {
    if (aligned)
        kv_quant_kernel<D, true><<<grid, kThreads, 0, stream>>>(p);
    else
        kv_quant_kernel<D, false><<<grid, kThreads, 0, stream>>>(p);
}

}  // namespace

cudaError_t launch_kv_append(const qstate_kv_cfg& c, const KvAppendParams& p, cudaStream_t stream) {
    bool aligned = true;   // every vector of 8 entries starts on 16 bytes
    for (int x = 0; x < p.tensors; ++x)
        aligned = aligned && reinterpret_cast<uintptr_t>(p.src[x]) % 16 == 0 && p.row[x] % 8 == 0 &&
                  (p.head[x] % 8 == 0 || p.Hkv == 1);
    const long long threads = static_cast<long long>(p.T) * p.Hkv * (p.d[0] / 8);
    const long long most = 8LL * device_sm_count();
    const int grid = static_cast<int>(std::min(most, (threads + kThreads - 1) / kThreads));
    if (c.store == QSTATE_KV_E4M3) {
        if (p.d[0] == 64) launch_quant<64>(aligned, grid, p, stream);
        else if (p.d[0] == 128) launch_quant<128>(aligned, grid, p, stream);
        else launch_quant<256>(aligned, grid, p, stream);
    } else if (aligned) {
        kv_copy_kernel<8><<<grid, kThreads, 0, stream>>>(p);
    } else {
        kv_copy_kernel<1><<<grid, kThreads, 0, stream>>>(p);
    }
    return cudaGetLastError();
}

}  // namespace qs
