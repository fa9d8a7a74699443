// qs_kv_attend.cu -- one new token of each request against its pages.
//
// The plain kernel: a CTA for each request and query head, its warps take tokens in turn, a lane
// holds every 32nd entry; running maximum and sum of the softmax per warp, joined at the end.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <cmath>

#include "qs_common.cuh"

namespace qs {
namespace {

constexpr int kWarps = 8;
constexpr int kMaxPer = 18;   // entries a lane holds: 576 / 32

__device__ __forceinline__ float load16(const void* p, size_t i, bool f16) {
    return f16 ? __half2float(static_cast<const __half*>(p)[i]) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

__device__ __forceinline__ float load8(const void* p, size_t i) {
    __nv_fp8_e4m3 x;
    x.__x = static_cast<const uint8_t*>(p)[i];
    return static_cast<float>(x);
}

__device__ __forceinline__ float power_of(int e) { return e == 255 ? __uint_as_float(0x7fffffffu) : __uint_as_float(e << 23); }

__global__ void __launch_bounds__(kWarps * 32) kv_attend_plain_kernel(const KvAttendParams p, int f16, int e4m3) {
    __shared__ float s_m[kWarps], s_l[kWarps], s_o[kWarps][512];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = blockIdx.x / p.Hq, hq = blockIdx.x - r * p.Hq, hk = hq / (p.Hq / p.Hkv);
    long long n = p.lens[r];
    const long long most = static_cast<long long>(p.max_pages) << p.page_shift;
    if (n < 0 || n > most) {
        raise_status(p.status, QS_DEV_PAGES);
        n = n < 0 ? 0 : most;
    }
    const int end = static_cast<int>(n), begin = p.window ? max(0, end - p.window) : 0;
    float q[kMaxPer], o[kMaxPer] = {}, m = -INFINITY, l = 0.0f;
    for (int i = 0; i < kMaxPer; ++i)
        q[i] = i * 32 < p.dk ? load16(p.q, r * p.q_row + hq * p.q_head + i * 32 + lane, f16) * p.scale : 0.0f;
    for (int t = begin + warp; t < end; t += kWarps) {
        const int id = p.table[static_cast<size_t>(r) * p.max_pages + (t >> p.page_shift)];
        if (id < 0 || id >= p.n_pages) {
            raise_status(p.status, QS_DEV_PAGES);
            continue;
        }
        const size_t at = ((static_cast<size_t>(id) * p.Hkv + hk) << p.page_shift) + (t & ((1 << p.page_shift) - 1));
        float z = 0.0f;
        for (int i = 0; i < kMaxPer; ++i)
            if (i * 32 < p.dk) {
                const size_t e = at * p.dk + i * 32 + lane;
                z += q[i] * (e4m3 ? load8(p.k, e) : load16(p.k, e, f16));
            }
        z = warp_sum(z);
        if (e4m3) z *= power_of(p.k_exp[at]);
        const float vs = e4m3 ? power_of(p.v_exp[at]) : 1.0f;
        const float top = fmaxf(m, z), c = expf(m - top), w = expf(z - top);
        const size_t vrow = p.v == p.k ? at * p.dk : at * p.dv;
        l = l * c + w;
        m = top;
        for (int i = 0; i < kMaxPer; ++i)
            if (i * 32 < p.dv) {
                const size_t e = vrow + i * 32 + lane;
                o[i] = o[i] * c + w * ((e4m3 ? load8(p.v, e) : load16(p.v, e, f16)) * vs);
            }
    }
    if (lane == 0) s_m[warp] = m, s_l[warp] = l;
    for (int i = 0; i < kMaxPer; ++i)
        if (i * 32 < p.dv) s_o[warp][i * 32 + lane] = o[i];
    __syncthreads();
    float M = -INFINITY, L = 0.0f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w]);
    for (int w = 0; w < kWarps; ++w)
        if (s_l[w] != 0.0f) L += s_l[w] * expf(s_m[w] - M);
    const size_t row = static_cast<size_t>(r) * p.Hq + hq;
    for (int i = threadIdx.x; i < p.dv; i += kWarps * 32) {
        float x = 0.0f;
        for (int w = 0; w < kWarps; ++w)
            if (s_l[w] != 0.0f) x += s_o[w][i] * expf(s_m[w] - M);
        if (L != 0.0f) x /= L;
        if (f16)
            static_cast<__half*>(p.o)[row * p.dv + i] = __float2half_rn(x);
        else
            static_cast<__nv_bfloat16*>(p.o)[row * p.dv + i] = __float2bfloat16_rn(x);
    }
    if (p.lse && threadIdx.x == 0) p.lse[row] = L != 0.0f ? M + logf(L) : -INFINITY;
}

}  // namespace

KvPartBytes kv_part_bytes(const qstate_kv_cfg& c) {
    if (c.kind == QSTATE_KV_LATENT) return {0, 0};
    return {static_cast<size_t>(kKvWorkers) * 2 * 16 * c.dv * sizeof(float), static_cast<size_t>(kKvWorkers) * 2 * 16 * 16};
}

cudaError_t launch_kv_attend(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    if (c.kind == QSTATE_KV_HEADS)
        return c.dk == 64 ? launch_kv_heads_64(c, p, stream)
                          : c.dk == 128 ? launch_kv_heads_128(c, p, stream) : launch_kv_heads_256(c, p, stream);
    kv_attend_plain_kernel<<<p.R * p.Hq, kWarps * 32, 0, stream>>>(p, c.dtype == QSTATE_KV_F16,
                                                                  c.store == QSTATE_KV_E4M3);
    return cudaGetLastError();
}

}  // namespace qs
