// qs_kv_copy.cu -- pages of one layer's cache copied to other places of the pool.
//
// Each page is one run of Hkv page d entries of each tensor (and Hkv page exponent bytes), read and written once: memory bounds
// it (2501 pages, 330 MB read and written in 52.6 us, 94 % of the copy rate), and for the few pages of a fork the launch does
// (36 pages of 16 KB: 3.1 us).  A CTA copies a piece of kPiece bytes of one page of one tensor, all of its loads in
// flight before the first store.
#include "qs_common.cuh"
#include "qs_kv.h"

namespace qs {
namespace {

constexpr int kThreads = 256, kLoads = 4;

// Pieces of page i, tensor after tensor; a piece is kThreads kLoads vectors.
template <class Vec>
__device__ __forceinline__ void copy_piece(const KvCopyParams& p, int tensor, int src, int dst, long long first) {
    const long long vectors = p.bytes[tensor] / static_cast<long long>(sizeof(Vec));
    const Vec* const from = reinterpret_cast<const Vec*>(static_cast<const char*>(p.data[tensor]) + src * p.bytes[tensor]);
    Vec* const to = reinterpret_cast<Vec*>(static_cast<char*>(p.data[tensor]) + dst * p.bytes[tensor]);
    Vec x[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const long long v = first + k * kThreads + threadIdx.x;
        if (v < vectors) x[k] = __ldcg(from + v);
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const long long v = first + k * kThreads + threadIdx.x;
        if (v < vectors) to[v] = x[k];
    }
}

__global__ void __launch_bounds__(kThreads) kv_copy_pages_kernel(const KvCopyParams p) {
    chain_wait();
    const long long items = static_cast<long long>(p.n) * p.pieces_all;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int i = static_cast<int>(item / p.pieces_all);
        int piece = static_cast<int>(item - static_cast<long long>(i) * p.pieces_all);
        const int src = __ldcg(p.src + i), dst = __ldcg(p.dst + i);
        if (src < 0 || dst < 0) continue;
        if (src >= p.n_pages || dst >= p.n_pages) {
            if (threadIdx.x == 0) raise_status(p.status, QS_DEV_PAGES);
            continue;
        }
        int tensor = 0;
        while (piece >= p.pieces[tensor]) piece -= p.pieces[tensor++];
        const long long first = static_cast<long long>(piece) * (kThreads * kLoads);
        if (p.width[tensor] == 16)
            copy_piece<uint4>(p, tensor, src, dst, first);
        else if (p.width[tensor] == 4)
            copy_piece<uint32_t>(p, tensor, src, dst, first);
        else
            copy_piece<uint8_t>(p, tensor, src, dst, first);
    }
}

}  // namespace

cudaError_t launch_kv_copy(KvCopyParams p, cudaStream_t stream) {
    p.pieces_all = 0;
    for (int t = 0; t < p.tensors; ++t) {
        const long long vectors = p.bytes[t] / p.width[t];
        p.pieces[t] = static_cast<int>((vectors + kThreads * kLoads - 1) / (kThreads * kLoads));
        p.pieces_all += p.pieces[t];
    }
    const long long items = static_cast<long long>(p.n) * p.pieces_all, most = 1LL << 30;
    return launch_chained(kv_copy_pages_kernel, static_cast<int>(items < most ? items : most), kThreads, 0, stream, true, p);
}

}  // namespace qs
