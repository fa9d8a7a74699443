// qs_kv_attend.cu -- attention over the paged cache: which kernel, and what it needs of the work space.
#include <mutex>

#include "qs_kv_latent.cuh"

namespace qs {
namespace kv {

// The driver's call comes through the runtime: the library does not link the driver library.
bool pool_map(CUtensorMap* map, const void* pool, int dk, long long rows) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Encode encode = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            encode = reinterpret_cast<Encode>(f);
    });
    if (!encode) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(dk), static_cast<cuuint64_t>(rows)}, strides[1] = {2ull * dk};
    const cuuint32_t shape[2] = {64, kLatTile}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(pool), dims, strides, shape, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace kv

// Two slots a worker.  Heads: 16 rows; latents: the groups' columns (workers x groups CTAs are at most
// two an SM).
KvPartBytes kv_part_bytes(const qstate_kv_cfg& c) {
    constexpr size_t split = kKvWorkers * 2 * sizeof(int);
    if (c.kind == QSTATE_KV_HEADS)
        return {static_cast<size_t>(kKvWorkers) * 2 * 16 * c.dv * sizeof(float),
                static_cast<size_t>(kKvWorkers) * 2 * 16 * 16, split};
    const kv::LatentGeo g = kv::latent_geo(c.Hq, c.dk, c.dv, kKvSms);
    const size_t rows = static_cast<size_t>(g.workers) * g.groups * 2 * g.columns;
    return {rows * c.dv * sizeof(float), rows * 16, split};
}

cudaError_t launch_kv_attend(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    if (c.kind == QSTATE_KV_HEADS)
        return c.dk == 64 ? launch_kv_heads_64(c, p, stream)
                          : c.dk == 128 ? launch_kv_heads_128(c, p, stream) : launch_kv_heads_256(c, p, stream);
    return c.dv == 128 ? launch_kv_latent_128(c, p, stream)
                       : c.dv == 256 ? launch_kv_latent_256(c, p, stream) : launch_kv_latent_512(c, p, stream);
}

}  // namespace qs
