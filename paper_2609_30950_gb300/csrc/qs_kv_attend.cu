// qs_kv_attend.cu -- attention over the paged cache: which kernel, and what it needs of the work space.
#include "qs_kv_latent.cuh"

namespace qs {

// Two slots a worker.  Heads: 16 rows; latents: the groups' columns (workers x groups CTAs are at most
// two an SM).
KvPartBytes kv_part_bytes(const qstate_kv_cfg& c) {
    constexpr size_t split = kKvWorkers * 2 * sizeof(int);
    if (c.kind == QSTATE_KV_HEADS)
        return {static_cast<size_t>(kKvWorkers) * 2 * 16 * c.dv * sizeof(float),
                static_cast<size_t>(kKvWorkers) * 2 * 16 * 16, split};
    const kv::LatentGeo g = kv::latent_geo(c.Hq, c.dk, kKvSms);
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
