// qs_kv_latent_256.cu -- attention over pages of latents whose first 256 entries are the values.
#include "qs_kv_latent.cuh"

namespace qs {

cudaError_t launch_kv_latent_256(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    return kv::launch_latent_of<256>(c, p, stream);
}

}  // namespace qs
