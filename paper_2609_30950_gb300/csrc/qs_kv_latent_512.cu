// qs_kv_latent_512.cu -- attention over pages of latents whose first 512 entries are the values.
#include "qs_kv_latent.cuh"

namespace qs {

cudaError_t launch_kv_latent_512(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    return kv::launch_latent_of<512>(c, p, stream);
}

}  // namespace qs
