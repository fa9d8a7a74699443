// qs_kv_latent_128.cu -- attention over pages of latents whose first 128 entries are the values.
#include "qs_kv_latent.cuh"

namespace qs {

cudaError_t launch_kv_latent_128(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    return kv::launch_latent_of<128>(c, p, stream);
}

}  // namespace qs
