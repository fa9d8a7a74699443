// qs_kv_shared_256.cu -- attention over pages that requests share, keys and values of 256 entries.
#include "qs_kv_shared.cuh"

namespace qs {

cudaError_t launch_kv_shared_256(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    return kv::launch_shared_of<256>(c, p, stream);
}

}  // namespace qs
