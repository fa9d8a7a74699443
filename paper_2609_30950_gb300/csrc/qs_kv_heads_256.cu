// qs_kv_heads_256.cu -- attention over pages of keys and values of 256 entries.
#include "qs_kv_heads.cuh"

namespace qs {

cudaError_t launch_kv_heads_256(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    constexpr int kStages = 3, kCtas = 1;
    if (c.store == QSTATE_KV_E4M3) return kv::launch_heads_of<256, false, true, kStages, kCtas>(p, stream);
    return c.dtype == QSTATE_KV_F16 ? kv::launch_heads_of<256, true, false, kStages, kCtas>(p, stream)
                                    : kv::launch_heads_of<256, false, false, kStages, kCtas>(p, stream);
}

}  // namespace qs
