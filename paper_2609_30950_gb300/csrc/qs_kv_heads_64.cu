// qs_kv_heads_64.cu -- attention over pages of keys and values of 64 entries.
#include "qs_kv_heads.cuh"

namespace qs {

cudaError_t launch_kv_heads_64(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    constexpr int kStages = 4, kCtas = 3;
    if (c.store == QSTATE_KV_E4M3) return kv::launch_heads_of<64, false, true, kStages, kCtas>(p, stream);
    return c.dtype == QSTATE_KV_F16 ? kv::launch_heads_of<64, true, false, kStages, kCtas>(p, stream)
                                    : kv::launch_heads_of<64, false, false, kStages, kCtas>(p, stream);
}

}  // namespace qs
