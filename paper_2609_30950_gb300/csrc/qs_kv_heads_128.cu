// qs_kv_heads_128.cu -- attention over pages of keys and values of 128 entries.
#include "qs_kv_heads.cuh"

namespace qs {

cudaError_t launch_kv_heads_128(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream) {
    // Codes take more instructions a byte: three CTAs an SM for them, two tiles each (159 us with two of three at
    // 0.81 GB, 147 so); in 16 bits it makes no difference (0.61 GB: 108 and 109 us).
    constexpr int kStages = 3, kCtas = 2;
    if (c.store == QSTATE_KV_E4M3) return kv::launch_heads_of<128, false, true, 2, 3>(p, stream);
    return c.dtype == QSTATE_KV_F16 ? kv::launch_heads_of<128, true, false, kStages, kCtas>(p, stream)
                                    : kv::launch_heads_of<128, false, false, kStages, kCtas>(p, stream);
}

}  // namespace qs
