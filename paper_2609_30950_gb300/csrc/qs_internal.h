// qs_internal.h -- kernel parameter blocks and launch entry points inside libqstate.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/qstate.h"

namespace qs {

// device status bits
enum : int {
    QS_DEV_LAYOUT = 1,  // widths/offsets inconsistent with the region
    QS_DEV_RATE = 2,    // a decay rate is not a positive finite number
    QS_DEV_TIMEOUT = 4, // a tensor-core product did not signal completion in time
    QS_DEV_CHUNK = 8,   // chunked form: a row's decay over a 16-token block leaves FP32 range
    QS_DEV_TEARDOWN = 16,  // chunked form: after a timeout, the wait for the products still in
                           // flight before freeing tensor memory also gave up
    QS_DEV_PAGES = 32,  // paged cache: a page id, slot or length outside the pool or table
};

// Default limit of the chunked form's bounded mbarrier waits (polls of mbarrier.try_wait).
constexpr int kDefaultWaitPolls = 1 << 24;

constexpr int kNFit = 16;

// Parameters of the fused write-back kernel.  src/dst are packed or dense depending on the
// kernel instantiation.
struct StepParams {
    int B, H, T;
    int t_begin, t_end, w_index;
    int erase;        // 1: delta rule (a = beta k, w = beta 1); 0: a = 0, w = 1 (or general)
    int general;      // 1: a and w given per token (a_in, w_in)
    int mode;         // 0: full write-back; 1: statistics only (ranges, EMAs, readouts; no
                      // packing); 2: full write-back leaving the EMAs in memory unchanged
    int decay_row;    // 1: per-row rates; 0: per-head rates
    int fit_every;
    int L;            // 2^gate_bits (0 when rates are FP32)
    int group_heads;
    long long region_bytes;
    int stage_bytes;  // shared-memory staging capacity for one head's rows (dk dv bmax / 8)
    float alpha;      // EMA weight 2 / (span + 1)
    int early;        // host: launch_chained's early
    int wait_polls;   // limit of the chunked form's waits for its tensor-core products (>= 0)
    // packed source / destination
    const uint8_t* in_payload;
    const uint16_t* in_scales;
    const uint8_t* in_widths;
    const uint32_t* in_head_off;
    const uint8_t* in_fidx;
    uint8_t* out_payload;
    uint16_t* out_scales;
    const uint8_t* out_widths;
    const uint32_t* out_head_off;
    uint8_t* out_fidx;
    // dense source / destination (B, H, dk, dv); src may be null (= zero state)
    const float* dense_in;
    float* dense_out;
    // token inputs
    const float* q;
    const float* k;
    const float* v;
    const float* s;
    const uint8_t* s_code;
    const float* s_lut;
    const float* beta;
    const float* a_in;
    const float* w_in;
    float* o;
    // statistics (may be null when there are no tokens)
    float* ema_s;
    float* ema_r;
    float* range;
    int* status;
};

struct AllocParams {
    int B, H, dk, dv, units, unit_row, group_heads, bmin, bmax;
    long long total;   // sum of widths per batch element
    int uniform;       // 1: ignore statistics, equal weights (initial widths)
    int weight_kind;   // QSTATE_WEIGHT_*
    int C;             // write-back period (write-back factor weight)
    int early;         // host: launch_chained's early
    int shuf_a, shuf_b;   // shuffled-decay bijection u -> (shuf_a u + shuf_b) mod units
    int ngroups, gshift, above_min;   // set by launch_alloc: normalisation groups, log2 of their
                                      // size (-1: no power of two), total - units bmin
    int vec;                          // set by launch_alloc: arrays aligned for 16-byte loads
    const float* ema_s;
    const float* ema_r;
    const float* range;
    uint8_t* widths;
    uint32_t* head_off;
    int* status;
    float e1[17];      // 1/k! (FP64 -> FP32) for the expm1 series, k = 1..16
};

// Launch of a kernel that begins with chain_wait() or its halves.  early: its CTAs may be placed, and run up
// to that point, while the launch before it in the stream still runs: the launch's latency and the kernel's
// start are then behind it (256 write-backs and allocations of one 64 x 64 head: 12.4 -> 9.6 us
// each; one-prompt prefill 811 -> 730 us).  The chains of a partitioned scan launch without it:
// CTAs that wait in one chain would hold SMs that another chain's work fills (KDA prefill, 2 chains:
// 1243 us with it, 1226 us without; KDA decode, 4 chains: 1442 against 1440 us).
// The paged cache's kernels all launch with it, so what the one before wrote (lengths, tables, slots) is read by
// ordinary loads (a step of a plan, 12 appends and 12 attentions for 4 requests of 100 tokens, in a graph:
// 86 us without, 76 with).
template <class... P, class... A>
cudaError_t launch_chained(void (*kern)(P...), int grid, int threads, size_t smem, cudaStream_t stream, bool early,
                           A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

// launchers (return cudaError_t of the launch)
cudaError_t launch_scan_fp32(int dk, int dv, const StepParams& p, cudaStream_t stream);
cudaError_t launch_alloc(const AllocParams& p, cudaStream_t stream);
cudaError_t launch_quant_decay(const float* s, long long count, int nchan, int g,
                               uint8_t* codes, float* lut, float* thr, int* status,
                               cudaStream_t stream);
long long quant_decay_scratch_capacity();
cudaError_t quant_decay_scratch(float** out);
// ---- paged cache of attention layers (qs_kv_*.cu) ---------------------------------------------
// Head of the work space: int32 counters, all zero between calls.
constexpr int kKvTicket = 0;          // qstate_kv_plan in place: CTAs that have read the old lengths
constexpr int kKvSms = 152;           // SMs that an attention launch takes at most
constexpr int kKvWorkers = 4 * kKvSms;  // and its CTAs
constexpr int kKvHeadBytes = 4096;
constexpr int kKvMaxRequests = 8192;

struct KvPlanParams {
    qstate_kv_pages pages;
    qstate_kv_slots slots;
    const int32_t* n_new;
    int R, page_shift, n_pages, max_pages;
    int in_place;      // lens_out or free_out is the array that is read
    int aligned;       // slot, pos and req can be written in 16 bytes
    int* ticket;
    int* status;
};

struct KvAppendParams {
    const void* src[2];            // k, v
    long long row[2], head[2];     // strides in elements
    void* dst[2];
    uint8_t* exps[2];
    const int32_t* slot;
    int T, Hkv, d[2], page_shift, tensors;
    long long n_slots;
    int* status;
};

struct KvAttendParams {
    const void* q;
    long long q_row, q_head;
    const void* k;
    const void* v;
    const uint8_t* k_exp;
    const uint8_t* v_exp;
    const int32_t* table;
    const int32_t* lens;
    void* o;
    float* lse;
    int R, Hq, Hkv, dk, dv, page_shift, n_pages, max_pages, window;
    float scale;
    float* part;     // partial results: sums, then references and weights
    float* part_ml;
    int* split;      // parts of the row that a worker begins (0: not split), and the row
    int workers;     // how many share the work out
    int whole_rows;  // by rows instead of tiles: no row is split
    int q_aligned;   // q can be read in 16 bytes
    int wait_polls;  // limit of the latent kernel's waits for copies and products
    int* status;
};

cudaError_t launch_kv_plan(const KvPlanParams& p, cudaStream_t stream);
cudaError_t launch_kv_append(const qstate_kv_cfg& c, const KvAppendParams& p, cudaStream_t stream);
cudaError_t launch_kv_attend(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_latent_128(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_latent_256(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_latent_512(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_heads_64(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_heads_128(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_heads_256(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
// partial results that an attention launch may use: bytes of sums, of references and weights, of the list of
// split rows
struct KvPartBytes {
    size_t sums, ml, split;
};
KvPartBytes kv_part_bytes(const qstate_kv_cfg& c);

// the calling thread's error text and the device status word (qs_api.cu)
int fail(int code, const char* fmt, ...);
int cuda_fail(cudaError_t e, const char* what);
int acquire_status(int** out);
int wait_polls();
// identity of the current CUDA context (false if unknown); see qs_api.cu
bool current_context_id(unsigned long long* id);
// streaming multiprocessors of the current device (cached per device)
int device_sm_count();

}  // namespace qs
