// qs_kv.h -- what the files of the paged cache (qs_kv_*.cu) share: parameters of its kernels, their launches.
#pragma once

#include "qs_internal.h"

namespace qs {

// A condition of the device status word beside those of the recurrence: a page id, slot or length outside the
// pool or the table.
constexpr int QS_DEV_PAGES = 32;

// The cache's kernels all launch early (launch_chained), so what the one before wrote (lengths, tables, slots) is read
// by ordinary loads (a step of a plan, 12 appends and 12 attentions for 4 requests of 100 tokens, in a graph:
// 86 us without, 76 with).

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

}  // namespace qs
