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
    // ---- requests that share their first tokens; null and unused without ----
    const int4* shared;      // of each request: tokens that it leaves to its group, the group's first block, blocks of a
                             // key head, the request's first row
    const int* groups;       // the groups (KvGroup)
    float* store;            // unsplit rows of a request's own tokens: sums, and references and weights
    float4* store_ml;
    int2* dir;               // of each row of work: the worker that begins it (-1: unsplit, in the store; -2: done), its parts
    float* pre_part;         // the same of the groups' blocks of rows
    float4* pre_ml;
    float* pre_store;
    float4* pre_store_ml;
    int2* pre_dir;
};

// Tokens of a tile, and rows (requests' heads) of a block, in the attention over tokens that requests share.
constexpr int kSharedTile = 64;
constexpr int kv_shared_rows(int d) { return d == 256 ? 128 : 256; }
constexpr int kSharedWeight = 3, kSharedHalfWeight = 2;   // units of a tile; of a block with one half (see SharedPart)
constexpr int kSharedRowUnits = 4;   // tiles that a block of rows costs by itself: its queries, its end
// What the launches and joins of shared tokens cost beside their tiles.  With 16-bit keys and values of 128 entries, sharing took and
// reading by oneself took: 4 requests of 8 key heads behind 3001 tokens 19.8 and 14.7 us, 16 x 12 behind 100 34.5 and 23.6, 38 x 3 of 3
// key heads behind 200 to 600 21.5 and 18.0; 35 x 7 of 7 key heads behind 50 to 370 34.7 and 39.7, 4 x 32 behind up to 2000 48.7 and 72.2.
constexpr long long kSharedLeastNs = 12000;

// What qstate_kv_group leaves behind: a head, the requests' records, the groups that share anything.  The head says what they
// were made for (groups_made_for in qs_kv_tiles.cuh).
struct KvGroupHead {
    int groups;              // that share
    int R, Hq, Hkv;
    int d, e4m3, window;
    int tokens;              // the most that one of them has in common
    long long units;         // of all blocks
};
struct KvGroup {
    int first, rows;         // its first request; requests times query heads of a key head
    int owner, tokens;       // the request whose pages are read, how many tokens
    int blocks, block0;      // blocks of rows of a key head; index of its first block
    long long unit0;         // units of the groups before it
};
constexpr int kKvGroupHeadBytes = 256;
static_assert(sizeof(KvGroupHead) == 40 && sizeof(KvGroupHead) <= kKvGroupHeadBytes && sizeof(KvGroup) == 32, "layout");
inline int kv_most_groups(int R) { return R / 2 + 1; }
// Blocks of rows of at most R / 2 groups over R requests.
inline long long kv_most_blocks(const qstate_kv_cfg& c, int R) {
    return c.Hkv * (static_cast<long long>(R) * (c.Hq / c.Hkv) / kv_shared_rows(c.dk) + kv_most_groups(R));
}

struct KvGroupParams {
    const int32_t* lens;
    const int32_t* start;
    const int32_t* common;
    int N, R, G, Hkv, tile, rows, window;
    long long most;          // tokens of a table's row
    // What a tile of shared tokens of one key head takes, in ns of the whole GPU: for each request that reads it by itself, and
    // for each half of a block of rows (e4m3: for each block).
    float alone_ns, block_ns;
    int half_rows;           // of what block_ns is for
    int light_rows;          // a block of up to so many has kSharedHalfWeight
    long long least_ns;      // that sharing has to gain, over all groups and key heads; 0: whatever it costs
    KvGroupHead head;        // host: what the head is to say, but for sums
    KvGroupHead* out;
    int4* shared;
    KvGroup* groups;
    int* status;
};

struct KvForkParams {
    qstate_kv_pages pages;
    qstate_kv_moves moves;
    int32_t* others;
    const int32_t* parent;
    const int32_t* keep;
    uint8_t* ok;
    int R, page_shift, n_pages, max_pages;
    int parts, chunk;        // of a request's columns: warps that share them, columns of each
    int* head;               // work space: entries of the list below the pages that come back
    int4* rec;
    int* count;              // pages of a part that come back; from kKvMaxRequests on, those of a CTA's parts
    int* owner;              // of each page: the last request that held it, plus 1; zeros between calls
    int* stage;              // the new rows
    int* status;
};

constexpr int kCompactSpan = 8192;   // pages that a CTA ranks at a time
struct KvCompactParams {
    qstate_kv_pages pages;
    qstate_kv_moves moves;
    int32_t* others;
    int32_t* table_out;
    int32_t* left;
    int R, limit, page_shift, n_pages, max_pages;
    int parts, chunk;
    int words;               // set by launch_kv_compact: words of bits that a thread ranks, one after another
    int* head;               // work space: pages that move
    uint32_t* used;          // a bit for each page; zeros between calls
    int2* spans;
    int* rank;
    int* status;
};

struct KvCopyParams {
    const int32_t* src;
    const int32_t* dst;
    int n, n_pages, tensors;
    void* data[4];           // k, v and their exponents
    long long bytes[4];      // of a page
    int width[4];            // of a load
    int pieces[4], pieces_all;
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
cudaError_t launch_kv_shared_64(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_shared_128(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_shared_256(const qstate_kv_cfg& c, const KvAttendParams& p, cudaStream_t stream);
cudaError_t launch_kv_group(const KvGroupParams& p, cudaStream_t stream);
cudaError_t launch_kv_fork(const KvForkParams& p, cudaStream_t stream);
cudaError_t launch_kv_compact(KvCompactParams p, cudaStream_t stream);
cudaError_t launch_kv_copy(KvCopyParams p, cudaStream_t stream);
int kv_column_parts(int R, int max_pages);
// Columns of a part, and one behind the last of a part that begins with column c0 >= 0.  The widest tables have 2^31 - 1024: neither
// sum here is an int there.
constexpr int kv_part_columns(int max_pages, int parts) { return static_cast<int>((static_cast<long long>(max_pages) + parts - 1) / parts); }
__host__ __device__ constexpr int kv_part_end(int c0, int chunk) { return chunk > 0x7fffffff - c0 ? 0x7fffffff : c0 + chunk; }
static_assert(kv_part_columns(0x7ffffc00, kKvMaxRequests) == 1 << 18 && kv_part_end((kKvMaxRequests - 1) << 18, 1 << 18) == 0x7fffffff, "");
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
long long shared_least_ns();

}  // namespace qs
