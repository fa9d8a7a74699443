// qs_kv_api.cu -- C entries of the paged cache of attention layers: checks and dispatch.
#include <atomic>
#include <cmath>
#include <cstring>

#include "qs_kv.h"

using namespace qs;

namespace {

// qstate_set_shared_gain
std::atomic<long long> g_least_ns{kSharedLeastNs};

int check_pool(const qstate_kv_cfg* c) {
    if (!c) return fail(QSTATE_EINVAL, "cfg is NULL");
    if (c->page < 1 || c->page > 1024 || (c->page & (c->page - 1)) != 0)
        return fail(QSTATE_EINVAL, "page must be a power of two in [1, 1024], got %d", c->page);
    if (c->n_pages < 1 || static_cast<long long>(c->n_pages) * c->page > 0x7fffffffLL)
        return fail(QSTATE_EINVAL, "need n_pages >= 1 and n_pages * page < 2^31");
    // the last tile of a request's tokens ends within 32 bits
    if (c->max_pages < 1 || static_cast<long long>(c->max_pages) * c->page > 0x80000000LL - 1024)
        return fail(QSTATE_EINVAL, "need max_pages >= 1 and max_pages * page <= 2^31 - 1024");
    return QSTATE_OK;
}

int check_cfg(const qstate_kv_cfg* c) {
    if (const int rc = check_pool(c)) return rc;
    if (c->kind != QSTATE_KV_HEADS && c->kind != QSTATE_KV_LATENT) return fail(QSTATE_EINVAL, "bad kind %d", c->kind);
    if (c->Hq < 1 || c->Hq > 1024 || c->Hkv < 1 || c->Hq % c->Hkv != 0)
        return fail(QSTATE_EINVAL, "need 1 <= Hq <= 1024 and Hkv dividing Hq");
    if (c->dtype != QSTATE_KV_BF16 && c->dtype != QSTATE_KV_F16) return fail(QSTATE_EINVAL, "bad dtype %d", c->dtype);
    if (c->store != QSTATE_KV_16 && c->store != QSTATE_KV_E4M3) return fail(QSTATE_EINVAL, "bad store %d", c->store);
    if (c->window < 0) return fail(QSTATE_EINVAL, "window must be >= 0");
    if (!std::isfinite(c->scale)) return fail(QSTATE_EINVAL, "scale is not finite");
    if (c->kind == QSTATE_KV_HEADS) {
        if (c->dk != c->dv || (c->dk != 64 && c->dk != 128 && c->dk != 256))
            return fail(QSTATE_EINVAL, "unsupported (dk, dv) = (%d, %d)", c->dk, c->dv);
        if (c->store == QSTATE_KV_E4M3 && c->dtype != QSTATE_KV_BF16)
            return fail(QSTATE_EINVAL, "an e4m3 cache needs bf16 queries");
    } else {
        const int rope = c->dk - c->dv;
        if (c->Hkv != 1) return fail(QSTATE_EINVAL, "latent attention has Hkv = 1");
        if ((c->dv != 128 && c->dv != 256 && c->dv != 512) || (rope != 0 && rope != 32 && rope != 64))
            return fail(QSTATE_EINVAL, "unsupported latent (dk, dv) = (%d, %d)", c->dk, c->dv);
        if (c->store != QSTATE_KV_16) return fail(QSTATE_EINVAL, "latents are stored in 16 bits");
    }
    return QSTATE_OK;
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Arrays of 32-bit entries; NULL counts as aligned.
template <class... P>
bool words(const P*... p) { return (aligned(p, 4) && ...); }

int check_cache(const qstate_kv_cfg* c, const qstate_kv_cache* cache) {
    const bool heads = c->kind == QSTATE_KV_HEADS, e4m3 = c->store == QSTATE_KV_E4M3;
    if (!cache || !cache->k || (heads && !cache->v)) return fail(QSTATE_EINVAL, "null cache pointer");
    if (!heads && cache->v) return fail(QSTATE_EINVAL, "latent attention has no separate values");
    if (e4m3 != (cache->k_exp != nullptr) || e4m3 != (cache->v_exp != nullptr))
        return fail(QSTATE_EINVAL, "exponents belong to an e4m3 cache, and only to one");
    if (!aligned(cache->k, 16) || !aligned(cache->v, 16))
        return fail(QSTATE_EINVAL, "the cache must be 16-byte aligned");
    if (!aligned(cache->k_exp, 4) || !aligned(cache->v_exp, 4))
        return fail(QSTATE_EINVAL, "exponents must be 4-byte aligned");
    return QSTATE_OK;
}

int shift_of(int page) {
    int s = 0;
    while ((1 << s) < page) ++s;
    return s;
}

// Work space of calls on pages.  What has to be zero between calls lies where R does not matter.
struct PagesWork {
    size_t owner, used, spans, rank, count, rec, stage, all;
};
size_t whole(size_t n) { return (n + 255) / 256 * 256; }
PagesWork pages_work(const qstate_kv_cfg& c, int R) {
    const size_t n = static_cast<size_t>(c.n_pages), r = static_cast<size_t>(R);
    PagesWork w;
    w.owner = kKvHeadBytes;
    w.used = w.owner + whole(n * sizeof(int));
    w.spans = w.used + whole((n / 32 + 1) * sizeof(uint32_t));
    w.rank = w.spans + whole((n / kCompactSpan + 1) * sizeof(int2));
    w.count = w.rank + whole(n * sizeof(int));
    w.rec = w.count + whole(2 * kKvMaxRequests * sizeof(int));   // of parts, of CTAs
    w.stage = w.rec + whole(r * sizeof(int4));
    w.all = w.stage + whole(r * static_cast<size_t>(c.max_pages) * sizeof(int));
    return w;
}

// And of the attention over shared tokens, behind what qstate_kv_attend uses.
struct SharedWork {
    size_t store, store_ml, dir, part, part_ml, pre_store, pre_store_ml, pre_dir, all;
};
SharedWork shared_work(const qstate_kv_cfg& c, int R) {
    const KvPartBytes b = kv_part_bytes(c);
    const size_t rows = static_cast<size_t>(R) * c.Hq, d = c.dv, slots = 2 * kKvSms * static_cast<size_t>(kv_shared_rows(c.dk));
    SharedWork w;
    w.store = whole(kKvHeadBytes + b.sums + b.ml + b.split);
    w.store_ml = w.store + whole(rows * d * sizeof(float));
    w.dir = w.store_ml + whole(rows * sizeof(float4));
    w.part = w.dir + whole(rows * sizeof(int2));
    w.part_ml = w.part + slots * d * sizeof(float);
    w.pre_store = w.part_ml + slots * sizeof(float4);
    w.pre_store_ml = w.pre_store + whole(2 * rows * d * sizeof(float));   // two streams
    w.pre_dir = w.pre_store_ml + whole(2 * rows * sizeof(float4));
    w.all = w.pre_dir + whole(static_cast<size_t>(kv_most_blocks(c, R)) * sizeof(int2));
    return w;
}

int check_requests(int32_t R) {
    return R < 0 || R > kKvMaxRequests ? fail(QSTATE_EINVAL, "need 0 <= R <= %d", kKvMaxRequests) : QSTATE_OK;
}

int check_shared(const qstate_kv_cfg* c) {
    if (const int rc = check_cfg(c)) return rc;
    return c->kind == QSTATE_KV_LATENT ? fail(QSTATE_EINVAL, "latents have no attention over shared tokens") : QSTATE_OK;
}

int check_moves(const qstate_kv_moves* m) {
    if (!m || m->n < 0 || (m->n > 0 && (!m->src || !m->dst))) return fail(QSTATE_EINVAL, "bad moves");
    return !words(m->src, m->dst) ? fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned") : QSTATE_OK;
}

// What both attentions are told.
void fill_attend(const qstate_kv_cfg* cfg, const qstate_kv_cache* cache, const void* q, int64_t q_row, int64_t q_head, const int32_t* table,
                 const int32_t* lens, int32_t R, void* o, float* lse, void* work, KvAttendParams* out) {
    KvAttendParams& p = *out;
    p.q = q;
    p.q_row = q_row;
    p.q_head = q_head;
    p.k = cache->k;
    p.v = cfg->kind == QSTATE_KV_HEADS ? cache->v : cache->k;
    p.k_exp = cache->k_exp;
    p.v_exp = cache->v_exp;
    p.table = table;
    p.lens = lens;
    p.o = o;
    p.lse = lse;
    p.R = R;
    p.Hq = cfg->Hq;
    p.Hkv = cfg->Hkv;
    p.dk = cfg->dk;
    p.dv = cfg->dv;
    p.page_shift = shift_of(cfg->page);
    p.n_pages = cfg->n_pages;
    p.max_pages = cfg->max_pages;
    p.window = cfg->window;
    p.scale = cfg->scale;
    p.part = reinterpret_cast<float*>(static_cast<char*>(work) + kKvHeadBytes);
    const KvPartBytes bytes = kv_part_bytes(*cfg);
    p.part_ml = p.part + bytes.sums / sizeof(float);
    p.split = reinterpret_cast<int*>(p.part_ml + bytes.ml / sizeof(float));
    p.wait_polls = wait_polls();
    p.q_aligned = aligned(q, 16) && q_row % 8 == 0 && q_head % 8 == 0;
}

int check_attend(const void* q, const int32_t* table, const int32_t* lens, const void* o, const float* lse, const void* work) {
    if (!q || !table || !lens || !o || !work) return fail(QSTATE_EINVAL, "null pointer");
    if (!aligned(q, 2)) return fail(QSTATE_EINVAL, "q must be 2-byte aligned");
    if (!words(table, lens, lse)) return fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned");
    if (!aligned(o, 16)) return fail(QSTATE_EINVAL, "o must be 16-byte aligned");
    if (!aligned(work, 256)) return fail(QSTATE_EINVAL, "the work space must be 256-byte aligned");
    return QSTATE_OK;
}

}  // namespace

long long qs::shared_least_ns() { return g_least_ns.load(); }

extern "C" {

int qstate_set_shared_gain(int32_t ns) {
    g_least_ns.store(ns < 0 ? kSharedLeastNs : ns);
    return QSTATE_OK;
}

int qstate_kv_validate(const qstate_kv_cfg* cfg) { return check_cfg(cfg); }

size_t qstate_kv_cache_bytes(const qstate_kv_cfg* cfg, int32_t v) {
    if (check_cfg(cfg)) return 0;
    if (v && cfg->kind == QSTATE_KV_LATENT) return 0;
    return static_cast<size_t>(cfg->n_pages) * cfg->page * cfg->Hkv * (v ? cfg->dv : cfg->dk) *
           (cfg->store == QSTATE_KV_E4M3 ? 1 : 2);
}

size_t qstate_kv_work_bytes(const qstate_kv_cfg* cfg) {
    if (cfg && !cfg->Hq && !cfg->Hkv && !cfg->dk && !cfg->dv) return check_pool(cfg) ? 0 : kKvHeadBytes;   // no layer: the plan's
    if (check_cfg(cfg)) return 0;
    const KvPartBytes b = kv_part_bytes(*cfg);
    return kKvHeadBytes + b.sums + b.ml + b.split;
}

int qstate_kv_plan(const qstate_kv_cfg* cfg, const qstate_kv_pages* pages, const int32_t* n_new, int32_t R,
                   const qstate_kv_slots* slots, void* work, void* stream) {
    int rc = check_pool(cfg);
    if (rc) return rc;
    if (!pages || !pages->free_list || !pages->free_count || !pages->free_out || !slots || !slots->cu || !work)
        return fail(QSTATE_EINVAL, "null pointer");
    if (R < 0 || R > kKvMaxRequests) return fail(QSTATE_EINVAL, "need 0 <= R <= %d", kKvMaxRequests);
    if (R > 0 && (!n_new || !pages->table || !pages->lens || !pages->lens_out || !slots->ok))
        return fail(QSTATE_EINVAL, "null pointer");
    if (slots->T < 0 || (slots->T > 0 && !slots->slot)) return fail(QSTATE_EINVAL, "bad rows");
    if (!words(pages->table, pages->lens, pages->lens_out, pages->free_list, pages->free_count, pages->free_out, n_new,
               slots->cu, slots->slot, slots->pos, slots->req))
        return fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned");
    if (!aligned(work, 256)) return fail(QSTATE_EINVAL, "the work space must be 256-byte aligned");
    KvPlanParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    p.pages = *pages;
    p.slots = *slots;
    p.n_new = n_new;
    p.R = R;
    p.page_shift = shift_of(cfg->page);
    p.n_pages = cfg->n_pages;
    p.max_pages = cfg->max_pages;
    p.in_place = pages->lens_out == pages->lens || pages->free_out == pages->free_count;
    p.aligned = aligned(slots->slot, 16) && aligned(slots->pos, 16) && aligned(slots->req, 16);
    p.ticket = static_cast<int*>(work) + kKvTicket;
    const cudaError_t e = launch_kv_plan(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "page plan kernel");
}

int qstate_kv_append(const qstate_kv_cfg* cfg, const qstate_kv_cache* cache, const void* k, int64_t k_row,
                     int64_t k_head, const void* v, int64_t v_row, int64_t v_head, const int32_t* slot, int32_t T,
                     void* stream) {
    int rc = check_cfg(cfg);
    if (rc || (rc = check_cache(cfg, cache))) return rc;
    const bool heads = cfg->kind == QSTATE_KV_HEADS;
    if (T < 0) return fail(QSTATE_EINVAL, "need T >= 0");
    if (T == 0) return QSTATE_OK;
    if (!heads && v) return fail(QSTATE_EINVAL, "latent attention has no separate values");
    if (!k || !slot || (heads && !v)) return fail(QSTATE_EINVAL, "null pointer");
    if (!words(slot)) return fail(QSTATE_EINVAL, "slots must be 4-byte aligned");
    if (!aligned(k, 2) || (heads && !aligned(v, 2))) return fail(QSTATE_EINVAL, "keys and values must be 2-byte aligned");
    KvAppendParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    p.src[0] = k;
    p.src[1] = v;
    p.row[0] = k_row;
    p.row[1] = v_row;
    p.head[0] = k_head;
    p.head[1] = v_head;
    p.dst[0] = cache->k;
    p.dst[1] = cache->v;
    p.exps[0] = cache->k_exp;
    p.exps[1] = cache->v_exp;
    p.slot = slot;
    p.T = T;
    p.Hkv = cfg->Hkv;
    p.d[0] = cfg->dk;
    p.d[1] = cfg->dv;
    p.page_shift = shift_of(cfg->page);
    p.tensors = heads ? 2 : 1;
    p.n_slots = static_cast<long long>(cfg->n_pages) * cfg->page;
    const cudaError_t e = launch_kv_append(*cfg, p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "cache append kernel");
}

int qstate_kv_attend(const qstate_kv_cfg* cfg, const qstate_kv_cache* cache, const void* q, int64_t q_row,
                     int64_t q_head, const int32_t* table, const int32_t* lens, int32_t R, void* o, float* lse,
                     void* work, void* stream) {
    int rc = check_cfg(cfg);
    if (rc || (rc = check_cache(cfg, cache)) || (rc = check_requests(R))) return rc;
    if (R == 0) return QSTATE_OK;
    if ((rc = check_attend(q, table, lens, o, lse, work))) return rc;
    KvAttendParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    fill_attend(cfg, cache, q, q_row, q_head, table, lens, R, o, lse, work, &p);
    const cudaError_t e = launch_kv_attend(*cfg, p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "cache attention kernel");
}

size_t qstate_kv_pages_work_bytes(const qstate_kv_cfg* cfg, int32_t R) {
    return check_pool(cfg) || check_requests(R) ? 0 : pages_work(*cfg, R).all;
}

size_t qstate_kv_group_bytes(const qstate_kv_cfg* cfg, int32_t R) {
    if (check_shared(cfg) || check_requests(R)) return 0;
    return kKvGroupHeadBytes + kv_most_groups(R) * sizeof(KvGroup) + static_cast<size_t>(R) * sizeof(int4);
}

size_t qstate_kv_shared_work_bytes(const qstate_kv_cfg* cfg, int32_t R) {
    return check_shared(cfg) || check_requests(R) ? 0 : shared_work(*cfg, R).all;
}

int qstate_kv_fork(const qstate_kv_cfg* cfg, const qstate_kv_pages* pages, int32_t* others, const int32_t* parent,
                   const int32_t* keep, int32_t R, const qstate_kv_moves* moves, uint8_t* ok, void* work, void* stream) {
    int rc = check_pool(cfg);
    if (rc || (rc = check_requests(R)) || (rc = check_moves(moves))) return rc;
    if (!pages || !pages->free_list || !pages->free_count || !pages->free_out || !work || !others) return fail(QSTATE_EINVAL, "null pointer");
    if (R > 0 && (!parent || !pages->table || !pages->lens || !pages->lens_out || !ok)) return fail(QSTATE_EINVAL, "null pointer");
    if (moves->n < R) return fail(QSTATE_EINVAL, "need an entry of moves for each request");
    if (!words(pages->table, pages->lens, pages->lens_out, pages->free_list, pages->free_count, pages->free_out, others, parent, keep))
        return fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned");
    if (!aligned(work, 256)) return fail(QSTATE_EINVAL, "the work space must be 256-byte aligned");
    KvForkParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    p.pages = *pages;
    p.moves = *moves;
    p.others = others;
    p.parent = parent;
    p.keep = keep;
    p.ok = ok;
    p.R = R;
    p.page_shift = shift_of(cfg->page);
    p.n_pages = cfg->n_pages;
    p.max_pages = cfg->max_pages;
    p.parts = kv_column_parts(R, cfg->max_pages);
    p.chunk = kv_part_columns(cfg->max_pages, p.parts);
    const PagesWork w = pages_work(*cfg, R);
    char* const base = static_cast<char*>(work);
    p.head = static_cast<int*>(work) + 1;
    p.rec = reinterpret_cast<int4*>(base + w.rec);
    p.count = reinterpret_cast<int*>(base + w.count);
    p.owner = reinterpret_cast<int*>(base + w.owner);
    p.stage = reinterpret_cast<int*>(base + w.stage);
    const cudaError_t e = launch_kv_fork(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "cache fork kernel");
}

int qstate_kv_compact(const qstate_kv_cfg* cfg, const qstate_kv_pages* pages, int32_t* others, int32_t R, int32_t limit,
                      const qstate_kv_moves* moves, int32_t* left, int32_t* table_out, void* work, void* stream) {
    int rc = check_pool(cfg);
    if (rc || (rc = check_requests(R)) || (rc = check_moves(moves))) return rc;
    if (limit < 1 || limit > cfg->n_pages) return fail(QSTATE_EINVAL, "need 1 <= limit <= n_pages");
    if (!pages || !pages->free_list || !pages->free_out || !work) return fail(QSTATE_EINVAL, "null pointer");
    if (R > 0 && (!pages->table || !pages->lens || !table_out)) return fail(QSTATE_EINVAL, "null pointer");
    if (!words(pages->table, pages->lens, pages->free_list, pages->free_out, others, left, table_out))
        return fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned");
    if (!aligned(work, 256)) return fail(QSTATE_EINVAL, "the work space must be 256-byte aligned");
    KvCompactParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    p.pages = *pages;
    p.moves = *moves;
    p.others = others;
    p.table_out = table_out;
    p.left = left;
    p.R = R;
    p.limit = limit;
    p.page_shift = shift_of(cfg->page);
    p.n_pages = cfg->n_pages;
    p.max_pages = cfg->max_pages;
    p.parts = kv_column_parts(R, cfg->max_pages);
    p.chunk = kv_part_columns(cfg->max_pages, p.parts);
    const PagesWork w = pages_work(*cfg, R);
    char* const base = static_cast<char*>(work);
    p.head = static_cast<int*>(work) + 2;
    p.spans = reinterpret_cast<int2*>(base + w.spans);
    p.used = reinterpret_cast<uint32_t*>(base + w.used);
    p.rank = reinterpret_cast<int*>(base + w.rank);
    const cudaError_t e = launch_kv_compact(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "cache compaction kernels");
}

int qstate_kv_copy(const qstate_kv_cfg* cfg, const qstate_kv_cache* cache, const qstate_kv_moves* moves, void* stream) {
    int rc = check_cfg(cfg);
    if (rc || (rc = check_cache(cfg, cache)) || (rc = check_moves(moves))) return rc;
    if (moves->n == 0) return QSTATE_OK;
    KvCopyParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    p.src = moves->src;
    p.dst = moves->dst;
    p.n = moves->n;
    p.n_pages = cfg->n_pages;
    const long long rows = static_cast<long long>(cfg->Hkv) * cfg->page, entry = cfg->store == QSTATE_KV_E4M3 ? 1 : 2;
    void* const data[4] = {cache->k, cache->v, cache->k_exp, cache->v_exp};
    const long long bytes[4] = {rows * cfg->dk * entry, rows * cfg->dv * entry, rows, rows};
    for (int t = 0; t < 4; ++t) {
        if (!data[t]) continue;
        p.data[p.tensors] = data[t];
        p.bytes[p.tensors] = bytes[t];
        p.width[p.tensors++] = bytes[t] % 16 == 0 && aligned(data[t], 16) ? 16 : bytes[t] % 4 == 0 ? 4 : 1;
    }
    const cudaError_t e = launch_kv_copy(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "cache copy kernel");
}

int qstate_kv_group(const qstate_kv_cfg* cfg, const int32_t* lens, int32_t R, const int32_t* start, const int32_t* common, int32_t N,
                    void* groups, void* stream) {
    int rc = check_shared(cfg);
    if (rc || (rc = check_requests(R))) return rc;
    if (N < 0 || N > R) return fail(QSTATE_EINVAL, "need 0 <= N <= R");
    if (!groups || !start || (R > 0 && !lens) || (N > 0 && !common)) return fail(QSTATE_EINVAL, "null pointer");
    if (!words(lens, start, common)) return fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned");
    if (!aligned(groups, 16)) return fail(QSTATE_EINVAL, "groups must be 16-byte aligned");
    KvGroupParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    p.lens = lens;
    p.start = start;
    p.common = common;
    p.N = N;
    p.R = R;
    p.G = cfg->Hq / cfg->Hkv;
    p.Hkv = cfg->Hkv;
    p.tile = kSharedTile;
    p.rows = kv_shared_rows(cfg->dk);
    p.window = cfg->window;
    p.most = static_cast<long long>(cfg->max_pages) * cfg->page;
    // Measured: requests that read the same pages find them in L2 (11 TB/s at 128 entries); a half of a block takes a tile's 64 tokens
    // through its softmax, or, in e4m3, a block turns its codes into bf16.
    const bool e4m3 = cfg->store == QSTATE_KV_E4M3;
    p.alone_ns = (e4m3 ? 0.026f : 0.023f) * cfg->dk;
    p.block_ns = e4m3 ? 0.1f * cfg->dk : cfg->dk == 64 ? 3.0f : cfg->dk == 128 ? 3.3f : 8.6f;
    p.half_rows = e4m3 ? p.rows : 128;
    p.light_rows = !e4m3 && p.rows == 256 ? 128 : 0;
    p.least_ns = shared_least_ns();
    p.head.R = R;
    p.head.Hq = cfg->Hq;
    p.head.Hkv = cfg->Hkv;
    p.head.d = cfg->dk;
    p.head.e4m3 = e4m3;
    p.head.window = cfg->window;
    char* const base = static_cast<char*>(groups);
    p.out = reinterpret_cast<KvGroupHead*>(base);
    p.groups = reinterpret_cast<KvGroup*>(base + kKvGroupHeadBytes);
    p.shared = reinterpret_cast<int4*>(base + kKvGroupHeadBytes + kv_most_groups(R) * sizeof(KvGroup));
    const cudaError_t e = launch_kv_group(p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "shared groups kernel");
}

int qstate_kv_attend_shared(const qstate_kv_cfg* cfg, const qstate_kv_cache* cache, const void* q, int64_t q_row,
                            int64_t q_head, const int32_t* table, const int32_t* lens, int32_t R, const void* groups, void* o,
                            float* lse, void* work, void* stream) {
    int rc = check_shared(cfg);
    if (rc || (rc = check_cache(cfg, cache)) || (rc = check_requests(R))) return rc;
    if (R == 0) return QSTATE_OK;
    if ((rc = check_attend(q, table, lens, o, lse, work))) return rc;
    if (!groups) return fail(QSTATE_EINVAL, "null pointer");
    if (!aligned(groups, 16)) return fail(QSTATE_EINVAL, "groups must be 16-byte aligned");
    KvAttendParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
    fill_attend(cfg, cache, q, q_row, q_head, table, lens, R, o, lse, work, &p);
    p.groups = static_cast<const int*>(groups);
    p.shared = reinterpret_cast<const int4*>(static_cast<const char*>(groups) + kKvGroupHeadBytes + kv_most_groups(R) * sizeof(KvGroup));
    const SharedWork w = shared_work(*cfg, R);
    char* const base = static_cast<char*>(work);
    p.store = reinterpret_cast<float*>(base + w.store);
    p.store_ml = reinterpret_cast<float4*>(base + w.store_ml);
    p.dir = reinterpret_cast<int2*>(base + w.dir);
    p.pre_part = reinterpret_cast<float*>(base + w.part);
    p.pre_ml = reinterpret_cast<float4*>(base + w.part_ml);
    p.pre_store = reinterpret_cast<float*>(base + w.pre_store);
    p.pre_store_ml = reinterpret_cast<float4*>(base + w.pre_store_ml);
    p.pre_dir = reinterpret_cast<int2*>(base + w.pre_dir);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cfg->dk == 64 ? launch_kv_shared_64(*cfg, p, s)
                                  : cfg->dk == 128 ? launch_kv_shared_128(*cfg, p, s) : launch_kv_shared_256(*cfg, p, s);
    if (e == cudaSuccess) e = launch_kv_attend(*cfg, p, s);
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "shared attention kernels");
}

}  // extern "C"
