// qs_kv_api.cu -- C entries of the paged cache of attention layers: checks and dispatch.
#include <cmath>
#include <cstring>

#include "qs_kv.h"

using namespace qs;

namespace {

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

}  // namespace

extern "C" {

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
    if (rc || (rc = check_cache(cfg, cache))) return rc;
    if (R < 0 || R > kKvMaxRequests) return fail(QSTATE_EINVAL, "need 0 <= R <= %d", kKvMaxRequests);
    if (R == 0) return QSTATE_OK;
    if (!q || !table || !lens || !o || !work) return fail(QSTATE_EINVAL, "null pointer");
    if (!aligned(q, 2)) return fail(QSTATE_EINVAL, "q must be 2-byte aligned");
    if (!words(table, lens, lse)) return fail(QSTATE_EINVAL, "arrays of 32-bit entries must be 4-byte aligned");
    if (!aligned(o, 16)) return fail(QSTATE_EINVAL, "o must be 16-byte aligned");
    if (!aligned(work, 256)) return fail(QSTATE_EINVAL, "the work space must be 256-byte aligned");
    KvAttendParams p;
    std::memset(&p, 0, sizeof(p));
    if ((rc = acquire_status(&p.status))) return rc;
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
    const cudaError_t e = launch_kv_attend(*cfg, p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? QSTATE_OK : cuda_fail(e, "cache attention kernel");
}

}  // extern "C"
