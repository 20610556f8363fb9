// Entry points of the paged cache: argument checks, and dispatch to the kernels of cache_rows.hip and cache_attend*.hip.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "cache.hpp"

#define BF_HIP(call)                                                   \
    do {                                                               \
        hipError_t e_ = (call);                                        \
        if (e_ != hipSuccess) return bf::record_hip_error(e_, #call);  \
    } while (0)

namespace {

bool spec_ok(const bifeat_cache_spec *s) {
    return s && (s->bits == 4 || s->bits == 8) && s->heads >= 1 && s->heads <= 1024 && s->head_dim >= 1 && s->head_dim <= 256 &&
           s->page_size >= 16 && s->page_size <= 1024 && (s->page_size & (s->page_size - 1)) == 0;
}

bool type_ok(int32_t d) { return d == BIFEAT_F32 || d == BIFEAT_F16 || d == BIFEAT_BF16; }
uintptr_t type_bytes(int32_t d) { return d == BIFEAT_F32 ? 4 : 2; }

// The batch alone; heads: rows a token that the call's kernels are launched for.
bool batch_ok(const bifeat_cache *c, const bifeat_cache_batch *b, int64_t heads) {
    if (!b || b->sequences < 0 || b->tokens < 0 || b->table_width < 0) return false;
    if (b->sequences > INT32_MAX || b->table_width > bf::kMostPositions / c->spec.page_size || b->tokens > (int64_t)INT32_MAX / heads) return false;
    if (b->tokens == 0) return true;
    if (b->sequences == 0 || !b->lengths || (b->table_width > 0 && !b->tables)) return false;
    if ((uintptr_t)b->lengths % 8 || (uintptr_t)b->indptr % 8 || (uintptr_t)b->tables % 4) return false;
    return b->indptr || b->tokens % b->sequences == 0;
}

bool rows_ok(const bifeat_head_rows *r, int32_t dtype) {
    return r && r->data && (uintptr_t)r->data % type_bytes(dtype) == 0 && r->token_stride >= 0 && r->head_stride >= 0;
}

bf::CachePages pages_of(const bifeat_cache *c, const uint8_t *pages) {
    return {const_cast<uint8_t *>(pages), c->head_bytes, c->page_bytes, c->spec.heads, c->spec.head_dim, c->rb,
            bf::ilog2(c->spec.page_size)};
}

bf::CacheBatch batch_of(const bifeat_cache_batch *b) {
    return {b->tables, b->lengths, b->indptr, b->table_width, b->tokens, (int)b->sequences,
            b->indptr ? 0 : (int)(b->tokens / b->sequences)};
}

bf::HeadRows rows_of(const bifeat_head_rows *r) { return {r->data, r->token_stride, r->head_stride}; }

int check(const bifeat_cache *c, int64_t num_pages, const bf::CacheBatch &b, hipStream_t s) {
    void *blk = nullptr;
    if (int rc = bf::take_block(&blk)) return rc;
    int32_t bad = 0;
    bf::launch_cache_check(b, bf::ilog2(c->spec.page_size), num_pages, (int32_t *)blk, s);
    hipError_t e = hipMemcpyAsync(&bad, blk, sizeof(bad), hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    if (e != hipSuccess) return bf::record_hip_error(e, "bifeat_cache_check");
    bf::give_block(blk);
    return bad ? BIFEAT_EINVAL : BIFEAT_OK;
}

// What the four calls ask of their common arguments.
int common(const bifeat_cache *c, const uint8_t *pages, int64_t num_pages, const bifeat_cache_batch *batch, int64_t heads,
           int32_t dtype) {
    if (!c || !type_ok(dtype) || num_pages < 0 || num_pages > INT32_MAX || !batch_ok(c, batch, heads)) return BIFEAT_EINVAL;
    if ((uintptr_t)pages % 16 || (batch->tokens > 0 && num_pages > 0 && !pages)) return BIFEAT_EINVAL;
    return BIFEAT_OK;
}

}  // namespace

extern "C" {

int bifeat_cache_create(const bifeat_cache_spec *spec, bifeat_cache **out) {
    if (!out) return BIFEAT_EINVAL;
    *out = nullptr;
    if (!spec_ok(spec)) return BIFEAT_EINVAL;
    bifeat_cache *c = new (std::nothrow) bifeat_cache();
    if (!c) return BIFEAT_EHIP;
    c->spec = *spec;
    c->rb = (spec->head_dim * spec->bits + 127) / 128 * 16;
    c->head_bytes = (int64_t)spec->page_size * (2 * c->rb + 16);
    c->page_bytes = c->head_bytes * spec->heads;
    *out = c;
    return BIFEAT_OK;
}

void bifeat_cache_destroy(bifeat_cache *c) {
    if (!c) return;
    while (bifeat_cache::Workspace *w = c->workspaces) {
        (void)hipFree(w->partial);
        c->workspaces = w->next;
        delete w;
    }
    delete c;
}

int64_t bifeat_cache_page_bytes(const bifeat_cache *c) { return c ? c->page_bytes : BIFEAT_EINVAL; }

int bifeat_cache_set_option(bifeat_cache *c, const char *name, int value) {
    if (!c || !name) return BIFEAT_EINVAL;
    if (!strcmp(name, "validate") && (value == 0 || value == 1)) {
        c->opt_validate = value;
        return BIFEAT_OK;
    }
    return BIFEAT_EINVAL;
}

int bifeat_cache_reserve(bifeat_cache *c, void *stream) {
    if (!c) return BIFEAT_EINVAL;
    const std::lock_guard<std::mutex> lock(c->mutex);
    return bf::workspace_of(c, (hipStream_t)stream) ? BIFEAT_OK : bf::record_hip_error(hipErrorOutOfMemory, "bifeat_cache_reserve");
}

int bifeat_cache_check(const bifeat_cache *c, int64_t num_pages, const bifeat_cache_batch *batch, void *stream) {
    if (!c || num_pages < 0 || !batch_ok(c, batch, 1)) return BIFEAT_EINVAL;
    if (batch->tokens == 0) return BIFEAT_OK;
    return check(c, num_pages, batch_of(batch), (hipStream_t)stream);
}

int bifeat_cache_write(bifeat_cache *c, uint8_t *pages, int64_t num_pages, const bifeat_cache_batch *batch, const bifeat_head_rows *k,
                       const bifeat_head_rows *v, int32_t dtype, void *stream) {
    if (int rc = common(c, pages, num_pages, batch, c ? 2 * c->spec.heads : 1, dtype)) return rc;
    if (batch->tokens == 0) return BIFEAT_OK;
    if (!rows_ok(k, dtype) || !rows_ok(v, dtype)) return BIFEAT_EINVAL;
    const bf::CacheBatch b = batch_of(batch);
    if (c->opt_validate)
        if (int rc = check(c, num_pages, b, (hipStream_t)stream)) return rc;
    BF_HIP(bf::launch_cache_write(pages_of(c, pages), b, rows_of(k), rows_of(v), c->spec.bits, dtype, (hipStream_t)stream));
    return BIFEAT_OK;
}

int bifeat_cache_append(bifeat_cache *c, uint8_t *pages, int64_t num_pages, const bifeat_cache_batch *batch, const bifeat_head_rows *q,
                        int32_t query_heads, const bifeat_head_rows *k, const bifeat_head_rows *v, int32_t dtype,
                        const bifeat_turn *turn, void *out, void *stream) {
    if (!c || query_heads < 0 || query_heads > 65536) return BIFEAT_EINVAL;
    if (int rc = common(c, pages, num_pages, batch, query_heads + 2 * c->spec.heads, dtype)) return rc;
    if (!turn || turn->pairs < 0 || turn->pairs > c->spec.head_dim / 2 || (turn->interleaved != 0 && turn->interleaved != 1) ||
        !isfinite(turn->scale) || (uintptr_t)turn->frequencies % 4)
        return BIFEAT_EINVAL;
    if (batch->tokens == 0) return BIFEAT_OK;
    if (!rows_ok(k, dtype) || !rows_ok(v, dtype) || (turn->pairs > 0 && !turn->frequencies)) return BIFEAT_EINVAL;
    if (query_heads > 0 && (!rows_ok(q, dtype) || !out || (uintptr_t)out % type_bytes(dtype))) return BIFEAT_EINVAL;
    const bf::CacheBatch b = batch_of(batch);
    if (c->opt_validate)
        if (int rc = check(c, num_pages, b, (hipStream_t)stream)) return rc;
    const bf::AppendCall a{query_heads ? rows_of(q) : bf::HeadRows{}, query_heads, rows_of(k), rows_of(v), c->spec.bits, dtype,
                           turn->frequencies, turn->pairs, turn->interleaved != 0, turn->scale, out, (hipStream_t)stream};
    BF_HIP(bf::launch_cache_append(pages_of(c, pages), b, a));
    return BIFEAT_OK;
}

int bifeat_cache_read(bifeat_cache *c, const uint8_t *pages, int64_t num_pages, const bifeat_cache_batch *batch, void *k, void *v,
                      int32_t dtype, void *stream) {
    if (int rc = common(c, pages, num_pages, batch, c ? 2 * c->spec.heads : 1, dtype)) return rc;
    if (batch->tokens == 0) return BIFEAT_OK;
    if (!k || !v || (uintptr_t)k % type_bytes(dtype) || (uintptr_t)v % type_bytes(dtype)) return BIFEAT_EINVAL;
    const bf::CacheBatch b = batch_of(batch);
    if (c->opt_validate)
        if (int rc = check(c, num_pages, b, (hipStream_t)stream)) return rc;
    BF_HIP(bf::launch_cache_read(pages_of(c, pages), b, k, v, c->spec.bits, dtype, (hipStream_t)stream));
    return BIFEAT_OK;
}

int bifeat_cache_attend(bifeat_cache *c, const uint8_t *pages, int64_t num_pages, const bifeat_cache_batch *batch,
                        const bifeat_head_rows *q, int32_t query_heads, int32_t dtype, const bifeat_attend_options *options, void *out,
                        void *stream) {
    if (!c || query_heads < 1 || query_heads > 65536 || query_heads % c->spec.heads) return BIFEAT_EINVAL;
    if (int rc = common(c, pages, num_pages, batch, query_heads, dtype)) return rc;
    if (batch->sequences > (1 << 30) / c->spec.heads) return BIFEAT_EINVAL;  // (items, which empty sequences have numbers for too, are ints)
    if (!options || !isfinite(options->scale) || !(options->softcap >= 0.f) || !isfinite(options->softcap) || options->window < 0 ||
        (uintptr_t)options->prefix % 8 || (uintptr_t)options->slopes % 4)
        return BIFEAT_EINVAL;
    if (batch->tokens == 0) return BIFEAT_OK;
    if (!rows_ok(q, dtype) || !out || (uintptr_t)out % type_bytes(dtype)) return BIFEAT_EINVAL;
    const bf::CacheBatch b = batch_of(batch);
    if (c->opt_validate)
        if (int rc = check(c, num_pages, b, (hipStream_t)stream)) return rc;
    const bf::AttendCall a{pages_of(c, pages), b, rows_of(q), query_heads / c->spec.heads, dtype, options->scale, options->softcap,
                           (int)std::min<int64_t>(options->window, bf::kMostPositions), options->prefix, options->slopes, out, (hipStream_t)stream};
    BF_HIP(bf::launch_cache_attend(c, a));
    return BIFEAT_OK;
}

}  // extern "C"
