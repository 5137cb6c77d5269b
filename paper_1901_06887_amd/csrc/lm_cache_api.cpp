// Host side of the calls on language models' caches: argument checks and launches.
#include <cmath>

#include "lm_cache.h"
#include "../../include/mt_debug.h"

using namespace mt;

namespace {

constexpr uint32_t kMaxEntries = 1u << 20;       // of a batch
constexpr uint32_t kMaxPairs = 1u << 23;         // of a batch's sequences and heads
constexpr uint32_t kMaxQueryHeads = 65535;       // (a grid's second dimension)

#define LM_TRY(c, expr)                                                                                                     \
    do {                                                                                                                    \
        const hipError_t e_ = (expr);                                                                                       \
        if (e_ != hipSuccess) {                                                                                             \
            (void)hipGetLastError();                                                                                        \
            return ctx_fail((c), e_ == hipErrorOutOfMemory ? MT_ENOMEM : MT_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
        }                                                                                                                   \
    } while (0)

bool off16(const void* p) { return (uintptr_t)p % 16 != 0; }

// Blocks of `block` elements, `pages` of them apart by `page` and `layers` by `layer`: none reaches into another.
bool apart(uint64_t block, uint64_t pages, uint64_t page, uint64_t layers, uint64_t layer)
{
    if (pages > 1 && page < block) return false;
    if (layers > 1 && layer < block) return false;
    if (pages == 1 || layers == 1) return true;
    typedef unsigned __int128 wide;
    return layer >= (wide)(pages - 1) * page + block || page >= (wide)(layers - 1) * layer + block;
}

mt_status check_cache(mt_ctx* c, const mt_kv_cache* k)
{
    if (!k) return ctx_fail(c, MT_EINVAL, "null cache");
    if (!k->k || !k->v || !k->table || !k->lengths) return ctx_fail(c, MT_EINVAL, "null keys, values, table or lengths");
    if (k->dtype != MT_F32 && k->dtype != MT_BF16 && k->dtype != MT_KV8) return ctx_fail(c, MT_EUNSUPPORTED, "a cache of dtype %u", k->dtype);
    const bool narrow = k->dtype == MT_KV8;
    if ((k->k_scales != nullptr) != narrow || (k->v_scales != nullptr) != narrow) return ctx_fail(c, MT_EINVAL, "scales come with 8-bit caches, and only with them");
    if (!k->layers || !k->n_pages || !k->heads || !k->seqs || !k->table_width) return ctx_fail(c, MT_EINVAL, "a cache of no layers, pages, heads, sequences or width");
    if (k->page_tokens < 16 || k->page_tokens > 256 || (k->page_tokens & (k->page_tokens - 1))) return ctx_fail(c, MT_EUNSUPPORTED, "pages of %u tokens", k->page_tokens);
    if (k->head_dim == 0 || k->head_dim > MT_KV_MAX_DIM || k->head_dim % 16) return ctx_fail(c, MT_EUNSUPPORTED, "heads of %u elements", k->head_dim);
    if (k->seqs > MT_KV_MAX_SEQS || k->table_width > MT_KV_MAX_WIDTH || k->n_pages > (uint32_t)INT32_MAX || k->layers > 65535 || k->heads > kMaxQueryHeads ||
        (uint64_t)k->heads * k->page_tokens * k->head_dim > 1u << 28)
        return ctx_fail(c, MT_EUNSUPPORTED, "%u sequences of %u pages, %u pages of %u heads in %u layers", k->seqs, k->table_width, k->n_pages, k->heads, k->layers);
    const uint64_t es = k->dtype == MT_F32 ? 4 : narrow ? 1 : 2, rows = (uint64_t)k->heads * k->page_tokens;
    if (off16(k->k) || off16(k->v) || k->page_stride * es % 16 || k->layer_stride * es % 16 ||
        (narrow && (off16(k->k_scales) || off16(k->v_scales) || k->scales_page_stride % 16 || k->scales_layer_stride % 16)))
        return ctx_fail(c, MT_EINVAL, "pages and scales start on 16 bytes");
    if (!apart(rows * k->head_dim, k->n_pages, k->page_stride, k->layers, k->layer_stride) || (narrow && !apart(rows, k->n_pages, k->scales_page_stride, k->layers, k->scales_layer_stride)))
        return ctx_fail(c, MT_EINVAL, "strides make pages or layers overlap");
    if (k->table_stride < k->table_width) return ctx_fail(c, MT_EINVAL, "a table stride below the width %u", k->table_width);
    return MT_OK;
}

mt_status check_batch(mt_ctx* c, const mt_kv_cache* k, const mt_kv_batch* b, uint32_t dtype, uint32_t layer)
{
    if (!b) return ctx_fail(c, MT_EINVAL, "null batch");
    if (dtype > MT_BF16 || (k->dtype != MT_KV8 && k->dtype != dtype)) return ctx_fail(c, MT_EUNSUPPORTED, "rows of dtype %u with a cache of dtype %u", dtype, k->dtype);
    if (layer >= k->layers) return ctx_fail(c, MT_EINVAL, "layer %u of %u", layer, k->layers);
    if (!b->first_row && b->rows != b->n_seqs) return ctx_fail(c, MT_EINVAL, "%u rows of %u sequences, but no first_row", b->rows, b->n_seqs);
    if (!b->seqs && b->n_seqs > k->seqs) return ctx_fail(c, MT_EINVAL, "%u sequences of a cache of %u", b->n_seqs, k->seqs);
    if (b->rows && b->max_new == 0) return ctx_fail(c, MT_EINVAL, "max_new is 0");
    if (b->n_seqs > kMaxEntries || (uint64_t)b->n_seqs * k->heads > kMaxPairs) return ctx_fail(c, MT_EUNSUPPORTED, "%u sequences in a batch", b->n_seqs);
    if (b->rows > (uint32_t)INT32_MAX) return ctx_fail(c, MT_EUNSUPPORTED, "%u rows", b->rows);
    return MT_OK;
}

// Every call on pages: the cache, its books, the list.
mt_status check_pages(mt_ctx* c, const mt_kv_cache* k, const void* list, uint32_t n, bool at_most_seqs)
{
    const mt_status st = check_cache(c, k);
    if (st != MT_OK) return st;
    if (!k->refs || !k->work || off16(k->work) || k->work_bytes < page_work_bytes(k->n_pages, k->seqs))
        return ctx_fail(c, MT_EINVAL, "calls on pages need refs and %llu bytes of work memory on a 16-byte boundary", (unsigned long long)page_work_bytes(k->n_pages, k->seqs));
    if (n && !list) return ctx_fail(c, MT_EINVAL, "null list");
    if (at_most_seqs && n > k->seqs) return ctx_fail(c, MT_EINVAL, "%u entries for %u sequences", n, k->seqs);
    if (n > (uint32_t)INT32_MAX) return ctx_fail(c, MT_EUNSUPPORTED, "%u pairs", n);
    return MT_OK;
}

template <typename F> mt_status call_pages(mt_ctx* c, uint32_t n, F f)
{
    const CtxView v = ctx_view(c);
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    if (n == 0) return MT_OK;
    LM_TRY(c, hipSetDevice(v.device));
    LM_TRY(c, f());
    return MT_OK;
}

}  // namespace

mt_status mt_kv_write(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, const mt_kv_batch* b, const mt_kv_write_args* a)
{
    if (!c) return MT_EINVAL;
    if (!a) return ctx_fail(c, MT_EINVAL, "null arguments");
    mt_status st = check_cache(c, k);
    if (st == MT_OK) st = check_batch(c, k, b, a->dtype, a->layer);
    if (st != MT_OK) return st;
    const uint64_t width = (uint64_t)k->heads * k->head_dim;
    if (b->rows && (!a->k || !a->v)) return ctx_fail(c, MT_EINVAL, "null rows");
    if (a->k_stride < width || a->v_stride < width) return ctx_fail(c, MT_EINVAL, "a stride is below the %llu elements of a row", (unsigned long long)width);
    const CtxView v = ctx_view(c);
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    if (b->rows == 0 || b->n_seqs == 0) return MT_OK;
    LM_TRY(c, hipSetDevice(v.device));
    LM_TRY(c, launch_kv_write(KvWriteArgs{*k, *b, *a}, (hipStream_t)hip_stream));
    return MT_OK;
}

void mt_debug_kv_write_places(uint32_t length, uint32_t first, uint32_t last, uint32_t after, uint32_t reach, uint32_t* begin, uint32_t* stop)
{
    const Places p = places_of_rows((int32_t)length, (int32_t)first, (int32_t)last, (int32_t)after, (int32_t)reach);
    if (begin) *begin = (uint32_t)p.begin;
    if (stop) *stop = (uint32_t)p.stop;
}

mt_status mt_attend_scratch_get(const mt_kv_cache* k, const mt_kv_batch* b, uint32_t q_heads, uint32_t max_length, uint64_t* bytes)
{
    if (!k || !b || !bytes || !k->heads || !k->page_tokens || !k->table_width || q_heads == 0 || q_heads % k->heads || q_heads > kMaxQueryHeads || b->n_seqs > kMaxEntries || (uint64_t)b->n_seqs * k->heads > kMaxPairs) return MT_EINVAL;
    if (k->head_dim == 0 || k->head_dim > MT_KV_MAX_DIM || k->head_dim % 16) return MT_EUNSUPPORTED;
    *bytes = b->n_seqs ? attend_scratch_bytes(*k, *b, q_heads, max_length) : 0;
    return MT_OK;
}

mt_status mt_attend(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, const mt_kv_batch* b, const mt_attend_args* a)
{
    if (!c) return MT_EINVAL;
    if (!a) return ctx_fail(c, MT_EINVAL, "null arguments");
    mt_status st = check_cache(c, k);
    if (st == MT_OK) st = check_batch(c, k, b, a->dtype, a->layer);
    if (st != MT_OK) return st;
    if (a->q_heads == 0 || a->q_heads % k->heads) return ctx_fail(c, MT_EINVAL, "%u query heads on %u heads", a->q_heads, k->heads);
    if (a->q_heads > kMaxQueryHeads || (uint64_t)b->rows * (a->q_heads / k->heads) > (uint32_t)INT32_MAX) return ctx_fail(c, MT_EUNSUPPORTED, "%u rows of %u query heads", b->rows, a->q_heads);
    const uint64_t width = (uint64_t)a->q_heads * k->head_dim;
    if (b->rows && (!a->q || !a->out)) return ctx_fail(c, MT_EINVAL, "null rows");
    if (a->q_stride < width || a->out_stride < width) return ctx_fail(c, MT_EINVAL, "a stride is below the %llu elements of a row", (unsigned long long)width);
    if (!std::isfinite(a->scale) || std::fabs(a->scale) > 1e38f) return ctx_fail(c, MT_EINVAL, "scale is not finite, or beyond 1e38");
    const uint64_t need = b->rows && b->n_seqs ? attend_scratch_bytes(*k, *b, a->q_heads, a->max_length) : 0;
    if (need && (!a->scratch || a->scratch_bytes < need || off16(a->scratch)))
        return ctx_fail(c, MT_EINVAL, "the call needs %llu bytes of scratch on a 16-byte boundary", (unsigned long long)need);
    const CtxView v = ctx_view(c);
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    if (b->rows == 0 || b->n_seqs == 0) return MT_OK;
    LM_TRY(c, hipSetDevice(v.device));
    LM_TRY(c, launch_attend(AttendArgs{*k, *b, *a}, (hipStream_t)hip_stream));
    return MT_OK;
}

mt_status mt_kv_work_get(uint32_t n_pages, uint32_t seqs, uint64_t* bytes)
{
    if (!bytes || n_pages == 0 || seqs == 0) return MT_EINVAL;
    if (seqs > MT_KV_MAX_SEQS || n_pages > (uint32_t)INT32_MAX) return MT_EUNSUPPORTED;
    *bytes = page_work_bytes(n_pages, seqs);
    return MT_OK;
}

mt_status mt_kv_grow(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, const int32_t* seqs, const int32_t* tokens, uint32_t n, int32_t* granted)
{
    if (!c) return MT_EINVAL;
    const mt_status st = check_pages(c, k, tokens, n, true);
    if (st != MT_OK) return st;
    return call_pages(c, n, [&] { return launch_kv_grow(PagesArgs{*k, seqs, tokens, granted, n}, (hipStream_t)hip_stream); });
}

mt_status mt_kv_fork(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, const int32_t* parents, const int32_t* children, uint32_t n, int32_t* granted)
{
    if (!c) return MT_EINVAL;
    const mt_status st = check_pages(c, k, parents && children ? parents : nullptr, n, true);
    if (st != MT_OK) return st;
    return call_pages(c, n, [&] { return launch_kv_fork(PagesArgs{*k, parents, children, granted, n}, (hipStream_t)hip_stream); });
}

mt_status mt_kv_free(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, const int32_t* seqs, uint32_t n)
{
    if (!c) return MT_EINVAL;
    const mt_status st = check_pages(c, k, seqs, n, true);
    if (st != MT_OK) return st;
    return call_pages(c, n, [&] { return launch_kv_free(PagesArgs{*k, seqs, nullptr, nullptr, n}, (hipStream_t)hip_stream); });
}

mt_status mt_kv_compact(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, int32_t* live)
{
    if (!c) return MT_EINVAL;
    const mt_status st = check_pages(c, k, nullptr, 0, true);
    if (st != MT_OK) return st;
    return call_pages(c, 1, [&] { return launch_kv_compact(PagesArgs{*k, nullptr, nullptr, live, 0}, (hipStream_t)hip_stream); });
}

mt_status mt_kv_copy(mt_ctx* c, void* hip_stream, const mt_kv_cache* k, const int32_t* from, const int32_t* to, uint32_t n)
{
    if (!c) return MT_EINVAL;
    const mt_status st = check_pages(c, k, from && to ? from : nullptr, n, false);
    if (st != MT_OK) return st;
    return call_pages(c, n, [&] { return launch_kv_copy(PagesArgs{*k, from, to, nullptr, n}, (hipStream_t)hip_stream); });
}

mt_status mt_sample_scratch_get(uint32_t, uint32_t classes, uint64_t* bytes)
{
    if (!bytes || classes == 0) return MT_EINVAL;
    if (classes > MT_SAMPLE_MAX_CLASSES) return MT_EUNSUPPORTED;
    *bytes = 0;                  // (a row is one workgroup's, in LDS)
    return MT_OK;
}

mt_status mt_sample(mt_ctx* c, void* hip_stream, const mt_sample_args* a)
{
    if (!c) return MT_EINVAL;
    if (!a) return ctx_fail(c, MT_EINVAL, "null arguments");
    if (a->dtype > MT_BF16) return ctx_fail(c, MT_EUNSUPPORTED, "logits of dtype %u", a->dtype);
    if (a->classes == 0) return ctx_fail(c, MT_EINVAL, "no classes");
    if (a->classes > MT_SAMPLE_MAX_CLASSES) return ctx_fail(c, MT_EUNSUPPORTED, "%u classes", a->classes);
    const CtxView v = ctx_view(c);
    if (a->rows) {
        if (!a->logits || !a->uniform) return ctx_fail(c, MT_EINVAL, "null logits or random numbers");
        if (!a->ids && !a->logprobs && !a->kept) return ctx_fail(c, MT_EINVAL, "no output");
        if (a->row_stride < a->classes || (a->allowed && a->allowed_stride < (a->classes + 31) / 32)) return ctx_fail(c, MT_EINVAL, "a stride is below the %u classes", a->classes);
    }
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    if (a->rows == 0) return MT_OK;
    LM_TRY(c, hipSetDevice(v.device));
    LM_TRY(c, launch_sample(SampleArgs{*a}, (hipStream_t)hip_stream));
    return MT_OK;
}
