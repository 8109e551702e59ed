// Entry points of the serving operators (include/nnjit.h): argument checks,
// parameters of the launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "nnjit.h"
#include "serving.h"

namespace nnjit {
namespace {

constexpr int64_t kMaxInt = 0x7fffffff;
constexpr int64_t kMaxHeads = (int64_t)1 << 30;   // of a row that is turned: steps from head to head stay inside 32 bits
constexpr int64_t kMaxGroups = 0xffffff;          // workgroups of 256 threads: a launch holds below 2^32 threads

bool is_dtype(int d) { return d == NNJIT_F32 || d == NNJIT_F16; }
int64_t bytes_of(int dtype) { return dtype == NNJIT_F32 ? 4 : 2; }

// rows whose pointer and strides are multiples of `elems` elements
bool in_units(const void *p, int64_t tok, int64_t head, int64_t elems, int dtype) {
    return (uintptr_t)p % (uintptr_t)(elems * bytes_of(dtype)) == 0 && tok % elems == 0 && head % elems == 0;
}

int check_rows(const char *name, const void *p, int64_t rows, int64_t heads, int64_t tok, int64_t head) {
    if (rows > 0 && heads > 0 && !p) return runtime_fail(NNJIT_EINVAL, "%s is NULL", name);
    if (tok < 0 || head < 0) return runtime_fail(NNJIT_EINVAL, "negative stride of %s", name);
    return NNJIT_OK;
}

// rows that are written: none may overlap
int check_written(const char *name, const void *p, int64_t rows, int64_t heads, int64_t dim, int64_t tok, int64_t head) {
    const int rc = check_rows(name, p, rows, heads, tok, head);
    if (rc != NNJIT_OK || heads == 0 || rows == 0) return rc;
    if (heads > 1 && head < dim) return runtime_fail(NNJIT_EINVAL, "head stride %lld of %s < %lld dims", (long long)head, name, (long long)dim);
    const int64_t least = heads > 1 && tok >= head ? (heads - 1) * head + dim : dim;
    const bool heads_outside = heads > 1 && tok < head;   // heads major, tokens within
    if (rows > 1 && (tok < least || (heads_outside && head < (rows - 1) * tok + dim)))
        return runtime_fail(NNJIT_EINVAL, "rows of %s overlap (token stride %lld, head stride %lld)", name, (long long)tok, (long long)head);
    return NNJIT_OK;
}

int check_dim(int64_t dim) {
    if (dim < 1 || dim > kMaxHeadDim) return runtime_fail(NNJIT_EINVAL, "head_dim=%lld out of [1, %d]", (long long)dim, kMaxHeadDim);
    return NNJIT_OK;
}

int check_rotary(const nnjit_rotary_table *r, int64_t dim) {
    if (!r->table) return runtime_fail(NNJIT_EINVAL, "the rotary table is NULL");
    if (r->positions < 1 || r->positions > kMaxInt) return runtime_fail(NNJIT_EINVAL, "rotary positions=%lld out of [1, 2^31)", (long long)r->positions);
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > dim)
        return runtime_fail(NNJIT_EINVAL, "rotary_dim=%lld must be even and in [2, head_dim=%lld]", (long long)r->rotary_dim, (long long)dim);
    if (r->layout != NNJIT_ROTARY_HALF && r->layout != NNJIT_ROTARY_INTERLEAVED)
        return runtime_fail(NNJIT_EINVAL, "unknown rotary layout %d", r->layout);
    return NNJIT_OK;
}

int check_cache(const nnjit_paged_kv *c) {
    if (!c) return runtime_fail(NNJIT_EINVAL, "the cache is NULL");
    if (!is_dtype(c->dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported cache dtype %d", c->dtype);
    const int rc = check_dim(c->head_dim);
    if (rc != NNJIT_OK) return rc;
    if (c->pages < 1 || c->pages > kMaxInt) return runtime_fail(NNJIT_EINVAL, "pages=%lld out of [1, 2^31)", (long long)c->pages);
    if (c->page_size < 1 || c->page_size > kMaxKeys) return runtime_fail(NNJIT_EINVAL, "page_size=%lld out of [1, 2^30]", (long long)c->page_size);
    if (c->kv_heads < 1 || c->kv_heads > kMaxInt) return runtime_fail(NNJIT_EINVAL, "kv_heads=%lld out of [1, 2^31)", (long long)c->kv_heads);
    if (!c->k || !c->v) return runtime_fail(NNJIT_EINVAL, "the cache's K or V is NULL");
    if (c->k_page < 0 || c->k_token < 0 || c->k_head < 0 || c->v_page < 0 || c->v_token < 0 || c->v_head < 0)
        return runtime_fail(NNJIT_EINVAL, "negative stride of the cache");
    if (std::max({c->k_page, c->k_token, c->v_page, c->v_token}) > (int64_t)0xffffffff)
        return runtime_fail(NNJIT_EINVAL, "page and token strides of the cache must be below 2^32 elements");
    return NNJIT_OK;
}

// slots that are written: none may overlap
int check_slots(const char *name, const nnjit_paged_kv *c, int64_t page, int64_t token, int64_t head) {
    struct { int64_t stride, count; } axis[3] = {{page, c->pages}, {token, c->page_size}, {head, c->kv_heads}};
    std::sort(axis, axis + 3, [](const auto &a, const auto &b) { return a.stride < b.stride; });
    double taken = (double)c->head_dim;                    // elements from the first to the last, axis by axis
    for (const auto &a : axis) {
        if (a.count == 1) continue;
        if ((double)a.stride < taken) return runtime_fail(NNJIT_EINVAL, "slots of the cache's %s overlap (stride %lld)", name, (long long)a.stride);
        taken += (double)a.stride * (double)(a.count - 1);
    }
    return NNJIT_OK;
}

int check_batch(const nnjit_paged_batch *b) {
    if (!b) return runtime_fail(NNJIT_EINVAL, "the batch is NULL");
    if (b->sequences < 0 || b->sequences > kMaxInt || b->tokens < 0 || b->tokens > kMaxInt)
        return runtime_fail(NNJIT_EINVAL, "sequences=%lld, tokens=%lld out of [0, 2^31)", (long long)b->sequences, (long long)b->tokens);
    if (b->table_pages < 0 || b->table_pages > kMaxInt) return runtime_fail(NNJIT_EINVAL, "table_pages=%lld out of [0, 2^31)", (long long)b->table_pages);
    if (b->ld_table < b->table_pages) return runtime_fail(NNJIT_EINVAL, "ld_table=%lld < %lld page table columns", (long long)b->ld_table, (long long)b->table_pages);
    if (b->sequences > 0 && b->tokens > 0) {
        if (!b->q_start || !b->kv_len) return runtime_fail(NNJIT_EINVAL, "q_start or kv_len is NULL");
        if (b->table_pages > 0 && !b->page_table) return runtime_fail(NNJIT_EINVAL, "page_table is NULL");
    }
    return NNJIT_OK;
}

PagePool pool_of(const nnjit_paged_kv *c) {
    PagePool p;
    p.k = c->k;
    p.v = c->v;
    p.k_page = (unsigned)c->k_page;
    p.k_tok = (unsigned)c->k_token;
    p.k_head = c->k_head;
    p.v_page = (unsigned)c->v_page;
    p.v_tok = (unsigned)c->v_token;
    p.v_head = c->v_head;
    p.pages = (int)c->pages;
    p.page_size = FastDiv((unsigned)c->page_size);
    return p;
}

PageBatch batch_of(const nnjit_paged_batch *b) {
    return PageBatch{b->q_start, b->kv_len, b->page_table, b->ld_table, (int)b->table_pages, (int)b->sequences, (int)b->tokens};
}

bool pool_in_units(const nnjit_paged_kv *c, int64_t elems) {
    return in_units(c->k, c->k_token, c->k_head, elems, c->dtype) && in_units(c->v, c->v_token, c->v_head, elems, c->dtype) &&
           c->k_page % elems == 0 && c->v_page % elems == 0;
}

struct RotaryCall {
    RotaryParams p{};
    bool append = false, vec = false;
    int src = 0, dst = 0;
    hipStream_t stream = nullptr;
};

hipError_t do_rotary(void *ctx, const RuntimeDevice &) {
    const RotaryCall &c = *(const RotaryCall *)ctx;
    return launch_rotary(c.p, c.append, c.src, c.dst, c.vec, c.stream);
}

struct AttentionCall {
    AttentionParams p{};
    AttentionPlan plan{};
    int dtype = 0;
    bool vec = false;
    int64_t max_q = 0, max_kv = 0;
    hipStream_t stream = nullptr;
};

int64_t attention_floats(void *ctx, int cus) {
    AttentionCall &c = *(AttentionCall *)ctx;
    const AttentionParams &p = c.p;
    c.plan = attention_plan(c.dtype, p.batch.tokens, p.batch.sequences, p.q_heads, p.q_heads / p.group, p.dim, c.max_q, c.max_kv,
                            p.causal, p.window, cus);
    return c.plan.ws_floats;
}

hipError_t do_attention(void *ctx, const RuntimeDevice &d) {
    AttentionCall &c = *(AttentionCall *)ctx;
    c.p.zero = d.zero;
    if (c.plan.splits > 1) {
        const int64_t rows = (int64_t)c.plan.splits * c.p.batch.tokens * c.p.q_heads;
        c.p.part_dim = (c.p.dim + 3) / 4 * 4;
        c.p.part = d.ws;
        c.p.stat = d.ws + rows * c.p.part_dim;
    }
    return launch_attention(c.p, c.plan, c.dtype, c.vec, c.stream);
}

struct TableCall {
    float *table;
    int positions, rot, scaling;
    double base, factor, original, fast, slow, magnitude;
    hipStream_t stream;
};

hipError_t do_table(void *ctx, const RuntimeDevice &) {
    const TableCall &c = *(const TableCall *)ctx;
    return launch_rotary_table(c.table, c.positions, c.rot, c.base, c.scaling, c.factor, c.original, c.fast, c.slow, c.magnitude, c.stream);
}

}  // namespace
}  // namespace nnjit

using namespace nnjit;

extern "C" {

int nnjit_rotary_fill(float *table, int64_t positions, int64_t rotary_dim, double base, const nnjit_rotary_scaling *scaling,
                      void *stream) {
    runtime_clear_error();
    if (positions < 0 || positions > kMaxInt) return runtime_fail(NNJIT_EINVAL, "positions=%lld out of [0, 2^31)", (long long)positions);
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > kMaxHeadDim)
        return runtime_fail(NNJIT_EINVAL, "rotary_dim=%lld must be even and in [2, %d]", (long long)rotary_dim, kMaxHeadDim);
    if (!(base > 1.0) || !std::isfinite(base)) return runtime_fail(NNJIT_EINVAL, "base=%g must be finite and above 1", base);
    const nnjit_rotary_scaling none = {NNJIT_ROTARY_PLAIN, 1.0, 1.0, 2.0, 1.0, 1.0};
    const nnjit_rotary_scaling &s = scaling ? *scaling : none;
    if (s.kind < NNJIT_ROTARY_PLAIN || s.kind > NNJIT_ROTARY_INDEX) return runtime_fail(NNJIT_EINVAL, "unknown rotary scaling %d", s.kind);
    if (s.kind != NNJIT_ROTARY_PLAIN && !(s.factor > 0.0 && std::isfinite(s.factor)))
        return runtime_fail(NNJIT_EINVAL, "scaling factor %g must be finite and above 0", s.factor);
    if ((s.kind == NNJIT_ROTARY_TURNS || s.kind == NNJIT_ROTARY_INDEX) &&
        !(s.original > 0.0 && s.slow > 0.0 && s.fast > s.slow && std::isfinite(s.original) && std::isfinite(s.fast)))
        return runtime_fail(NNJIT_EINVAL, "a ramp needs original > 0 and fast > slow > 0 (got %g, %g, %g)", s.original, s.fast, s.slow);
    if (!std::isfinite(s.magnitude)) return runtime_fail(NNJIT_EINVAL, "magnitude is not finite");
    if (positions == 0) return NNJIT_OK;
    if (positions * (rotary_dim / 2) > kMaxGroups * 256) return runtime_fail(NNJIT_EINVAL, "a table of %lld positions: below 2^32 pairs are served", (long long)positions);
    if (!table) return runtime_fail(NNJIT_EINVAL, "table is NULL");
    TableCall c{table, (int)positions, (int)rotary_dim, s.kind, base, s.factor, s.original, s.fast, s.slow, s.magnitude, (hipStream_t)stream};
    return runtime_launch(c.stream, nullptr, do_table, &c, "rotary_table");
}

int nnjit_rotary(const nnjit_rotary_table *rotary, int64_t tokens, int64_t heads, int64_t head_dim, const int32_t *positions,
                 const void *x, int64_t x_token, int64_t x_head, int x_dtype, void *y, int64_t y_token, int64_t y_head,
                 int y_dtype, int transpose, void *stream) {
    runtime_clear_error();
    if (!is_dtype(x_dtype) || !is_dtype(y_dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d to %d", x_dtype, y_dtype);
    if (tokens < 0 || tokens > kMaxInt || heads < 0 || heads > kMaxHeads)
        return runtime_fail(NNJIT_EINVAL, "tokens=%lld out of [0, 2^31) or heads=%lld out of [0, 2^30]", (long long)tokens, (long long)heads);
    int rc = check_dim(head_dim);
    if (rc != NNJIT_OK) return rc;
    if (!rotary) return runtime_fail(NNJIT_EINVAL, "rotary is NULL");
    if ((rc = check_rotary(rotary, head_dim)) != NNJIT_OK) return rc;
    if ((rc = check_rows("x", x, tokens, heads, x_token, x_head)) != NNJIT_OK) return rc;
    if ((rc = check_written("y", y, tokens, heads, head_dim, y_token, y_head)) != NNJIT_OK) return rc;
    if (tokens == 0 || heads == 0) return NNJIT_OK;
    if (tokens > kMaxGroups) return runtime_fail(NNJIT_EINVAL, "%lld tokens in one call: below 2^24 are served", (long long)tokens);
    if (!positions) return runtime_fail(NNJIT_EINVAL, "positions is NULL");
    RotaryCall c;
    c.p.q = HeadRows{x, x_token, x_head};
    c.p.qo = HeadRows{y, y_token, y_head};
    c.p.q_heads = (int)heads;
    c.p.positions = positions;
    c.p.table = rotary->table;
    c.p.table_rows = (int)rotary->positions;
    c.p.rot = (int)rotary->rotary_dim;
    c.p.dim = (int)head_dim;
    c.p.tokens = (int)tokens;
    c.p.interleaved = rotary->layout == NNJIT_ROTARY_INTERLEAVED;
    c.p.sign = transpose ? -1.f : 1.f;
    c.vec = head_dim % 8 == 0 && c.p.rot % 8 == 0 && in_units(x, x_token, x_head, 4, x_dtype) && in_units(y, y_token, y_head, 4, y_dtype);
    c.src = x_dtype;
    c.dst = y_dtype;
    c.stream = (hipStream_t)stream;
    return runtime_launch(c.stream, nullptr, do_rotary, &c, "rotary");
}

int nnjit_kv_append(const nnjit_paged_kv *cache, const nnjit_paged_batch *batch, const nnjit_rotary_table *rotary, const void *k,
                    int64_t k_token, int64_t k_head, const void *v, int64_t v_token, int64_t v_head, int64_t q_heads, const void *q,
                    int64_t q_token, int64_t q_head, void *q_out, int64_t qo_token, int64_t qo_head, int src_dtype, void *stream) {
    runtime_clear_error();
    int rc = check_cache(cache);
    if (rc != NNJIT_OK) return rc;
    if ((rc = check_batch(batch)) != NNJIT_OK) return rc;
    if (!is_dtype(src_dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d", src_dtype);
    if (q_heads < 0 || q_heads > kMaxHeads - 2 * cache->kv_heads)
        return runtime_fail(NNJIT_EINVAL, "q_heads=%lld out of [0, 2^30 - 2 kv_heads]", (long long)q_heads);
    const int64_t dim = cache->head_dim;
    if ((rc = check_slots("K", cache, cache->k_page, cache->k_token, cache->k_head)) != NNJIT_OK) return rc;
    if ((rc = check_slots("V", cache, cache->v_page, cache->v_token, cache->v_head)) != NNJIT_OK) return rc;
    if (rotary && (rc = check_rotary(rotary, dim)) != NNJIT_OK) return rc;
    if ((rc = check_rows("k", k, batch->tokens, cache->kv_heads, k_token, k_head)) != NNJIT_OK) return rc;
    if ((rc = check_rows("v", v, batch->tokens, cache->kv_heads, v_token, v_head)) != NNJIT_OK) return rc;
    if ((rc = check_rows("q", q, batch->tokens, q_heads, q_token, q_head)) != NNJIT_OK) return rc;
    if ((rc = check_written("q_out", q_out, batch->tokens, q_heads, dim, qo_token, qo_head)) != NNJIT_OK) return rc;
    if (batch->tokens == 0 || batch->sequences == 0) return NNJIT_OK;
    if (batch->tokens > kMaxGroups) return runtime_fail(NNJIT_EINVAL, "%lld tokens in one call: below 2^24 are served", (long long)batch->tokens);
    RotaryCall c;
    c.p.q = HeadRows{q, q_token, q_head};
    c.p.qo = HeadRows{q_out, qo_token, qo_head};
    c.p.q_heads = (int)q_heads;
    c.p.k = HeadRows{k, k_token, k_head};
    c.p.v = HeadRows{v, v_token, v_head};
    c.p.kv_heads = (int)cache->kv_heads;
    c.p.pool = pool_of(cache);
    c.p.batch = batch_of(batch);
    c.p.table = rotary ? rotary->table : nullptr;
    c.p.table_rows = rotary ? (int)rotary->positions : 1;
    c.p.rot = rotary ? (int)rotary->rotary_dim : 0;
    c.p.dim = (int)dim;
    c.p.tokens = (int)batch->tokens;
    c.p.interleaved = rotary && rotary->layout == NNJIT_ROTARY_INTERLEAVED;
    c.p.sign = 1.f;
    c.append = true;
    c.vec = dim % 8 == 0 && c.p.rot % 8 == 0 && in_units(k, k_token, k_head, 4, src_dtype) && in_units(v, v_token, v_head, 4, src_dtype) &&
            (q_heads == 0 || (in_units(q, q_token, q_head, 4, src_dtype) && in_units(q_out, qo_token, qo_head, 4, cache->dtype))) &&
            pool_in_units(cache, 4);
    c.src = src_dtype;
    c.dst = cache->dtype;
    c.stream = (hipStream_t)stream;
    return runtime_launch(c.stream, nullptr, do_rotary, &c, "kv_append");
}

int nnjit_paged_attention(const nnjit_paged_kv *cache, const nnjit_paged_batch *batch, int64_t q_heads, const void *q, int64_t q_token,
                          int64_t q_head, void *out, int64_t out_token, int64_t out_head, float scale, int causal, int64_t window,
                          void *stream) {
    runtime_clear_error();
    int rc = check_cache(cache);
    if (rc != NNJIT_OK) return rc;
    if ((rc = check_batch(batch)) != NNJIT_OK) return rc;
    if (q_heads < 1 || q_heads > kMaxInt || q_heads % cache->kv_heads)
        return runtime_fail(NNJIT_EINVAL, "q_heads=%lld is no multiple of kv_heads=%lld", (long long)q_heads, (long long)cache->kv_heads);
    if (batch->max_q < 0 || batch->max_q > kMaxInt) return runtime_fail(NNJIT_EINVAL, "max_q=%lld out of [0, 2^31)", (long long)batch->max_q);
    if (batch->max_kv < 0 || batch->max_kv > kMaxKeys) return runtime_fail(NNJIT_EINVAL, "max_kv=%lld out of [0, 2^30]", (long long)batch->max_kv);
    if (!std::isfinite(scale)) return runtime_fail(NNJIT_EINVAL, "scale is not finite");
    if (window < 0) return runtime_fail(NNJIT_EINVAL, "window=%lld is negative", (long long)window);
    if (window > 0 && !causal) return runtime_fail(NNJIT_EINVAL, "a window needs causal attention");
    const int64_t dim = cache->head_dim, rows = batch->tokens;
    if ((rc = check_rows("q", q, rows, q_heads, q_token, q_head)) != NNJIT_OK) return rc;
    if ((rc = check_written("out", out, rows, q_heads, dim, out_token, out_head)) != NNJIT_OK) return rc;
    if (rows == 0 || batch->sequences == 0 || batch->max_q == 0) return NNJIT_OK;
    const int64_t units = (cache->dtype == NNJIT_F16) ? 8 : 4;   // elements of 16 bytes
    AttentionCall c;
    c.p.q = HeadRows{q, q_token, q_head};
    c.p.o = HeadRows{out, out_token, out_head};
    c.p.q_heads = (int)q_heads;
    c.p.group = (int)(q_heads / cache->kv_heads);
    c.p.group_div = FastDiv((unsigned)c.p.group);
    c.p.dim = (int)dim;
    c.p.pool = pool_of(cache);
    c.p.batch = batch_of(batch);
    // a scale of 0 (all keys alike) would make NaNs of masked logits: 2^-100 leaves
    // the weights of all q . k below 2^76 alike to the last bit
    c.p.scale_log2 = (float)std::fmin(std::fmax(std::fabs((double)scale) * 1.4426950408889634074, 0x1p-100), (double)std::numeric_limits<float>::max());
    c.p.negate = scale < 0.f;
    c.p.causal = causal != 0;
    c.p.window = (int)std::min<int64_t>(window, kMaxInt);
    c.dtype = cache->dtype;
    c.vec = dim % units == 0 && in_units(q, q_token, q_head, units, c.dtype) && in_units(out, out_token, out_head, units, c.dtype) &&
            pool_in_units(cache, units);
    c.max_q = std::min(batch->max_q, rows);
    const int64_t room = batch->table_pages * cache->page_size;
    c.max_kv = std::min(batch->max_kv, room);
    c.stream = (hipStream_t)stream;
    if (rows * q_heads > kMaxInt || c.max_q * c.p.group > kMaxInt - 64)
        return runtime_fail(NNJIT_EINVAL, "%lld rows of %lld heads in one call: below 2^31 are served", (long long)rows, (long long)q_heads);
    const AttentionPlan least = attention_plan(c.dtype, rows, batch->sequences, c.p.q_heads, (int)cache->kv_heads, c.p.dim, c.max_q, c.max_kv,
                                               c.p.causal, c.p.window, 1024);
    if ((double)least.row_tiles * least.splits * (double)cache->kv_heads * (double)batch->sequences > (double)kMaxGroups)
        return runtime_fail(NNJIT_EINVAL, "more than 2^24 - 1 workgroups (sequences times key heads times tiles)");
    return runtime_launch(c.stream, attention_floats, do_attention, &c, "paged_attention");
}

}  // extern "C"
