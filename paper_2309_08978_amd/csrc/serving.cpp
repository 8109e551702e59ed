// Entry points of the serving operators (include/nnjit.h): argument checks,
// parameters of the launches.
#include "serving_checks.h"

namespace nnjit {
namespace {

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

    AttentionPlan plan_for(int cus) const
    {
        const int kv_heads = p.q_heads / p.group;
        // (a tree's rows see over their window and the new tokens behind it)
        return p.mask ? tree_plan(dtype, p.batch.tokens, p.batch.sequences, p.q_heads, kv_heads, p.dim, max_q, max_kv,
                                  p.window > 0 ? p.window + max_q : 0, cus)
                      : attention_plan(dtype, p.batch.tokens, p.batch.sequences, p.q_heads, kv_heads, p.dim, max_q, max_kv, p.causal, p.window, cus);
    }
};

int64_t attention_floats(void *ctx, int cus) {
    AttentionCall &c = *(AttentionCall *)ctx;
    c.plan = c.plan_for(cus);
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

// What plain, causal and tree attention have in common; c.p: the mask of trees.
int attend(AttentionCall &c, const nnjit_paged_kv *cache, const nnjit_paged_batch *batch, int64_t q_heads, const void *q, int64_t q_token,
           int64_t q_head, void *out, int64_t out_token, int64_t out_head, float scale, int causal, int64_t window, void *stream, const char *what) {
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
    // (a plan has tiles of 16 rows or more and up to 256 splits: most calls need no closer look)
    const double lanes = (double)cache->kv_heads * (double)batch->sequences;
    const AttentionPlan least = ((c.max_q * c.p.group + 15) / 16) * 256 * lanes <= (double)kMaxGroups ? AttentionPlan{} : c.plan_for(1024);
    if (least.row_tiles * (double)least.splits * lanes > (double)kMaxGroups)
        return runtime_fail(NNJIT_EINVAL, "more than 2^24 - 1 workgroups (sequences times key heads times tiles)");
    return runtime_launch(c.stream, attention_floats, do_attention, &c, what);
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
    AttentionCall c;
    return attend(c, cache, batch, q_heads, q, q_token, q_head, out, out_token, out_head, scale, causal, window, stream, "paged_attention");
}

int nnjit_tree_attention(const nnjit_paged_kv *cache, const nnjit_paged_batch *batch, const uint32_t *mask, int64_t ld_mask,
                         int64_t mask_words, const int32_t *positions, int64_t q_heads, const void *q, int64_t q_token, int64_t q_head,
                         void *out, int64_t out_token, int64_t out_head, float scale, int64_t window, void *stream) {
    runtime_clear_error();
    if (mask_words < 1 || mask_words > 1 << 20) return runtime_fail(NNJIT_EINVAL, "mask_words=%lld out of [1, 2^20]", (long long)mask_words);
    if (ld_mask < 0) return runtime_fail(NNJIT_EINVAL, "negative ld_mask");
    if (!mask && batch && batch->tokens > 0) return runtime_fail(NNJIT_EINVAL, "mask is NULL");
    if (window > 0 && !positions && batch && batch->tokens > 0) return runtime_fail(NNJIT_EINVAL, "a window needs positions");
    AttentionCall c;
    c.p.mask = mask;
    c.p.ld_mask = ld_mask;
    c.p.mask_words = (int)mask_words;
    c.p.positions = positions;
    return attend(c, cache, batch, q_heads, q, q_token, q_head, out, out_token, out_head, scale, 1, window, stream, "tree_attention");
}

}  // extern "C"
