// Entry points of a step of drafted tokens (include/nnjit.h): argument checks,
// parameters of the launches.
#include "serving_checks.h"

namespace nnjit {
namespace {

template <typename P>
struct Call {
    P p{};
    bool append = false, vec = false;
    int src = 0, dst = 0, unit = 0, groups = 0;
    const char *refused = nullptr;        // why, for calls that are looked at once there is a GPU
    hipStream_t stream = nullptr;
};

hipError_t do_step(void *ctx, const RuntimeDevice &) {
    const auto &c = *(const Call<StepParams> *)ctx;
    return launch_paged_step(c.p, c.stream);
}

int64_t norm_refused(void *ctx, int) {
    const auto &c = *(const Call<NormParams> *)ctx;
    return c.refused ? runtime_fail(NNJIT_EINVAL, "%s", c.refused) : 0;
}

hipError_t do_norm(void *ctx, const RuntimeDevice &) {
    const auto &c = *(const Call<NormParams> *)ctx;
    return launch_norm_rotary(c.p, c.append, c.src, c.dst, c.vec, c.stream);
}

int64_t norm_grad_floats(void *ctx, int cus) {
    auto &c = *(Call<NormParams> *)ctx;
    const bool per_head = c.p.qw_head > 0;
    c.groups = norm_grad_groups(c.p.tokens, c.p.q_heads, c.p.dim, per_head, c.vec, cus);
    return c.p.dw && c.groups > 1 ? (int64_t)c.groups * c.p.dim * (per_head ? c.p.q_heads : 1) : 0;
}

hipError_t do_norm_grad(void *ctx, const RuntimeDevice &d) {
    auto &c = *(Call<NormParams> *)ctx;
    c.p.part = d.ws;
    return launch_norm_rotary_grad(c.p, c.src, c.dst, c.vec, c.groups, c.stream);
}

hipError_t do_move(void *ctx, const RuntimeDevice &) {
    const auto &c = *(const Call<MoveParams> *)ctx;
    return launch_kv_move(c.p, (int)bytes_of(c.src), c.unit, c.stream);
}

hipError_t do_logits(void *ctx, const RuntimeDevice &d) {
    const auto &c = *(const Call<LogitParams> *)ctx;
    return launch_adjust_logits(c.p, c.src, c.dst, c.vec, d.cus, c.stream);
}

// a norm's weight: one row, or one a head
int check_weight(const char *name, const void *w, int64_t w_head, int dtype, float eps, int64_t dim) {
    if (!is_dtype(dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d of norm weights", dtype);
    if (!(eps >= 0.f) || !std::isfinite(eps)) return runtime_fail(NNJIT_EINVAL, "eps=%g must be finite and >= 0", (double)eps);
    if (w && (w_head < 0 || (w_head > 0 && w_head < dim)))
        return runtime_fail(NNJIT_EINVAL, "head stride %lld of %s: 0 (one weight) or at least %lld dims", (long long)w_head, name, (long long)dim);
    return NNJIT_OK;
}

int check_turned(const nnjit_rotary_table *rotary, const int32_t *positions, int64_t tokens, int64_t dim) {
    if (!rotary) return NNJIT_OK;
    const int rc = check_rotary(rotary, dim);
    if (rc != NNJIT_OK) return rc;
    if (tokens > 0 && !positions) return runtime_fail(NNJIT_EINVAL, "positions is NULL");
    return NNJIT_OK;
}

void set_rotary(NormParams &p, const nnjit_rotary_table *rotary, const int32_t *positions) {
    p.positions = positions;
    p.table = rotary ? rotary->table : nullptr;
    p.table_rows = rotary ? (int)rotary->positions : 1;
    p.rot = rotary ? (int)rotary->rotary_dim : 0;
    p.interleaved = rotary && rotary->layout == NNJIT_ROTARY_INTERLEAVED;
}

// weights and angles can be taken four at a time, and steps from head to head fit 32 bits
bool norm_in_units(const NormParams &p) {
    const int dtype = p.weight_half ? NNJIT_F16 : NNJIT_F32;
    return (!p.q_weight || in_units(p.q_weight, 0, p.qw_head, 4, dtype)) && (!p.k_weight || in_units(p.k_weight, 0, p.kw_head, 4, dtype)) &&
           (!p.table || in_units(p.table, 0, 0, 4, NNJIT_F32)) &&
           std::max({p.q.head, p.qo.head, p.k.head, p.v.head, p.dy.head, p.pool.k_head, p.pool.v_head}) <= (long long)0xffffffff;
}

// what nnjit_norm_rotary and its gradient have in common: *done: nothing is to be done
int check_norm_rows(const nnjit_rotary_table *rotary, int64_t tokens, int64_t heads, int64_t dim, const int32_t *positions, const void *weight,
                    int64_t w_head, int w_dtype, float eps, const void *x, int64_t x_token, int64_t x_head) {
    if (tokens < 0 || tokens > kMaxInt || heads < 0 || heads > kMaxHeads)
        return runtime_fail(NNJIT_EINVAL, "tokens=%lld out of [0, 2^31) or heads=%lld out of [0, 2^30]", (long long)tokens, (long long)heads);
    int rc = check_dim(dim);
    if (rc != NNJIT_OK) return rc;
    if ((rc = check_weight("weight", weight, w_head, w_dtype, eps, dim)) != NNJIT_OK) return rc;
    if ((rc = check_turned(rotary, positions, tokens, dim)) != NNJIT_OK) return rc;
    if ((rc = check_rows("x", x, tokens, heads, x_token, x_head)) != NNJIT_OK) return rc;
    if (heads > 0 && !weight) return runtime_fail(NNJIT_EINVAL, "weight is NULL");
    if (tokens > kMaxGroups) return runtime_fail(NNJIT_EINVAL, "%lld tokens in one call: below 2^24 are served", (long long)tokens);
    return NNJIT_OK;
}

}  // namespace
}  // namespace nnjit

using namespace nnjit;

extern "C" {

int nnjit_paged_step(const nnjit_page_pool *pool, const nnjit_step_arrays *step, void *stream) {
    runtime_clear_error();
    if (!pool || !step) return runtime_fail(NNJIT_EINVAL, "the pool or the step is NULL");
    const nnjit_step_arrays &s = *step;
    if (s.sequences < 0 || s.sequences > kStepSequences)
        return runtime_fail(NNJIT_EINVAL, "sequences=%lld out of [0, %d]", (long long)s.sequences, kStepSequences);
    if (s.tokens < 0 || s.tokens > kMaxGroups) return runtime_fail(NNJIT_EINVAL, "tokens=%lld out of [0, 2^24)", (long long)s.tokens);
    if (s.page_size < 1 || s.page_size > kMaxKeys) return runtime_fail(NNJIT_EINVAL, "page_size=%lld out of [1, 2^30]", (long long)s.page_size);
    if (s.table_pages < 0 || s.table_pages > kMaxInt) return runtime_fail(NNJIT_EINVAL, "table_pages=%lld out of [0, 2^31)", (long long)s.table_pages);
    if (s.ld_table < s.table_pages) return runtime_fail(NNJIT_EINVAL, "ld_table=%lld < %lld page table columns", (long long)s.ld_table, (long long)s.table_pages);
    if (pool->capacity < 0 || pool->capacity > kMaxInt) return runtime_fail(NNJIT_EINVAL, "capacity=%lld out of [0, 2^31)", (long long)pool->capacity);
    if (!pool->count || !pool->count_out || (pool->capacity > 0 && !pool->free_pages))
        return runtime_fail(NNJIT_EINVAL, "free_pages, count or count_out is NULL");
    if (!s.q_start || !s.status) return runtime_fail(NNJIT_EINVAL, "q_start or status is NULL");
    if (s.sequences > 0 && (!s.held || !s.added || !s.kv_len || (s.table_pages > 0 && !s.page_table)))
        return runtime_fail(NNJIT_EINVAL, "held, added, kv_len or page_table is NULL");
    // lengths are replaced in place where kv_len is held or keep as a whole; any other overlap would be read and written at once
    const auto kv_len_meets = [&](const int32_t *p, int64_t n) {
        return p && (uintptr_t)p < (uintptr_t)(s.kv_len + s.sequences) && (uintptr_t)s.kv_len < (uintptr_t)(p + n);
    };
    if (s.sequences > 0 && (kv_len_meets(s.added, s.sequences) || kv_len_meets(s.q_start, s.sequences + 1) ||
                            (s.kv_len != s.held && kv_len_meets(s.held, s.sequences)) || (s.kv_len != s.keep && kv_len_meets(s.keep, s.sequences))))
        return runtime_fail(NNJIT_EINVAL, "kv_len may be held or keep; it must not overlap a part of them, or added or q_start");
    const bool masks = s.parent || (s.mask && s.mask_words != 0);
    if (masks) {
        if (s.mask_words < 1 || s.mask_words > kStepWords)
            return runtime_fail(NNJIT_EINVAL, "mask_words=%lld out of [1, %d]", (long long)s.mask_words, kStepWords);
        if (s.ld_mask < s.mask_words) return runtime_fail(NNJIT_EINVAL, "ld_mask=%lld < %lld words", (long long)s.ld_mask, (long long)s.mask_words);
        if (s.tokens > 0 && !s.mask) return runtime_fail(NNJIT_EINVAL, "mask is NULL");
    }
    Call<StepParams> c;
    c.p.held = s.held;
    c.p.keep = s.keep == s.held ? nullptr : s.keep;
    c.p.added = s.added;
    c.p.parent = s.parent;
    c.p.page_table = s.page_table;
    c.p.ld_table = s.ld_table;
    c.p.table_pages = (int)s.table_pages;
    c.p.sequences = (int)s.sequences;
    c.p.tokens = (int)s.tokens;
    c.p.page_size = FastDiv((unsigned)s.page_size);
    c.p.q_start = s.q_start;
    c.p.kv_len = s.kv_len;
    c.p.positions = s.positions;
    c.p.slots = (long long *)s.slots;
    c.p.mask = masks ? s.mask : nullptr;
    c.p.ld_mask = s.ld_mask;
    c.p.mask_words = masks ? (int)s.mask_words : 0;
    c.p.status = s.status;
    c.p.free_pages = pool->free_pages;
    c.p.capacity = (int)pool->capacity;
    c.p.count = pool->count;
    c.p.count_out = pool->count_out;
    c.stream = (hipStream_t)stream;
    return runtime_launch(c.stream, nullptr, do_step, &c, "paged_step");
}

int nnjit_kv_append_slots(const nnjit_paged_kv *cache, int64_t tokens, const int64_t *slots, const int32_t *positions,
                          const nnjit_rotary_table *rotary, const nnjit_head_norm *norm, const void *k, int64_t k_token, int64_t k_head,
                          const void *v, int64_t v_token, int64_t v_head, int64_t q_heads, const void *q, int64_t q_token, int64_t q_head,
                          void *q_out, int64_t qo_token, int64_t qo_head, int src_dtype, void *stream) {
    runtime_clear_error();
    int rc = check_cache(cache);
    if (rc != NNJIT_OK) return rc;
    if (!is_dtype(src_dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d", src_dtype);
    if (tokens < 0 || tokens > kMaxGroups) return runtime_fail(NNJIT_EINVAL, "tokens=%lld out of [0, 2^24)", (long long)tokens);
    if (q_heads < 0 || q_heads > kMaxHeads - 2 * cache->kv_heads)
        return runtime_fail(NNJIT_EINVAL, "q_heads=%lld out of [0, 2^30 - 2 kv_heads]", (long long)q_heads);
    const int64_t dim = cache->head_dim;
    if ((rc = check_slots("K", cache, cache->k_page, cache->k_token, cache->k_head)) != NNJIT_OK) return rc;
    if ((rc = check_slots("V", cache, cache->v_page, cache->v_token, cache->v_head)) != NNJIT_OK) return rc;
    if (norm && (rc = check_weight("q_weight", norm->q_weight, norm->q_head, norm->dtype, norm->eps, dim)) != NNJIT_OK) return rc;
    if (norm && (rc = check_weight("k_weight", norm->k_weight, norm->k_head, norm->dtype, norm->eps, dim)) != NNJIT_OK) return rc;
    if ((rc = check_turned(rotary, positions, tokens, dim)) != NNJIT_OK) return rc;
    if ((rc = check_rows("k", k, tokens, cache->kv_heads, k_token, k_head)) != NNJIT_OK) return rc;
    if ((rc = check_rows("v", v, tokens, cache->kv_heads, v_token, v_head)) != NNJIT_OK) return rc;
    if ((rc = check_rows("q", q, tokens, q_heads, q_token, q_head)) != NNJIT_OK) return rc;
    if ((rc = check_written("q_out", q_out, tokens, q_heads, dim, qo_token, qo_head)) != NNJIT_OK) return rc;
    if (tokens > 0 && !slots) return runtime_fail(NNJIT_EINVAL, "slots is NULL");
    if (tokens == 0) return NNJIT_OK;
    Call<NormParams> c;
    c.p.q = HeadRows{q, q_token, q_head};
    c.p.qo = HeadRows{q_out, qo_token, qo_head};
    c.p.q_heads = (int)q_heads;
    c.p.k = HeadRows{k, k_token, k_head};
    c.p.v = HeadRows{v, v_token, v_head};
    c.p.kv_heads = (int)cache->kv_heads;
    c.p.pool = pool_of(cache);
    c.p.slots = (const long long *)slots;
    set_rotary(c.p, rotary, positions);
    c.p.dim = (int)dim;
    c.p.tokens = (int)tokens;
    if (norm) {
        c.p.q_weight = norm->q_weight;
        c.p.k_weight = norm->k_weight;
        c.p.qw_head = norm->q_head;
        c.p.kw_head = norm->k_head;
        c.p.weight_half = norm->dtype == NNJIT_F16;
        c.p.eps = norm->eps;
    }
    c.append = true;
    c.vec = dim % 8 == 0 && c.p.rot % 8 == 0 && norm_in_units(c.p) && in_units(k, k_token, k_head, 4, src_dtype) && in_units(v, v_token, v_head, 4, src_dtype) &&
            (q_heads == 0 || (in_units(q, q_token, q_head, 4, src_dtype) && in_units(q_out, qo_token, qo_head, 4, cache->dtype))) &&
            pool_in_units(cache, 4);
    c.src = src_dtype;
    c.dst = cache->dtype;
    c.stream = (hipStream_t)stream;
    const Laid turned = laid(q_out, tokens, qo_token, q_heads, qo_head, dim, cache->dtype), rows = laid(q, tokens, q_token, q_heads, q_head, dim, src_dtype);
    if (!(same_place(rows, turned) || apart(rows, turned)) || !apart(laid(k, tokens, k_token, cache->kv_heads, k_head, dim, src_dtype), turned) ||
        !apart(laid(v, tokens, v_token, cache->kv_heads, v_head, dim, src_dtype), turned))
        c.refused = "q_out may be q with its strides and type, but not overlap it otherwise, nor k or v";
    return runtime_launch(c.stream, norm_refused, do_norm, &c, "kv_append_slots");
}

int nnjit_norm_rotary(const nnjit_rotary_table *rotary, int64_t tokens, int64_t heads, int64_t head_dim, const int32_t *positions,
                      const void *weight, int64_t w_head, int w_dtype, float eps, const void *x, int64_t x_token, int64_t x_head, int x_dtype,
                      void *y, int64_t y_token, int64_t y_head, int y_dtype, void *stream) {
    runtime_clear_error();
    if (!is_dtype(x_dtype) || !is_dtype(y_dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d to %d", x_dtype, y_dtype);
    int rc = check_norm_rows(rotary, tokens, heads, head_dim, positions, weight, w_head, w_dtype, eps, x, x_token, x_head);
    if (rc != NNJIT_OK) return rc;
    if ((rc = check_written("y", y, tokens, heads, head_dim, y_token, y_head)) != NNJIT_OK) return rc;
    if (tokens == 0 || heads == 0) return NNJIT_OK;
    Call<NormParams> c;
    c.p.q = HeadRows{x, x_token, x_head};
    c.p.qo = HeadRows{y, y_token, y_head};
    c.p.q_heads = (int)heads;
    set_rotary(c.p, rotary, positions);
    c.p.dim = (int)head_dim;
    c.p.tokens = (int)tokens;
    c.p.q_weight = weight;
    c.p.qw_head = w_head;
    c.p.weight_half = w_dtype == NNJIT_F16;
    c.p.eps = eps;
    c.vec = head_dim % 8 == 0 && c.p.rot % 8 == 0 && norm_in_units(c.p) && in_units(x, x_token, x_head, 4, x_dtype) && in_units(y, y_token, y_head, 4, y_dtype);
    c.src = x_dtype;
    c.dst = y_dtype;
    c.stream = (hipStream_t)stream;
    const Laid from = laid(x, tokens, x_token, heads, x_head, head_dim, x_dtype), to = laid(y, tokens, y_token, heads, y_head, head_dim, y_dtype);
    if (!same_place(from, to) && !apart(from, to)) c.refused = "y may be x with its strides and type, but not overlap it otherwise";
    return runtime_launch(c.stream, norm_refused, do_norm, &c, "norm_rotary");
}

int nnjit_norm_rotary_grad(const nnjit_rotary_table *rotary, int64_t tokens, int64_t heads, int64_t head_dim, const int32_t *positions,
                           const void *weight, int64_t w_head, int w_dtype, float eps, const void *x, int64_t x_token, int64_t x_head,
                           int x_dtype, const void *dy, int64_t dy_token, int64_t dy_head, int dy_dtype, void *dx, int64_t dx_token,
                           int64_t dx_head, float *dw, void *stream) {
    runtime_clear_error();
    if (!is_dtype(x_dtype) || !is_dtype(dy_dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d, %d", x_dtype, dy_dtype);
    int rc = check_norm_rows(rotary, tokens, heads, head_dim, positions, weight, w_head, w_dtype, eps, x, x_token, x_head);
    if (rc != NNJIT_OK) return rc;
    if ((rc = check_rows("dy", dy, tokens, heads, dy_token, dy_head)) != NNJIT_OK) return rc;
    if (dx && (rc = check_written("dx", dx, tokens, heads, head_dim, dx_token, dx_head)) != NNJIT_OK) return rc;
    if (dw && !weight) return runtime_fail(NNJIT_EINVAL, "weight is NULL");
    // (no rows: dx has none, the sum of dw is 0)
    if ((!dx && !dw) || ((tokens == 0 || heads == 0) && !dw) || (heads == 0 && w_head > 0)) return NNJIT_OK;
    if (tokens * heads > kMaxInt || (w_head > 0 && heads > 0xffff))
        return runtime_fail(NNJIT_EINVAL, "%lld rows of %lld heads in one call: below 2^31 rows (a weight a head: 2^16 heads) are served",
                            (long long)tokens, (long long)heads);
    if (dx) {
        const Laid to = laid(dx, tokens, dx_token, heads, dx_head, head_dim, x_dtype);
        for (const Laid &from : {laid(x, tokens, x_token, heads, x_head, head_dim, x_dtype), laid(dy, tokens, dy_token, heads, dy_head, head_dim, dy_dtype)})
            if (!same_place(from, to) && !apart(from, to))
                return runtime_fail(NNJIT_EINVAL, "dx may be x or dy with its strides and type, but not overlap them otherwise");
    }
    Call<NormParams> c;
    c.p.q = HeadRows{x, x_token, x_head};
    c.p.qo = HeadRows{dx, dx_token, dx_head};
    c.p.dy = HeadRows{dy, dy_token, dy_head};
    c.p.q_heads = (int)heads;
    set_rotary(c.p, rotary, positions);
    c.p.dim = (int)head_dim;
    c.p.tokens = (int)tokens;
    c.p.q_weight = weight;
    c.p.qw_head = w_head;
    c.p.weight_half = w_dtype == NNJIT_F16;
    c.p.eps = eps;
    c.p.dw = dw;
    c.vec = head_dim % 8 == 0 && c.p.rot % 8 == 0 && norm_in_units(c.p) && in_units(x, x_token, x_head, 4, x_dtype) && in_units(dy, dy_token, dy_head, 4, dy_dtype) &&
            (!dx || in_units(dx, dx_token, dx_head, 4, x_dtype));
    c.src = x_dtype;
    c.dst = dy_dtype;
    c.stream = (hipStream_t)stream;
    return runtime_launch(c.stream, norm_grad_floats, do_norm_grad, &c, "norm_rotary_grad");
}

int nnjit_kv_move(const nnjit_paged_kv *cache, const nnjit_paged_batch *batch, const int32_t *path, int64_t ld_path, int64_t path_len,
                  const int32_t *accepted, void *stream) {
    runtime_clear_error();
    int rc = check_cache(cache);
    if (rc != NNJIT_OK) return rc;
    if ((rc = check_batch(batch)) != NNJIT_OK) return rc;
    if ((rc = check_slots("K", cache, cache->k_page, cache->k_token, cache->k_head)) != NNJIT_OK) return rc;
    if ((rc = check_slots("V", cache, cache->v_page, cache->v_token, cache->v_head)) != NNJIT_OK) return rc;
    if (path_len < 0 || path_len > kMaxInt || ld_path < path_len)
        return runtime_fail(NNJIT_EINVAL, "path_len=%lld out of [0, 2^31) or ld_path=%lld below it", (long long)path_len, (long long)ld_path);
    if (batch->tokens == 0 || batch->sequences == 0 || path_len == 0) return NNJIT_OK;
    if (!path || !accepted) return runtime_fail(NNJIT_EINVAL, "path or accepted is NULL");
    if (batch->table_pages == 0) return NNJIT_OK;
    const int64_t elem = bytes_of(cache->dtype), row = cache->head_dim * elem;
    Call<MoveParams> c;
    c.unit = (int)elem;
    for (int64_t unit = 16; unit > elem; unit /= 2) {      // the widest piece that every offset and row is a multiple of
        if (row % unit || !pool_in_units(cache, unit / elem)) continue;
        c.unit = (int)unit;
        break;
    }
    const double threads = 2.0 * (double)cache->kv_heads * (double)(row / c.unit);
    if (batch->sequences > kMaxGroups || threads > 65535.0 * 16)
        return runtime_fail(NNJIT_EINVAL, "sequences=%lld (below 2^24) of rows of %lld heads (65535 workgroups of 16 pieces) are too many",
                            (long long)batch->sequences, (long long)cache->kv_heads);
    c.p.pool = pool_of(cache);
    c.p.batch = batch_of(batch);
    c.p.path = path;
    c.p.accepted = accepted;
    c.p.ld_path = ld_path;
    c.p.path_len = (int)path_len;
    c.p.kv_heads = (int)cache->kv_heads;
    c.p.row_bytes = (int)row;
    c.src = cache->dtype;
    c.stream = (hipStream_t)stream;
    return runtime_launch(c.stream, nullptr, do_move, &c, "kv_move");
}

int nnjit_adjust_logits(const nnjit_logit_rules *rules, int64_t rows, int64_t vocab, const void *x, int64_t ldx, int x_dtype, void *y,
                        int64_t ldy, int y_dtype, void *stream) {
    runtime_clear_error();
    if (!rules) return runtime_fail(NNJIT_EINVAL, "the rules are NULL");
    if (!is_dtype(x_dtype) || !is_dtype(y_dtype)) return runtime_fail(NNJIT_EDTYPE, "unsupported dtype %d to %d", x_dtype, y_dtype);
    if (rows < 0 || rows >= 1 << 20 || vocab < 0 || vocab >= 1 << 30)
        return runtime_fail(NNJIT_EINVAL, "rows=%lld out of [0, 2^20) or vocab=%lld out of [0, 2^30)", (long long)rows, (long long)vocab);
    if (ldx < 0 || ldy < 0 || (rows > 1 && ldy < vocab)) return runtime_fail(NNJIT_EINVAL, "rows of y overlap, or a stride is negative (ldx=%lld, ldy=%lld)", (long long)ldx, (long long)ldy);
    const nnjit_logit_rules &r = *rules;
    if (r.history && (r.history_len < 0 || r.history_len > kMaxInt || r.ld_history < 0))
        return runtime_fail(NNJIT_EINVAL, "history_len=%lld out of [0, 2^31) or a negative ld_history", (long long)r.history_len);
    if ((r.bias_token == nullptr) != (r.bias_value == nullptr)) return runtime_fail(NNJIT_EINVAL, "bias_token and bias_value go together");
    if (r.bias_token && (r.bias_len < 0 || r.bias_len > kMaxInt - 1 || r.ld_bias < 0))
        return runtime_fail(NNJIT_EINVAL, "bias_len=%lld out of [0, 2^31) or a negative ld_bias", (long long)r.bias_len);
    if (!r.history && r.history_len != 0) return runtime_fail(NNJIT_EINVAL, "history is NULL with history_len=%lld", (long long)r.history_len);
    if (r.mask && (r.ld_mask < 0 || r.mask_rows < 1 || r.mask_rows > kMaxInt))
        return runtime_fail(NNJIT_EINVAL, "mask_rows=%lld out of [1, 2^31) or a negative ld_mask", (long long)r.mask_rows);
    if (!r.mask && r.mask_row) return runtime_fail(NNJIT_EINVAL, "mask_row without mask");
    if (rows == 0 || vocab == 0) return NNJIT_OK;
    if (!x || !y) return runtime_fail(NNJIT_EINVAL, "x or y is NULL");
    const Laid from = laid(x, rows, ldx, 1, 0, vocab, x_dtype), to = laid(y, rows, ldy, 1, 0, vocab, y_dtype);
    if (!same_place(from, to) && !apart(from, to)) return runtime_fail(NNJIT_EINVAL, "y may be x with its stride and type, but not overlap it otherwise");
    if ((double)rows * (double)((vocab + 1023) / 1024) > (double)kMaxGroups)
        return runtime_fail(NNJIT_EINVAL, "%lld rows of %lld logits in one call: below 2^24 pieces of 1024 are served", (long long)rows, (long long)vocab);
    Call<LogitParams> c;
    c.p.history = r.history_len > 0 ? r.history : nullptr;
    c.p.length = r.length;
    c.p.prompt = r.prompt;
    c.p.ld_history = r.ld_history;
    c.p.history_len = (int)r.history_len;
    c.p.repetition = r.repetition;
    c.p.presence = r.presence;
    c.p.frequency = r.frequency;
    c.p.bias_token = r.bias_len > 0 ? r.bias_token : nullptr;
    c.p.bias_value = r.bias_value;
    c.p.ld_bias = r.ld_bias;
    c.p.bias_len = (int)r.bias_len;
    c.p.mask = r.mask;
    c.p.ld_mask = r.ld_mask;
    c.p.mask_rows = (int)r.mask_rows;
    c.p.mask_row = r.mask_row;
    c.p.rows = (int)rows;
    c.p.vocab = (int)vocab;
    c.p.x = x;
    c.p.y = y;
    c.p.ldx = ldx;
    c.p.ldy = ldy;
    c.src = x_dtype;
    c.dst = y_dtype;
    c.vec = in_units(x, ldx, 0, 4, x_dtype) && in_units(y, ldy, 0, 4, y_dtype);
    c.stream = (hipStream_t)stream;
    return runtime_launch(c.stream, nullptr, do_logits, &c, "adjust_logits");
}

}  // extern "C"
