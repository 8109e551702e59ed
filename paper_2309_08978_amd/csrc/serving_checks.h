// Argument checks of the serving entry points, and their parameters from the
// descriptions of include/nnjit.h.
#pragma once

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

// Where rows lie: n0 by n1 runs of `width` bytes, s0 and s1 bytes apart.
struct Laid {
    const void *p;
    int64_t n0, s0, n1, s1, width;
    int dtype;
};

Laid laid(const void *p, int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t dim, int dtype) {
    const int64_t e = bytes_of(dtype);
    return Laid{p, rows, row * e, heads, head * e, dim * e, dtype};
}

// the very same elements, each at its own place
bool same_place(const Laid &a, const Laid &b) {
    return a.p == b.p && a.dtype == b.dtype && a.n0 == b.n0 && a.n1 == b.n1 && a.width == b.width && (a.n0 < 2 || a.s0 == b.s0) && (a.n1 < 2 || a.s1 == b.s1);
}

// No byte of a is one of b: by their ends, or because both repeat with a period within which their
// runs lie apart, as column ranges of one tensor do.  (Says no of runs that mesh over several periods.)
bool apart(const Laid &a, const Laid &b) {
    typedef __int128 wide;
    if (a.n0 < 1 || a.n1 < 1 || b.n0 < 1 || b.n1 < 1 || a.width < 1 || b.width < 1) return true;
    const wide pa = (wide)(uintptr_t)a.p, pb = (wide)(uintptr_t)b.p;
    // what is left of the runs once whole periods (0: none) are taken off: n runs, s apart; false: still two axes of them
    struct Runs {
        wide n, s, width, end;
    };
    const auto runs_of = [](const Laid &l, int64_t period, Runs &r) {
        const bool more0 = l.n0 > 1 && !(period && l.s0 % period == 0), more1 = l.n1 > 1 && !(period && l.s1 % period == 0);
        r = Runs{more0 ? l.n0 : more1 ? l.n1 : 1, more0 ? l.s0 : l.s1, l.width, 0};
        r.end = (more0 ? (wide)(l.n0 - 1) * l.s0 : 0) + (more1 ? (wide)(l.n1 - 1) * l.s1 : 0) + l.width;
        return !(more0 && more1);
    };
    Runs ra, rb;
    runs_of(a, 0, ra);
    runs_of(b, 0, rb);
    if (pa + ra.end <= pb || pb + rb.end <= pa) return true;
    const int64_t periods[4] = {a.n0 > 1 ? a.s0 : 0, a.n1 > 1 ? a.s1 : 0, b.n0 > 1 ? b.s0 : 0, b.n1 > 1 ? b.s1 : 0};
    // both within one period, b's runs beginning `from` behind a's
    const auto lie_apart = [](const Runs &a, const Runs &b, wide from, wide period, bool lines) {
        if (a.end > period || from + b.end > period) return false;
        if (a.end <= from) return true;
        if (!lines || a.n > 4096) return false;
        for (wide i = 0; i < a.n; ++i) {
            const wide x = i * a.s - from;                               // a's run i, as seen from b's first
            // the first of b's runs that ends behind x: does it begin before x + width?
            const wide j = x < b.width ? 0 : b.s > 0 ? (x - b.width) / b.s + 1 : b.n;
            if (j < b.n && j * b.s < x + a.width) return false;
        }
        return true;
    };
    for (const int64_t period : periods) {
        if (period <= 0) continue;
        const bool lines = runs_of(a, period, ra) & runs_of(b, period, rb);
        const wide from = ((pb - pa) % period + period) % period;
        if (lie_apart(ra, rb, from, period, lines) || lie_apart(rb, ra, (period - from) % period, period, lines)) return true;
    }
    return false;
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

}  // namespace
}  // namespace nnjit
