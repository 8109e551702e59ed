// Internal declarations of the serving operators: rotary positions, appends
// to a paged cache, attention over it.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace nnjit {

// Largest head dimension of the serving operators.
constexpr int kMaxHeadDim = 256;
// Most keys of a sequence: max_kv is refused above, and later keys do not exist.
constexpr long long kMaxKeys = 1ll << 30;

// n / d for 0 <= n < 2^31 by one multiplication (d >= 1): with
// 2^(l-1) < d <= 2^l, l >= 1, and mul = ceil(2^(31+l) / d), which is below
// 2^32, the quotient is floor(n mul / 2^(31+l)) (Granlund and Montgomery,
// "Division by invariant integers using multiplication", 1994).  d = 1 takes n
// itself in the place of the product's upper half.
struct FastDiv {
    unsigned d, mul;
    int shift;                 // l - 1
    unsigned self;             // all ones for d = 1
    FastDiv() : FastDiv(1) {}
    explicit FastDiv(unsigned div) : d(div), mul(0), shift(0), self(~0u)
    {
        if (div == 1) return;
        int l = 1;
        while ((1ull << l) < div) ++l;
        mul = (unsigned)(((1ull << (31 + l)) + div - 1) / div);
        shift = l - 1;
        self = 0;
    }
    __host__ __device__ __forceinline__ int quot(int n) const
    {
        const unsigned upper = (unsigned)(((unsigned long long)(unsigned)n * mul) >> 32);
        return (int)((upper + ((unsigned)n & self)) >> shift);
    }
};

// One tensor of head rows: element (row, head, i) at p[row * tok + head * head + i].
struct HeadRows {
    const void *p;
    long long tok, head;
};

// The pool of pages: element (page, slot, head, i) of K at
// k[page * k_page + slot * k_tok + head * k_head + i], V alike.
struct PagePool {
    void *k, *v;
    unsigned k_page, k_tok, v_page, v_tok;   // below 2^32 elements; offsets are taken in 64 bits
    long long k_head, v_head;
    int pages;
    FastDiv page_size;
};

__device__ __forceinline__ long long page_offset(int page, unsigned page_stride, int slot, unsigned tok_stride)
{
    return (long long)((unsigned long long)(unsigned)page * page_stride + (unsigned long long)(unsigned)slot * tok_stride);
}

// The batch: device arrays as described in include/nnjit.h.
struct PageBatch {
    const int *q_start, *kv_len, *page_table;
    long long ld_table;
    int table_pages, sequences, tokens;
};

struct RotaryParams {
    HeadRows q, qo;            // rows turned to rows; heads 0 .. q_heads - 1
    int q_heads;
    HeadRows k, v;             // appended rows (kv_heads heads each; 0 without a cache)
    int kv_heads;
    PagePool pool;
    PageBatch batch;
    const int *positions;      // without a cache: the position of every row
    const float *table;        // NULL: nothing is turned
    int table_rows;
    int rot, dim, tokens;
    int interleaved;
    float sign;                // +1, or -1 for the transposed turn
    int heads_per_block;
};

hipError_t launch_rotary_table(float *table, int positions, int rot, double base, int scaling, double factor,
                               double original, double fast, double slow, double magnitude, hipStream_t stream);
// src_dtype, dst_dtype: NNJIT_F32 / NNJIT_F16; vec: rows can be taken four elements at a time.
hipError_t launch_rotary(const RotaryParams &p, bool append, int src_dtype, int dst_dtype, bool vec, hipStream_t stream);

struct AttentionParams {
    HeadRows q, o;
    int q_heads, group, dim;   // group: query heads of one key head
    FastDiv group_div;
    PagePool pool;
    PageBatch batch;
    float scale_log2;          // |scale| log2(e), finite and above 0, so that -inf stays -inf
    int negate;                // the scale is negative: queries are taken negated
    int causal, window;
    int row_tiles;             // row tiles of a sequence and key head
    int splits;                // workgroups along the keys
    int split_keys;            // keys of one split (a multiple of the key tile)
    int may_leave_out;         // splits are joined, and a sequence may have more rows than tiles
    int part_dim;              // dim rounded up to a multiple of 4
    float *part;               // splits > 1: [splits][tokens * q_heads][part_dim], not normalised
    float *stat;               // splits > 1: [splits][tokens * q_heads][2]: reference (attention_common.h), sum
    const void *zero;          // >= 64 bytes of zeros
};

// How one call is laid out on the chip; sizes the scratch.
struct AttentionPlan {
    int tile_rows;             // rows of a tile.  16: attention_rows.hip; 64, 128: attention_tiles.h
    int row_tiles, splits, split_keys;
    int waves;                 // waves of a workgroup of attention_rows.hip, 4 or 8
    int64_t ws_floats;         // partial sums and statistics
};
AttentionPlan attention_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t max_q,
                             int64_t max_kv, int causal, int64_t window, int cus);
hipError_t launch_attention_tiles_f16(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream);
hipError_t launch_attention_tiles_f32(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream);
hipError_t launch_attention(AttentionParams p, const AttentionPlan &plan, int dtype, bool vec, hipStream_t stream);

// Runtime services for entry points outside runtime.cpp.
int runtime_fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
void runtime_clear_error();
struct RuntimeDevice {
    float *ws;                 // the stream's scratch (NULL if none was asked for)
    const void *zero;          // 256 bytes of zeros
    int cus;
};
// Readies the current device, takes its stream's scratch and calls
// launch(ctx, device) under the library's lock; `floats` (may be NULL)
// returns how much scratch the launch needs on a device of so many CUs.
// Reports errors as the entry points do; lets no exception out.
int runtime_launch(hipStream_t stream, int64_t (*floats)(void *ctx, int cus), hipError_t (*launch)(void *ctx, const RuntimeDevice &),
                   void *ctx, const char *what);

}  // namespace nnjit
