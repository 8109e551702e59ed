// Device-side helpers shared by the attention kernels.
#pragma once

#include "kcommon.h"
#include "serving.h"

namespace nnjit {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
// memory that no one writes while the kernel runs: read by scalar loads
typedef __attribute__((address_space(4))) int constant_int;
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// What one workgroup works on: a tile of rows of one sequence and key head.
// Row r of the (sequence, key head) is query head (r % group) of new token
// r / group, so the query heads that share keys share a tile.
struct RowTile {
    int q0, new_tokens;   // first row of q, new tokens of the sequence
    int past;             // position of its first new token (below zero: it and maybe others see no key)
    int keys;             // keys in the cache
    int r0, rows;         // first row of the tile, rows in it (<= 0: nothing to do)
    const int *table;     // the sequence's page table row

    // (64 bits: a window of any size behind a position below zero)
    __device__ __forceinline__ int first_key(const AttentionParams &p, int r) const
    {
        if (!p.causal || p.window == 0) return 0;
        return (int)min(max((long long)past + p.group_div.quot(r) - p.window + 1, 0ll), (long long)keys);
    }
    __device__ __forceinline__ int end_key(const AttentionParams &p, int r) const
    {
        return p.causal ? min(keys, max(past + p.group_div.quot(r) + 1, 0)) : keys;
    }
};

__device__ __forceinline__ RowTile row_tile(const AttentionParams &p, int seq, int tile, int tile_rows)
{
    RowTile t;
    const PageBatch &b = p.batch;
    t.q0 = min(max(b.q_start[seq], 0), b.tokens);
    t.new_tokens = min(max(b.q_start[seq + 1] - t.q0, 0), b.tokens - t.q0);
    // (key indices stay well inside 32 bits, whatever kv_len holds)
    const long long room = min((long long)b.table_pages * p.pool.page_size.d, kMaxKeys);
    t.keys = (int)min((long long)max(b.kv_len[seq], 0), room);
    // positions follow kv_len as it stands, like those that an append turns and stores by: keys that
    // the table has no column for do not exist, but move no other key's position
    // (no position passes kv_len, so their sums stay in 32 bits)
    t.past = (int)max((long long)b.kv_len[seq] - ((long long)b.q_start[seq + 1] - t.q0), -0x7fffffffll);
    t.r0 = tile * tile_rows;
    t.rows = min((long long)tile_rows, (long long)t.new_tokens * p.group - t.r0);
    t.table = b.page_table + (long long)seq * b.ld_table;
    return t;
}

// Rows of the sequence behind the last tile (max_q was too small for it) are
// left alone; where splits are joined, the join has to be told: their
// reference in the first split is a NaN, which no row that was computed has.  By the
// THREADS threads of the last tile's first split, and only where the batch has more
// rows than the tiles of one sequence.
template <int THREADS>
__device__ __forceinline__ void mark_left_out(const AttentionParams &p, const RowTile &t, int head, int tile, int split, int tile_rows)
{
    if (!p.may_leave_out || split != 0 || tile != p.row_tiles - 1) return;
    const long long rows = (long long)t.new_tokens * p.group;
    for (long long r = (long long)p.row_tiles * tile_rows + threadIdx.x; r < rows; r += THREADS) {
        const int tok = p.group_div.quot((int)r);
        p.stat[((long long)(t.q0 + tok) * p.q_heads + head * p.group + (int)r - tok * p.group) * 2] = __builtin_nanf("");
    }
}

// A page id that can be read whatever the table holds.
__device__ __forceinline__ int safe_page(const AttentionParams &p, int id) { return min(max(id, 0), p.pool.pages - 1); }

// Values that are not finite in places that a row must not see.  A masked
// probability is 0, but 0 times an infinity or a NaN is a NaN, so in a key
// tile that some rows of a tile see only in part, values that are not finite
// are taken out of the product and what the rows that do see them get is
// added afterwards: their count by class, one matrix-core product of classes
// (1: +inf, 64: -inf, 4096: NaN) by visibility.  At most 32 keys a product:
// the three counts do not meet.
constexpr float kPosInf = 1.f, kNegInf = 64.f, kNan = 4096.f;

__device__ __forceinline__ bool finite(_Float16 v) { return (__builtin_bit_cast(unsigned short, v) & 0x7c00u) != 0x7c00u; }
__device__ __forceinline__ bool finite(float v) { return (__builtin_bit_cast(unsigned, v) & 0x7f800000u) != 0x7f800000u; }

// (by integer operations: no branches)
__device__ __forceinline__ _Float16 class_of(_Float16 v)
{
    const unsigned u = __builtin_bit_cast(unsigned short, v), size = u & 0x7fffu;
    const unsigned inf = u & 0x8000u ? 0x5400u : 0x3c00u;   // 64, 1
    return __builtin_bit_cast(_Float16, (unsigned short)(size > 0x7c00u ? 0x6c00u : size == 0x7c00u ? inf : 0u));
}

__device__ __forceinline__ float class_of(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v), size = u & 0x7fffffffu;
    const float inf = u & 0x80000000u ? kNegInf : kPosInf;
    return size > 0x7f800000u ? kNan : size == 0x7f800000u ? inf : 0.f;
}

__device__ __forceinline__ float add_classes(float sum, float counts)
{
    const unsigned n = (unsigned)counts;
    const unsigned pos = n & 63u, neg = n & 0xfc0u;
    unsigned add = pos ? 0x7f800000u : neg ? 0xff800000u : 0u;
    add = (pos && neg) || n >= 4096u ? 0x7fc00000u : add;
    return sum + __builtin_bit_cast(float, add);
}

// Elements col .. col + 7 of a row, zeros at and past `room`.
template <bool VEC>
__device__ __forceinline__ f32x8 load_eight(const float *row, int col, int room)
{
    f32x8 x = {};
    if constexpr (VEC) {
        f32x4 a = {}, b = {};
        if (col < room) a = *(const f32x4 *)(row + col);
        if (col + 4 < room) b = *(const f32x4 *)(row + col + 4);
        x = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        for (int i = 0; i < 8; ++i) x[i] = col + i < room ? row[col + i] : 0.f;
    }
    return x;
}

// Whether eight values are their bf16 parts' sums: finite, and none rounds to a bf16 infinity.
__device__ __forceinline__ bool splittable(f32x8 x)
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = x[i];
        top = max(top, __builtin_bit_cast(unsigned, v) & 0x7fffffffu);
    }
    return top < 0x7f7f8000u;
}

// Largest magnitude of halves, two at a time as integers (an infinity or NaN is
// the largest of all).
struct Largest16 {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
    template <typename V>
    __device__ __forceinline__ void take(V v)
    {
        typedef unsigned words __attribute__((ext_vector_type(sizeof(V) / 4)));
        const words w = __builtin_bit_cast(words, v);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(V) / 4); ++i) {
            const unsigned u = w[i] & 0x7fff7fffu;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, u));
        }
    }
    __device__ __forceinline__ bool finite() const { return top[0] < 0x7c00 && top[1] < 0x7c00; }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's weights are taken against its reference, about its largest logit so
// far.  As it moves from step to step, and from wave to wave and split to split
// when their sums are joined, weights and sums have to be taken against the very
// same value: a reference is kept as it was rounded.
//   fp32: a logit (tall tiles: plus a constant); a weight takes the difference first, so
//   it is off by a few roundings of its own exponent however large the logits are;
//   fp16: scaled, for one fma a weight (a difference first costs prompts 3 to 7% of
//   their time); what its rounding is off by is the same for all weights.  And
//   2^LIFT below the logit: fp16 weights lose bits below 2^-14, so that many more of the
//   small ones, which may be all of a result if the largest meets a value near zero,
//   keep theirs; it cancels in the division.  Rounded up by two to four units in the last
//   place: the weight of `top` must not pass 2^LIFT, nor that of a logit a rounded sum
//   above it what the sum says, where such a unit is worth more than fp16's room above.
template <bool HALF, int LIFT>
__device__ __forceinline__ float reference(const AttentionParams &p, float top)
{
    if (!HALF) return top;
    const float ref = fmaf(top, p.scale_log2, -(float)LIFT);
    return fmaf(fabsf(ref), 0x1p-22f, ref);               // (-inf gives a NaN, which no fmaxf() takes)
}

// ... as weights take it: 0 while the row has seen nothing (or only -inf), so
// that its weights are exp2(-inf) = 0
__device__ __forceinline__ float started(float ref) { return ref == -__builtin_inff() ? 0.f : ref; }

// Weight of the logit x.
template <bool HALF>
__device__ __forceinline__ float weight(const AttentionParams &p, float x, float ref)
{
    return exp2_fast(HALF ? fmaf(x, p.scale_log2, -ref) : (x - ref) * p.scale_log2);
}

// What sums against the reference `from` are multiplied by against `to`.
template <bool HALF>
__device__ __forceinline__ float moved(const AttentionParams &p, float from, float to)
{
    return exp2_fast(HALF ? from - to : (from - to) * p.scale_log2);
}

// Reference and sum of a row's split, as the join takes them.
// A sum that is a NaN stays one (weight exp2(inf - inf)); keys seen, but only
// logits of -inf: 0 / 0 unless another split has more.
__device__ __forceinline__ void store_stat(const AttentionParams &p, long long at, float ref, float sum, bool sees)
{
    p.stat[at * 2] = sum != sum ? __builtin_inff() : ref;
    p.stat[at * 2 + 1] = sees && sum == 0.f ? __builtin_nanf("") : sum;
}

}  // namespace nnjit
