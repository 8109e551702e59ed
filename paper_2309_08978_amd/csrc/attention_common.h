// Device-side helpers shared by the attention kernels.
#pragma once

#include "kcommon.h"
#include "serving.h"

namespace nnjit {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// What one workgroup works on: a tile of rows of one sequence and key head.
// Row r of the (sequence, key head) is query head (r % group) of new token
// r / group, so the query heads that share keys share a tile.
struct RowTile {
    int q0, new_tokens;   // first row of q, new tokens of the sequence
    int past;             // position of its first new token
    int keys;             // keys in the cache
    int r0, rows;         // first row of the tile, rows in it (<= 0: nothing to do)
    const int *table;     // the sequence's page table row

    __device__ __forceinline__ int first_key(const AttentionParams &p, int r) const
    {
        if (!p.causal || p.window == 0) return 0;
        return min(max(past + p.group_div.quot(r) - p.window + 1, 0), keys);
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
    const long long room = (long long)b.table_pages * p.pool.page_size.d;
    t.keys = (int)min((long long)max(b.kv_len[seq], 0), room);
    t.past = t.keys - t.new_tokens;
    t.r0 = tile * tile_rows;
    t.rows = min((long long)tile_rows, (long long)t.new_tokens * p.group - t.r0);
    t.table = b.page_table + (long long)seq * b.ld_table;
    return t;
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

template <typename T>
__device__ __forceinline__ T class_of(T v)
{
    return finite(v) ? (T)0 : v != v ? (T)kNan : v > (T)0 ? (T)kPosInf : (T)kNegInf;
}

__device__ __forceinline__ float add_classes(float sum, float counts)
{
    const int n = (int)counts;
    if (n == 0) return sum;
    const bool pos = n & 63, neg = (n >> 6) & 63, nan = n >= 4096;
    const float inf = __builtin_inff();
    return sum + ((nan || (pos && neg)) ? __builtin_nanf("") : pos ? inf : -inf);
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

}  // namespace nnjit
