// Attention over a paged cache for few rows (decode): tiles of 16 rows.
//
//   o[r] = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q_r . k_j - m)
//
// in one pass over the keys with a running reference m (attention_common.h) and sum.  A decode step
// reads every key and value once for a handful of multiplications each:
// bandwidth-bound, so the kernel keeps loads in flight and everything else in
// registers.
//
// Each wave takes key tiles of its own (KT keys: 32 in fp16, 16 in fp32) for
// all 16 rows and multiplies them on the matrix cores, straight from the
// registers that the loads fill, without LDS or barriers:
//
//   S^T = K Q^T   (16 keys x 16 rows a product: lane c = lane % 16 loads the
//                 16 bytes at chunk g = lane / 16 of key c, so lane (c, g)
//                 receives row c's logits of the keys 4 g + j, j = 0 .. 3)
//   O^T = V^T P^T (the probabilities are the second operand exactly as they
//                 lie: lane (c, g) holds row c, keys 4 g + j.  The first
//                 operand wants dims along c and the same keys: lane (c, g)
//                 loads the VE consecutive dims VE c .. of keys 4 g + j -- 16
//                 lanes read a whole value row -- and element e of them is
//                 the operand of product e, which gives dims VE m + e)
//
// so lane (c, g) ends up with 4 VE consecutive dims of row c, next to row c's
// maximum and sum: rescaling needs no exchange, the maximum two shuffles a
// tile.  In fp16 the eight keys of an operand are gathered from eight loaded
// vectors by byte permutes.  Weights go into the products in two fp16 parts (p =
// hi + lo: matrix cores have nothing else to do here) and are up to 2^15: they are
// held to 22 bits, or to 2^-40 of the row's largest.
//
// The waves of a workgroup are joined through LDS at the end.  Keys are split
// over workgroups where sequences and key heads alone leave the chip idle; a
// second kernel joins the splits in their order, so results do not depend on
// which workgroup finishes first.  (The last workgroup of a row could join
// them without a second launch, but its fences across the XCDs' caches cost
// as much once many workgroups take part.)
//
// Measured, heads of 128 in fp16, with the join: 32 ragged sequences of up to
// 4096 keys, 32 query heads on 8 key heads: 71 us, 4.3 TB/s of keys and values
// (with the join of eight splits); one sequence of 65536 keys: 61 us, 4.4 TB/s (55 + 6); both wait
// for memory (matrix cores busy 4% of the time).  One sequence of 1023 keys,
// 32 heads: 11.6 us, of which two launches are 5.
#pragma once

#include "attention_common.h"

namespace nnjit {

namespace {

constexpr int kLiftRows = 15;                 // fp16 weights are at most 2^15 (the largest half: 2^16)

template <typename T> struct RowsOf;
template <> struct RowsOf<_Float16> {
    static constexpr int KT = 32;               // keys of a wave's tile
    static constexpr int CH = 8;                // elements of a 16-byte chunk
    typedef f16x8 chunk;
};
template <> struct RowsOf<float> {
    static constexpr int KT = 16;
    static constexpr int CH = 4;
    typedef f32x4 chunk;
};

// n consecutive elements, of which those at or past `valid` are zero.  STREAM: not
// to be kept in the caches.
template <typename V, bool VEC, bool STREAM, typename T>
__device__ __forceinline__ V load_some(const T *src, int valid, int n)
{
    if constexpr (VEC) {
        V v = {};
        if (valid > 0) {                        // valid is a multiple of n here
            if constexpr (STREAM) v = __builtin_nontemporal_load((const V *)src);
            else v = *(const V *)src;
        }
        return v;
    } else {
        V v;
        for (int i = 0; i < n; ++i) v[i] = i < valid ? src[i] : (T)0;
        return v;
    }
}

// STREAM: keys and values pass the caches by, where nothing of a cache line is
// read twice: one row tile, heads of whole lines (32 sequences of 4096 keys, heads
// of 128: 110 -> 102 us; two row tiles would lose, 39 -> 46, as would heads of 96
// dims, 22 -> 27, and of 64, whose loads take half a line, 24 -> 27).
// TREE: drafted trees: a row sees its sequence's cached keys (with a window from
// first_cached() on) and the new tokens that its mask names.  Only tiles of keys that hold new
// tokens look at masks.  24 nodes behind 1000 keys, 12 heads of 64 in fp32: 7.8 us and 4.4 for
// the join.
template <typename T, int DP, bool VEC, bool PAGE16, bool STREAM, int NW, bool TREE>
__global__ void __launch_bounds__(NW * 64)
attention_rows_kernel(AttentionParams p)
{
    typedef RowsOf<T> R;
    constexpr bool HALF = sizeof(T) == 2;
    constexpr int KT = R::KT, CH = R::CH, SUB = KT / 16;
    typedef typename R::chunk chunk;
    constexpr int STEPS = DP / (4 * CH);                  // chunks of a key per lane
    constexpr int VE = DP / 16 < CH ? DP / 16 : CH;       // dims of a value vector
    constexpr int VH = DP / (16 * VE);                    // value vectors of a key per lane
    constexpr int BLK = DP / 16;                          // products (of 16 dims) of a tile
    typedef T vvec __attribute__((ext_vector_type(VE)));

    __shared__ __attribute__((aligned(16))) float lds_o[NW][16][DP + 4];
    __shared__ float lds_m[NW][16], lds_l[NW][16];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;

    // row tiles of one sequence and key head run on one XCD; with one row tile nothing
    // is shared, and the (split, sequence) pairs go round the XCDs, each with all its
    // heads, a sequence's splits to different XCDs: sequences of random lengths
    // 2% (fp16) and 4% (fp32) faster than with neighbours on one XCD, up to 28% (three
    // of up to 10000 keys, 32 heads of 128: 166 -> 119 us); equal ones 0 .. 2% slower.
    // (A head a XCD would leave most channels of its L2 idle: its rows lie 2 KB apart.)
    const int kv_heads = p.q_heads / p.group;
    int tile = 0, split, head, seq;
    if (p.row_tiles == 1 && p.splits > 1 && p.batch.sequences > 1) {
        const int b = blockIdx.x, n = p.batch.sequences, size = 8 * kv_heads, round = b / size, whole = gridDim.x - gridDim.x % size;
        const int pair = round * 8 + (b % 8 + (n < 8 ? round : round * 8 / n)) % 8;
        int id = b < whole ? pair * kv_heads + b % size / 8 : whole + xcd_remap(b - whole, gridDim.x - whole);
        head = id % kv_heads;
        id /= kv_heads;
        seq = id % n;
        split = id / n;
    } else {
        int id = xcd_remap(blockIdx.x, gridDim.x);
        tile = id % p.row_tiles;
        id /= p.row_tiles;
        split = id % p.splits;
        id /= p.splits;
        head = id % kv_heads;
        seq = id / kv_heads;
    }
    const RowTile t = row_tile(p, seq, tile, 16);
    if (t.rows <= 0) return;
    mark_left_out<NW * 64>(p, t, head, tile, split, 16);

    // keys of the tile's rows, and of this split
    const int r_last = t.r0 + t.rows - 1;
    const int lo_min = TREE ? t.first_cached(p, 0) : t.first_key(p, t.r0);
    const int lo_max = TREE ? t.first_cached(p, t.new_tokens - 1) : t.first_key(p, r_last);
    const int hi_min = TREE ? t.cached : t.end_key(p, t.r0), hi_max = TREE ? t.keys : t.end_key(p, r_last);
    const int base = lo_min & ~31;
    const long long begin = base + (long long)split * p.split_keys;
    const int k0 = (int)min(begin, (long long)hi_max);
    // (trees: the last split goes to the end, for sequences of more new tokens than max_q)
    const int k1 = TREE && split == p.splits - 1 ? hi_max : (int)min(begin + p.split_keys, (long long)hi_max);
    const bool rows_differ = TREE || lo_min != lo_max || hi_min != hi_max;

    // this lane's row (rows past the tile's repeat its last one; not stored)
    const int r = min(t.r0 + c, r_last);
    const int token = t.q0 + p.group_div.quot(r);
    const int q_head = head * p.group + r - p.group_div.quot(r) * p.group;
    const int lo = max(TREE ? t.first_cached_of(p, token) : t.first_key(p, r), k0), hi = min(TREE ? t.cached : t.end_key(p, r), k1);

    chunk q[STEPS];
    {
        const T *src = (const T *)p.q.p + (long long)token * p.q.tok + (long long)q_head * p.q.head;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int d = (4 * s + g) * CH;
            q[s] = load_some<chunk, VEC, false>(src + d, p.dim - d, CH);
            if (p.negate) q[s] = -q[s];
        }
    }

    const T *kp = (const T *)p.pool.k + (long long)head * p.pool.k_head;
    const T *vp = (const T *)p.pool.v + (long long)head * p.pool.v_head;
    const int page_size = p.pool.page_size.d;
    const int last_key = max(hi_max - 1, 0);

    // page ids of a tile's keys: per 16 keys where pages hold multiples of 16
    // (one scalar load each), else for the keys that the lane loads
    constexpr int IDS_K = SUB, IDS_V = PAGE16 ? 0 : SUB * 4;
    struct Ids {
        int k[IDS_K], v[IDS_V > 0 ? IDS_V : 1];
    };
    auto ids_of = [&](int kt) {
        Ids ids;
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const int at = p.pool.page_size.quot(min(kt + 16 * s + (PAGE16 ? 0 : c), last_key));
            if constexpr (PAGE16) ids.k[s] = ((const constant_int *)t.table)[__builtin_amdgcn_readfirstlane(at)];
            else ids.k[s] = t.table[at];
        }
        if constexpr (!PAGE16) {
#pragma unroll
            for (int i = 0; i < SUB * 4; ++i) {
                const int key = min(kt + 16 * (i / 4) + 4 * g + i % 4, last_key);
                ids.v[i] = t.table[p.pool.page_size.quot(key)];
            }
        }
        return ids;
    };
    // slot of a key; keys past the last one are read at some slot of the last
    // page (PAGE16) or as the last key, and masked
    auto slot_of = [&](int sub_key, int within) {
        if constexpr (PAGE16) return sub_key - p.pool.page_size.quot(sub_key) * page_size + within;
        const int key = min(sub_key + within, last_key);
        return key - p.pool.page_size.quot(key) * page_size;
    };

    chunk kreg[SUB][STEPS];
    vvec vreg[SUB * 4][VH];
    auto load_k = [&](const Ids &ids, int kt) {
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const T *row = kp + page_offset(safe_page(p, ids.k[s]), p.pool.k_page, slot_of(kt + 16 * s, c), p.pool.k_tok);
#pragma unroll
            for (int e = 0; e < STEPS; ++e) {
                const int d = (4 * e + g) * CH;
                kreg[s][e] = load_some<chunk, VEC, STREAM>(row + d, p.dim - d, CH);
            }
        }
    };
    auto load_v = [&](const Ids &ids, int kt) {
#pragma unroll
        for (int i = 0; i < SUB * 4; ++i) {
            const int s = i / 4;
            const T *row = vp + page_offset(safe_page(p, PAGE16 ? ids.k[s] : ids.v[i]), p.pool.v_page,
                                            slot_of(kt + 16 * s, 4 * g + i % 4), p.pool.v_tok);
#pragma unroll
            for (int h = 0; h < VH; ++h) {
                const int d = h * 16 * VE + c * VE;
                vreg[i][h] = load_some<vvec, VEC, STREAM>(row + d, p.dim - d, VE);
            }
        }
    };

    f32x4 acc[BLK];
#pragma unroll
    for (int b = 0; b < BLK; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ref = -__builtin_inff(), l = 0.f;

    const int tiles = (k1 - k0 + KT - 1) / KT;
    Ids ids;
    if (wave < tiles) {
        ids = ids_of(k0 + wave * KT);
        const Ids now = ids;
        load_k(now, k0 + wave * KT);
        ids = ids_of(k0 + (wave + NW) * KT);
        load_v(now, k0 + wave * KT);
    }
    for (int it = wave; it < tiles; it += NW) {
        const int kt = k0 + it * KT;
        const int kn = kt + NW * KT;
        const bool more = it + NW < tiles;
        // fp32: a logit is summed in four parts: one chain over all dims rounds twice as
        // much off (heads of 64, 500 keys: results off by 5.3e-7, in four parts by 2.7e-7)
        constexpr int CHAINS = HALF ? 1 : 4;
        f32x4 x[SUB];
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            f32x4 sum[CHAINS] = {};
#pragma unroll
            for (int e = 0; e < STEPS; ++e) {
                if constexpr (HALF) {
                    sum[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kreg[s][e], q[e], sum[0], 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kreg[s][e][i], q[e][i], sum[i], 0, 0, 0);
                }
            }
            if constexpr (HALF) x[s] = sum[0];
            else x[s] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        // the look-ups of the tile after the next are asked for between its keys and its values:
        // loads come in order, and theirs must not wait for the values
        const Ids now = ids;
        if (more) {
            load_k(now, kn);
            ids = ids_of(kn + NW * KT);
        }

        const bool whole = kt >= lo_max && kt + KT <= min(hi_min, k1);
        unsigned seen = ~0u;
        if (!whole) {
            seen = 0;
            [[maybe_unused]] unsigned drafted = 0;
#pragma unroll
            for (int i = 0; i < SUB * 4; ++i) {
                const int key = kt + 16 * (i / 4) + 4 * g + i % 4;
                bool see = key >= lo && key < hi;
                if constexpr (TREE) {
                    if (i % 4 == 0) drafted = t.drafted4(p, token, key);
                    see |= key >= t.cached && key < k1 && (drafted >> i % 4 & 1);
                }
                x[i / 4][i % 4] = see ? x[i / 4][i % 4] : -__builtin_inff();
                seen |= see ? 1u << i : 0u;
                // keys that no row of the tile sees: whatever lies there
                const bool any = key >= max(lo_min, k0) && key < k1;
#pragma unroll
                for (int h = 0; h < VH; ++h)
#pragma unroll
                    for (int e = 0; e < VE; ++e) vreg[i][h][e] = any ? vreg[i][h][e] : (T)0;
            }
        }

        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < SUB * 4; ++i) top = fmaxf(top, x[i / 4][i % 4]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float next = fmaxf(ref, reference<HALF, kLiftRows>(p, top)), off = started(next);
        const float shrink = moved<HALF>(p, ref, off);
        ref = next;
        float pr[SUB * 4], sum = 0.f;
#pragma unroll
        for (int i = 0; i < SUB * 4; ++i) {
            pr[i] = weight<HALF>(p, x[i / 4][i % 4], off);
            sum += pr[i];
        }
        l = l * shrink + sum;
#pragma unroll
        for (int b = 0; b < BLK; ++b) acc[b] *= shrink;

        if constexpr (HALF) {
            // an infinity times the second part of a probability, which may be zero or
            // negative, is a NaN: a tile with values that are not finite is taken carefully
            Largest16 largest;
#pragma unroll
            for (int i = 0; i < SUB * 4; ++i)
#pragma unroll
                for (int h = 0; h < VH; ++h) largest.take(vreg[i][h]);
            const bool careful = __any(!largest.finite());
            f16x8 hi8, lo8, vis8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                hi8[i] = (_Float16)pr[i];
                lo8[i] = (_Float16)(pr[i] - (float)hi8[i]);
                vis8[i] = (_Float16)((seen >> i & 1) ? 1.f : 0.f);
            }
#pragma unroll
            for (int b = 0; b < BLK; ++b) {
                f16x8 v;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = vreg[i][b / VE][b % VE];
                if (careful) {
                    f16x8 cls;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        cls[i] = class_of(v[i]);
                        v[i] = finite(v[i]) ? v[i] : (_Float16)0.f;
                    }
                    const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_f16(cls, vis8, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[b][j] = add_classes(acc[b][j], n[j]);
                }
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, hi8, acc[b], 0, 0, 0);
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, lo8, acc[b], 0, 0, 0);
            }
        } else {
            const bool careful = !whole && rows_differ;
#pragma unroll
            for (int b = 0; b < BLK; ++b) {
                float v[4];
                bool bad = false;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = vreg[j][b / VE][b % VE];
                    bad |= !finite(v[j]);
                }
                if (careful && __any(bad)) {
                    f32x4 n = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        n = __builtin_amdgcn_mfma_f32_16x16x4f32(class_of(v[j]), (seen >> j & 1) ? 1.f : 0.f, n, 0, 0, 0);
                        v[j] = finite(v[j]) ? v[j] : 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[b][j] = add_classes(acc[b][j], n[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], pr[j], acc[b], 0, 0, 0);
            }
        }
        if (more) load_v(now, kn);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // join the waves: their sums against the largest reference
    if (g == 0) {
        lds_m[wave][c] = ref;
        lds_l[wave][c] = l;
    }
    if (c < t.rows) {
#pragma unroll
        for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < VE; ++e) lds_o[wave][c][h * 16 * VE + (4 * g + j) * VE + e] = acc[h * VE + e][j];
    }
    __syncthreads();
    const int dim = p.dim;
    constexpr int QUADS = DP / 4;
    for (int i = threadIdx.x; i < t.rows * QUADS; i += NW * 64) {
        const int row = i / QUADS, d = (i % QUADS) * 4;
        if (d >= dim) continue;
        float most = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < NW; ++w) most = fmaxf(most, lds_m[w][row]);
        const float off = started(most);
        float total = 0.f;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float part = moved<HALF>(p, lds_m[w][row], off);
            total += part * lds_l[w][row];
            o += part * *(const f32x4 *)&lds_o[w][row][d];
        }
        const int rr = t.r0 + row, tok = p.group_div.quot(rr);
        const int oh = head * p.group + rr - tok * p.group;
        const bool sees = TREE ? t.drafted_any(p, t.q0 + tok, k0, k1) : min(t.end_key(p, rr), k1) > max(t.first_key(p, rr), k0);
        if (p.splits == 1) {
            // a row without a key is 0; one whose logits are all -inf is 0 / 0
            T *dst = (T *)p.o.p + (long long)(t.q0 + tok) * p.o.tok + (long long)oh * p.o.head + d;
            typedef T quad __attribute__((ext_vector_type(4)));
            quad out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = (T)(sees ? o[e] / total : 0.f);
            if constexpr (VEC) {
                *(quad *)dst = out;
            } else {
                for (int e = 0; e < 4 && d + e < dim; ++e) dst[e] = out[e];
            }
        } else {
            const long long at = ((long long)split * p.batch.tokens + t.q0 + tok) * p.q_heads + oh;
            *(f32x4 *)(p.part + at * p.part_dim + d) = o;
            if (d == 0) store_stat(p, at, most, total, sees);
        }
    }
}

template <typename T, int DP, bool VEC, bool STREAM, bool TREE, int NW>
hipError_t launch_paged(const AttentionParams &p, int grid, hipStream_t stream)
{
    if (p.pool.page_size.d % 16 == 0) attention_rows_kernel<T, DP, VEC, true, STREAM, NW, TREE><<<grid, NW * 64, 0, stream>>>(p);
    else attention_rows_kernel<T, DP, VEC, false, STREAM, NW, TREE><<<grid, NW * 64, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T, int DP, bool VEC, bool STREAM, bool TREE>
hipError_t launch_waves(const AttentionParams &p, int waves, int grid, hipStream_t stream)
{
    if constexpr (VEC && DP <= 128) {
        if (waves == 8) return launch_paged<T, DP, VEC, STREAM, TREE, 8>(p, grid, stream);
    }
    return launch_paged<T, DP, VEC, STREAM, TREE, 4>(p, grid, stream);
}

template <typename T, int DP, bool VEC, bool TREE>
hipError_t launch_rows(const AttentionParams &p, int waves, int grid, hipStream_t stream)
{
    if constexpr (VEC && DP >= 128) {
        if (p.dim == DP && p.row_tiles == 1) return launch_waves<T, DP, VEC, true, TREE>(p, waves, grid, stream);
    }
    return launch_waves<T, DP, VEC, false, TREE>(p, waves, grid, stream);
}

template <typename T, bool TREE>
hipError_t launch_typed(const AttentionParams &p, bool vec, int waves, int grid, hipStream_t stream)
{
    if (!vec) return p.dim <= 128 ? launch_rows<T, 128, false, TREE>(p, waves, grid, stream) : launch_rows<T, 256, false, TREE>(p, waves, grid, stream);
    if (p.dim <= 64) return launch_rows<T, 64, true, TREE>(p, waves, grid, stream);
    if (p.dim <= 128) return launch_rows<T, 128, true, TREE>(p, waves, grid, stream);
    return launch_rows<T, 256, true, TREE>(p, waves, grid, stream);
}

}  // namespace

}  // namespace nnjit
