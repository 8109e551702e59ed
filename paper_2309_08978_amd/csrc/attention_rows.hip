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
#include <algorithm>
#include <cmath>

#include "attention_common.h"
#include "nnjit.h"

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
template <typename T, int DP, bool VEC, bool PAGE16, bool STREAM, int NW>
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
    const int lo_min = t.first_key(p, t.r0), lo_max = t.first_key(p, r_last);
    const int hi_min = t.end_key(p, t.r0), hi_max = t.end_key(p, r_last);
    const int base = lo_min & ~31;
    const long long begin = base + (long long)split * p.split_keys;
    const int k0 = (int)min(begin, (long long)hi_max);
    const int k1 = (int)min(begin + p.split_keys, (long long)hi_max);
    const bool rows_differ = lo_min != lo_max || hi_min != hi_max;

    // this lane's row (rows past the tile's repeat its last one; not stored)
    const int r = min(t.r0 + c, r_last);
    const int token = t.q0 + p.group_div.quot(r);
    const int q_head = head * p.group + r - p.group_div.quot(r) * p.group;
    const int lo = max(t.first_key(p, r), k0), hi = min(t.end_key(p, r), k1);

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
#pragma unroll
            for (int i = 0; i < SUB * 4; ++i) {
                const int key = kt + 16 * (i / 4) + 4 * g + i % 4;
                const bool see = key >= lo && key < hi;
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
        const bool sees = min(t.end_key(p, rr), k1) > max(t.first_key(p, rr), k0);
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

// Joins the splits of every row: o = sum_s w_s o_s / sum_s w_s l_s, w_s = exp(scale (m_s - M))
// for the references m_s and the largest of them, M.
// A group of LPR lanes takes four dims a lane of one row; GPR groups of a
// workgroup share a row, group i the splits i, i + GPR, ..., added in order:
// 1 where rows fill the chip by themselves, else all groups of the workgroup,
// so that a decode step's few rows of many splits are read in parallel.
template <typename T, int LPR, int GPR>
__global__ void __launch_bounds__(256)
attention_join_kernel(AttentionParams p)
{
    constexpr bool HALF = sizeof(T) == 2;
    constexpr int GROUPS = 256 / LPR, ROWS = GROUPS / GPR;
    __shared__ f32x4 lds_o[GPR > 1 ? GROUPS : 1][LPR];
    __shared__ float lds_l[GROUPS];
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    const long long rows = (long long)p.batch.tokens * p.q_heads;
    const long long row = (long long)blockIdx.x * ROWS + group / GPR;
    const int token = (int)(row / p.q_heads), head = (int)(row % p.q_heads);
    const bool live = row < rows && token >= p.batch.q_start[0] && token < p.batch.q_start[p.batch.sequences];

    float most = -__builtin_inff(), total = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    int marks = 0;                                             // 1: 0 / 0, 2: left out (mark_left_out)
    if (live) {
        // the largest reference: a lane per split
        for (int s = lane; s < p.splits; s += LPR) {
            const f32x2 st = *(const f32x2 *)(p.stat + (s * rows + row) * 2);
            most = fmaxf(most, st[0]);
            marks |= (st[1] != st[1] ? 1 : 0) | (st[0] != st[0] ? 2 : 0);
        }
    }
#pragma unroll
    for (int i = 1; i < LPR; i <<= 1) {
        most = fmaxf(most, __shfl_xor(most, i));
        marks |= __shfl_xor(marks, i);
    }
    if (live) {
        const float off = started(most);
        const int d = min(4 * lane, p.part_dim - 4);
#pragma unroll 8
        for (int s = group % GPR; s < p.splits; s += GPR) {
            const long long at = s * rows + row;
            const f32x2 st = *(const f32x2 *)(p.stat + at * 2);
            const f32x4 part = *(const f32x4 *)(p.part + at * p.part_dim + d);
            const bool seen = st[0] != -__builtin_inff();          // else it has seen nothing, or only -inf
            const float w = moved<HALF>(p, st[0], off);
            total += seen ? w * st[1] : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += seen ? w * part[e] : 0.f;
        }
    }
    if constexpr (GPR > 1) {
        lds_o[group][lane] = o;
        if (lane == 0) lds_l[group] = total;
        __syncthreads();
        if (group % GPR != 0) return;
        o = f32x4{0.f, 0.f, 0.f, 0.f};
        total = 0.f;
        for (int g = 0; g < GPR; ++g) {
            o += lds_o[group + g][lane];
            total += lds_l[group + g];
        }
    }
    if (!live || (marks & 2)) return;
    const bool empty = most == -__builtin_inff();
    T *dst = (T *)p.o.p + (long long)token * p.o.tok + (long long)head * p.o.head + 4 * lane;
    for (int e = 0; e < 4; ++e)
        if (4 * lane + e < p.dim) dst[e] = (T)(empty ? ((marks & 1) ? __builtin_nanf("") : 0.f) : o[e] / total);
}

template <typename T>
hipError_t launch_join(const AttentionParams &p, hipStream_t stream)
{
    const long long rows = (long long)p.batch.tokens * p.q_heads;
    // below four rows a compute unit, a workgroup a row
    const bool few = rows < 1024;
    auto grid = [&](int per) { return (unsigned)((rows + per - 1) / per); };
    if (p.dim <= 64) {
        if (few) attention_join_kernel<T, 16, 16><<<grid(1), 256, 0, stream>>>(p);
        else attention_join_kernel<T, 16, 1><<<grid(16), 256, 0, stream>>>(p);
    } else if (p.dim <= 128) {
        if (few) attention_join_kernel<T, 32, 8><<<grid(1), 256, 0, stream>>>(p);
        else attention_join_kernel<T, 32, 1><<<grid(8), 256, 0, stream>>>(p);
    } else {
        if (few) attention_join_kernel<T, 64, 4><<<grid(1), 256, 0, stream>>>(p);
        else attention_join_kernel<T, 64, 1><<<grid(4), 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

template <typename T, int DP, bool VEC, bool STREAM, int NW>
hipError_t launch_paged(const AttentionParams &p, int grid, hipStream_t stream)
{
    if (p.pool.page_size.d % 16 == 0) attention_rows_kernel<T, DP, VEC, true, STREAM, NW><<<grid, NW * 64, 0, stream>>>(p);
    else attention_rows_kernel<T, DP, VEC, false, STREAM, NW><<<grid, NW * 64, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T, int DP, bool VEC, bool STREAM>
hipError_t launch_waves(const AttentionParams &p, int waves, int grid, hipStream_t stream)
{
    if constexpr (VEC && DP <= 128) {
        if (waves == 8) return launch_paged<T, DP, VEC, STREAM, 8>(p, grid, stream);
    }
    return launch_paged<T, DP, VEC, STREAM, 4>(p, grid, stream);
}

template <typename T, int DP, bool VEC>
hipError_t launch_rows(const AttentionParams &p, int waves, int grid, hipStream_t stream)
{
    if constexpr (VEC && DP >= 128) {
        if (p.dim == DP && p.row_tiles == 1) return launch_waves<T, DP, VEC, true>(p, waves, grid, stream);
    }
    return launch_waves<T, DP, VEC, false>(p, waves, grid, stream);
}

template <typename T>
hipError_t launch_typed(const AttentionParams &p, bool vec, int waves, int grid, hipStream_t stream)
{
    if (!vec) return p.dim <= 128 ? launch_rows<T, 128, false>(p, waves, grid, stream) : launch_rows<T, 256, false>(p, waves, grid, stream);
    if (p.dim <= 64) return launch_rows<T, 64, true>(p, waves, grid, stream);
    if (p.dim <= 128) return launch_rows<T, 128, true>(p, waves, grid, stream);
    return launch_rows<T, 256, true>(p, waves, grid, stream);
}

// Keys that one tile can see: with a window, from the first row's first key
// (rounded down to a multiple of 32) to the last row's last.
int64_t seen_span(int64_t max_kv, int64_t window, int tile_rows, int64_t group)
{
    return window > 0 ? std::min(max_kv, window + (tile_rows + group - 1) / group + 32) : max_kv;
}

// Up to 16 rows of a sequence and key head: chosen are the splits and the waves of a
// workgroup.  Estimated time (us, d = head dim / 128): steps of a split times the
// largest of a step's latency, its share of a compute unit's cores (a unit of four
// waves) and its bytes at 6.6 TB/s; workgroups in whole rounds count for the most
// part, and sequences of different lengths take longer unless there are many
// workgroups, which take 0.4 us each to start.  A split costs a second launch and
// the partial sums.  Fitted to times measured over
// 100 .. 10000 keys, 8 .. 1024 sequences times key heads, dims 64 and 128, lengths
// alike and spread from 5% to all: within 2.7% of the best choice on the geometric mean.
struct FewRowsCost {
    double latency0, latency1, share0, share1;   // x0 + x1 d
    double rounds;                               // weight of whole rounds
    double spread, even;                         // 1 + spread exp(-workgroups a CU / even)
    double join;
};
constexpr FewRowsCost kFewF16 = {2.9, 0.45, 0.48, 0.26, 0.9, 0.37, 5, 6.5}, kFewF32 = {2.4, 1.25, 0.33, 1.9, 1, 0.215, 7.3, 7.9};

// Eight waves, unsplit, take half the steps where workgroups are no more than
// compute units (32 sequences, 8 key heads, 1000 keys, heads of 128 in fp32: 47 us against
// 52 unsplit and 50 in two splits of four waves; 24 sequences, heads of 64 in fp16:
// 13.7 against 16.7 and 17.8); with more, four waves are ahead (48 sequences:
// 20.8 against 24.3).
AttentionPlan few_rows_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t span, int cus)
{
    const bool half = dtype == NNJIT_F16;
    const FewRowsCost &c = half ? kFewF16 : kFewF32;
    const int64_t lanes = (int64_t)kv_heads * sequences;
    const double d = dim / 128.0, part_us = (double)tokens * q_heads * dim * 8 / 3.3e6;   // partial sums of a split, written and read
    AttentionPlan best{};
    double least = 0;
    for (int waves = 4; waves <= (dim <= 128 && lanes <= cus ? 8 : 4); waves += 4) {
        const int keys = waves * (half ? 32 : 16);          // of a step
        for (int64_t want = 1; want <= (waves == 4 ? 256 : 1); want = want < 4 ? want + 1 : want * 3 / 2 - want * 3 / 2 % 2) {
            const int64_t per = (span + want - 1) / want;
            const int64_t split_keys = std::max<int64_t>((per + 31) / 32 * 32, 32);
            const int64_t splits = std::max<int64_t>((span + split_keys - 1) / split_keys, 1);
            const double per_cu = (double)lanes * splits / cus, units = per_cu * waves / 4;
            const double rounds = per_cu < 1 ? 1 : per_cu < 4 ? per_cu + c.rounds * (std::ceil(per_cu) - per_cu) : per_cu;
            double bytes_us = 2.0 * keys * dim * (half ? 2 : 4) * rounds * cus / 6.6e6;
            if (sequences > 1) bytes_us *= 1 + c.spread * std::exp(-per_cu / c.even);
            const double step = std::max({c.latency0 + c.latency1 * d, (c.share0 + c.share1 * d) * units, bytes_us});
            const double cost = (std::min(split_keys, span) + keys - 1) / keys * step + 0.4 * per_cu + (splits > 1 ? c.join + splits * part_us : 0);
            if (best.tile_rows == 0 || cost < least) {
                least = cost;
                best = AttentionPlan{16, 1, (int)splits, (int)split_keys, waves, 0};
            }
            if (splits < want || per_cu > 16) break;       // more splits than keys, or than the chip holds
        }
    }
    return best;
}

// More rows: estimated time of a step of a kernel's workgroups: max(a, b o) us with `o`
// workgroups to a compute unit, linear in the head dimension d (in units of
// 128), and no less than its bytes at 5.5 TB/s.  Fitted to measured times
// (within about 15% over 64 .. 8192 keys, 8 .. 384 sequences times key heads,
// dims 64 and 128): a is a step's latency, b its share of a CU's matrix cores
// and LDS.
struct StepCost {
    int tile_rows, keys;       // rows of a tile; keys of a step
    double a0, a1, b0, b1;     // a = a0 + a1 d, b = b0 + b1 d
};
constexpr StepCost kStepF16[] = {{16, 128, 1.5, 0, 1.0, 2.0}, {64, 64, 0.35, 0.8, 0.325, 0.35}, {128, 64, 0.5, 1.1, 0.4, 0.65}};
constexpr StepCost kStepF32[] = {{16, 64, 0.9, 1.2, 0.5, 1.0}, {64, 64, 0.4, 4.2, -0.7, 5.8}, {128, 64, -0.3, 7.6, 0.7, 4.65}};

// The kernel and the splits of the keys that these estimates call cheapest.
// Tall tiles read keys and values least often but leave CUs idle where rows are
// few (512 new tokens on 3584 cached, 32 heads of 128, in us: 128 rows unsplit 93,
// 64 rows 82, in two splits 59, 128 rows in four 55; 777 alone: 25, 23, 40, 42);
// up to 128 rows of up to 128 keys the 16-row kernel starts soonest (7 against 8);
// a split costs a second launch and writes and reads the partial sums (512 new
// tokens alone: 16 unsplit, 28 in two).
AttentionPlan many_rows_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t rows,
                             int64_t max_kv, int64_t window, int cus)
{
    const int64_t group = q_heads / kv_heads, lanes = (int64_t)kv_heads * sequences;
    const int elt = dtype == NNJIT_F16 ? 2 : 4;
    const double d = dim / 128.0, part_us = (double)tokens * q_heads * dim * 8 / 3.3e6;   // partial sums of a split, written and read
    AttentionPlan best{};
    double least = 0;
    for (const StepCost &c : dtype == NNJIT_F16 ? kStepF16 : kStepF32) {
        if (c.tile_rows == 64 && dim > 128) continue;      // not built: registers
        const int64_t row_tiles = (rows + c.tile_rows - 1) / c.tile_rows;
        const int64_t span = seen_span(max_kv, window, c.tile_rows, group);
        for (int64_t want = 1; want <= 256; want = want < 4 ? want + 1 : want * 3 / 2 - want * 3 / 2 % 2) {
            const int64_t per = (span + want - 1) / want;
            const int64_t split_keys = std::max<int64_t>((per + 31) / 32 * 32, 32);
            const int64_t splits = std::max<int64_t>((span + split_keys - 1) / split_keys, 1);
            const double o = (double)row_tiles * lanes * splits / cus;
            // keys and values come once from memory for all row tiles; one workgroup a CU does
            // not draw its full rate, a few CUs with one more take longer, and so do
            // sequences of different lengths unless there are many workgroups
            const double even = o < 4 ? std::ceil(o) : o;
            double bytes_us = 2.0 * c.keys * dim * elt * (even / row_tiles) * 256 / (5.5e6 * std::min(1.0, 0.9 + 0.05 * o));
            if (sequences > 1 && o < 8) bytes_us *= 1.15;
            // fp32 products fill the matrix cores of a CU: its second workgroup takes as long again
            const double share = elt == 4 && c.tile_rows > 16 ? std::ceil(o) : o;
            const double step = std::max({c.a0 + c.a1 * d, (c.b0 + c.b1 * d) * share, bytes_us});
            const double cost = ((split_keys < span ? split_keys : span) + c.keys - 1) / c.keys * step + (splits > 1 ? 3.8 + splits * part_us : 0) +
                                (c.tile_rows == 16 ? 0 : 1.5);   // a later start: copies, then products
            if (best.tile_rows == 0 || cost < least) {
                least = cost;
                best.tile_rows = c.tile_rows;
                best.row_tiles = (int)row_tiles;
                best.splits = (int)splits;
                best.split_keys = (int)split_keys;
                best.waves = 4;
            }
            if (splits < want || o > 16) break;            // more splits than keys, or than the chip holds
        }
    }
    return best;
}

}  // namespace

AttentionPlan attention_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t max_q,
                             int64_t max_kv, int causal, int64_t window, int cus)
{
    const int64_t group = q_heads / kv_heads, rows = max_q * group;
    if (!causal) window = 0;
    AttentionPlan plan = rows <= 16 ? few_rows_plan(dtype, tokens, sequences, q_heads, kv_heads, dim, seen_span(max_kv, window, 16, group), cus)
                                    : many_rows_plan(dtype, tokens, sequences, q_heads, kv_heads, dim, rows, max_kv, window, cus);
    plan.ws_floats = plan.splits > 1 ? plan.splits * tokens * q_heads * ((dim + 3) / 4 * 4 + 2) : 0;
    return plan;
}

hipError_t launch_attention(AttentionParams p, const AttentionPlan &plan, int dtype, bool vec, hipStream_t stream)
{
    p.row_tiles = plan.row_tiles;
    p.splits = plan.splits;
    p.split_keys = plan.split_keys;
    p.may_leave_out = plan.splits > 1 && (int64_t)plan.row_tiles * plan.tile_rows < (int64_t)p.batch.tokens * p.group;
    const int grid = plan.row_tiles * plan.splits * (p.q_heads / p.group) * p.batch.sequences;
    hipError_t e;
    if (dtype == NNJIT_F16)
        e = plan.tile_rows == 16 ? launch_typed<_Float16>(p, vec, plan.waves, grid, stream) : launch_attention_tiles_f16(p, plan.tile_rows, vec, grid, stream);
    else
        e = plan.tile_rows == 16 ? launch_typed<float>(p, vec, plan.waves, grid, stream) : launch_attention_tiles_f32(p, plan.tile_rows, vec, grid, stream);
    if (e != hipSuccess || plan.splits == 1) return e;
    return dtype == NNJIT_F16 ? launch_join<_Float16>(p, stream) : launch_join<float>(p, stream);
}

}  // namespace nnjit
