// Attention over a paged cache for many rows (prompts): tiles of 32 rows a
// wave, keys and values shared through LDS.
//
// The mathematics is that of attention_rows.hip: one pass over the keys with a
// running reference m and sum; here the matrix cores bound it.  A workgroup has WR x WK
// waves: WR row groups of 32 rows, WK groups that take different keys of a
// step (joined through LDS at the end).  A step takes BN = 32 KB WK keys: K and
// V rows go from their pages to LDS by direct copies, one step ahead of the
// products (two buffers, one barrier a step).  A lane's copies may come from
// any address, so pages cost nothing but their look-up, which runs one step
// ahead of the copies.
//
//   S^T = K Q^T   32 keys x 32 rows: lane l holds row l % 32 and the logits of
//                 the keys 8 i + 4 h + j (h = l / 32, i, j = 0 .. 3)
//   O^T = V^T P^T the probabilities are the second operand as they lie; its
//                 k slots are those keys, in that order, so V rows are
//                 read from LDS in the same order: fp16 by transposing reads
//                 (ds_read_b64_tr_b16: a lane gets four keys of one dim), fp32
//                 plainly (a product takes two keys, one per half wave)
//
// so a row's statistics stay in its own two lanes, next to its sums: no
// exchange but one shuffle for the maximum.
//
// LDS layout: rows of K and V of PITCH bytes, their 16-byte chunks permuted by
// an XOR with the key (made by the choice of the global chunk that a lane
// copies), so that the 16 lanes that a 128-bit read serves at a time -- 16
// keys at one chunk -- and the four keys of a transposing read fall on
// different banks.
//
// The reference m of a row moves only when a logit passes it by 2^8 (the
// weights then are at most 2^8, no less exact in fp16 or fp32): the sums are
// rescaled in the first steps and hardly ever again.
//
// fp16 probabilities are rounded once to 11 bits.  The sum that divides takes
// them unrounded; rounding is unbiased, and its share of the result's
// error is that of the result's own rounding to fp16.
#pragma once

#include "attention_common.h"

namespace nnjit {

namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// What a row's weights may exceed 1 by before its reference is moved: 2^8.
constexpr float kSlack = 8.f;

template <typename T, int DP, bool VEC, int WR, int WK, int KB>
__global__ void __launch_bounds__(WR * WK * 64, DP <= 128 ? 2 : 1)
attention_tiles_kernel(AttentionParams p)
{
    constexpr bool HALF = sizeof(T) == 2;
    constexpr int NW = WR * WK;
    constexpr int CH = 16 / sizeof(T);                    // elements of a chunk
    constexpr int PITCH = (DP <= 64 ? 64 : DP <= 128 ? 128 : 256) * (int)sizeof(T);
    constexpr int CPR = PITCH / 16;                       // chunks of a row
    constexpr int BN = 32 * KB * WK;                      // keys of a step
    constexpr int TILE = BN * PITCH;
    constexpr int NI = BN * CPR / 64 / NW;                // copies of a wave, K and V each
    static_assert(NI * 64 * NW == BN * CPR, "copies must split evenly over waves");
    constexpr int QS = HALF ? DP / 16 : DP / 8;           // chunks of a query row per lane
    constexpr int BLK = DP / 32;                          // output blocks of 32 dims
    constexpr int VW = HALF ? 1 : DP % 128 == 0 ? 4 : DP % 64 == 0 ? 2 : 1;   // dims a lane reads side by side
    typedef T chunk __attribute__((ext_vector_type(CH)));

    __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];   // K, K, V, V
    auto k_buf = [&](int b) -> lds_char * { return (lds_char *)smem + b * TILE; };
    auto v_buf = [&](int b) -> lds_char * { return (lds_char *)smem + (2 + b) * TILE; };

    // chunk c of key row `key` sits at c ^ swizzle
    auto k_swz = [](int key) { return CPR >= 16 ? (key & 15) : ((key >> 1) & 7); };
    auto v_swz = [](int key) { return !HALF ? 0 : CPR >= 16 ? (key & 3) << 2 : ((key >> 1) & 1) << 2; };

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave / WK, wk = wave % WK;
    const int n = lane & 31, h = lane >> 5;

    // row tiles of one sequence and key head run on one XCD, the longest (last) first
    int id = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = p.row_tiles - 1 - id % p.row_tiles;
    id /= p.row_tiles;
    const int split = id % p.splits;
    id /= p.splits;
    const int kv_heads = p.q_heads / p.group;
    const int head = id % kv_heads;
    const int seq = id / kv_heads;
    const RowTile t = row_tile(p, seq, tile, 32 * WR);
    if (t.rows <= 0) return;

    const int r_last = t.r0 + t.rows - 1;
    const int lo_min = t.first_key(p, t.r0), hi_max = t.end_key(p, r_last);
    const long long begin = (lo_min & ~31) + (long long)split * p.split_keys;
    const int k0 = (int)min(begin, (long long)hi_max);
    const int k1 = (int)min(begin + p.split_keys, (long long)hi_max);
    const int first = max(lo_min, k0);                    // keys first .. k1 - 1 are seen by a row of the tile

    // the wave's rows, and this lane's (rows past the end repeat the last one)
    const int w0 = min(t.r0 + 32 * wr, r_last), w1 = min(t.r0 + 32 * wr + 31, r_last);
    const bool wave_rows = t.r0 + 32 * wr <= r_last;
    const int lo_w = max(t.first_key(p, w0), k0), lo_all = t.first_key(p, w1);
    const int hi_w = min(t.end_key(p, w1), k1), hi_all = min(t.end_key(p, w0), k1);
    const int r = min(t.r0 + 32 * wr + n, r_last);
    const int token = t.q0 + p.group_div.quot(r);
    const int q_head = head * p.group + r - p.group_div.quot(r) * p.group;
    const int lo = max(t.first_key(p, r), k0), hi = min(t.end_key(p, r), k1);
    const int dim = p.dim;

    chunk q[QS];
    {
        const T *src = (const T *)p.q.p + (long long)token * p.q.tok + (long long)q_head * p.q.head;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            const int d = (2 * s + h) * CH;
            if constexpr (VEC) {
                q[s] = chunk{};
                if (d < dim) q[s] = *(const chunk *)(src + d);
            } else {
                for (int i = 0; i < CH; ++i) q[s][i] = d + i < dim ? src[d + i] : (T)0;
            }
            if (p.negate) q[s] = -q[s];
        }
    }

    const T *kp = (const T *)p.pool.k + (long long)head * p.pool.k_head;
    const T *vp = (const T *)p.pool.v + (long long)head * p.pool.v_head;
    const int page_size = p.pool.page_size.d;
    const int last_key = max(hi_max - 1, 0);

    // the keys of this lane's copies, relative to the step's first
    int key_of[NI];
    int k_col[NI], v_col[NI];                             // logical element columns
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int at = (i * NW + wave) * 64 + lane;
        key_of[i] = at / CPR;
        k_col[i] = ((at % CPR) ^ k_swz(key_of[i])) * CH;
        v_col[i] = ((at % CPR) ^ v_swz(key_of[i])) * CH;
    }
    struct Ids {
        int page[NI];
    };
    auto ids_of = [&](int kt) {
        Ids ids;
#pragma unroll
        for (int i = 0; i < NI; ++i) ids.page[i] = t.table[p.pool.page_size.quot(min(kt + key_of[i], last_key))];
        return ids;
    };
    auto copy_step = [&](const Ids &ids, int kt, int b) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int key = min(kt + key_of[i], last_key);
            const int slot = key - p.pool.page_size.quot(key) * page_size;
            const long long page = safe_page(p, ids.page[i]);
            const T *ks = kp + page * p.pool.k_page + (long long)slot * p.pool.k_tok + k_col[i];
            const T *vs = vp + page * p.pool.v_page + (long long)slot * p.pool.v_tok + v_col[i];
            // keys that no row sees are zeros: what lies in their slots must not be multiplied, not even by 0
            const bool ok = kt + key_of[i] >= first && kt + key_of[i] < k1;
            const unsigned at = (unsigned)((i * NW + wave) * 1024);
            if constexpr (VEC) {
                copy16_to_lds(ok && k_col[i] < dim ? ks : (const T *)p.zero, (unsigned)(uintptr_t)k_buf(b) + at);
                copy16_to_lds(ok && v_col[i] < dim ? vs : (const T *)p.zero, (unsigned)(uintptr_t)v_buf(b) + at);
            } else {
                chunk kc, vc;
                for (int e = 0; e < CH; ++e) {
                    kc[e] = ok && k_col[i] + e < dim ? ks[e] : (T)0;
                    vc[e] = ok && v_col[i] + e < dim ? vs[e] : (T)0;
                }
                *(__attribute__((address_space(3))) chunk *)(k_buf(b) + at + lane * 16) = kc;
                *(__attribute__((address_space(3))) chunk *)(v_buf(b) + at + lane * 16) = vc;
            }
        }
    };

    f32x16 acc[BLK];
#pragma unroll
    for (int b = 0; b < BLK; ++b) acc[b] = f32x16{};
    float m = -__builtin_inff(), l = 0.f;
    const float scale = p.scale_log2, slack = kSlack / p.scale_log2;

    // lane parts of the LDS addresses
    const int kw = wk * KB * 32;                          // first key of this wave in a step
    const int k_row = (kw + n) * PITCH;
    const int tr_r = (lane & 15) >> 2;                    // transposing reads: row of the group of four
    const int v_row = HALF ? (kw + 4 * h + tr_r) * PITCH + (lane & 3) * 8 : (kw + 4 * h) * PITCH + n * VW * 4;
    const int v_unit = HALF ? (lane >> 4) & 1 : 0;

    auto compute = [&](int kt, int b) {
        const int key0 = kt + kw;
        if (!wave_rows || key0 >= hi_w || key0 + 32 * KB <= lo_w) return;
        f32x16 x[KB];
        lds_char *kb_ = k_buf(b), *vb_ = v_buf(b);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            x[kb] = f32x16{};
#pragma unroll
            for (int s = 0; s < QS; ++s) {
                const int c = (2 * s + h) ^ k_swz(n);
                const chunk a = *(__attribute__((address_space(3))) chunk *)(kb_ + k_row + kb * 32 * PITCH + c * 16);
                if constexpr (HALF) {
                    x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q[s], x[kb], 0, 0, 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], q[s][i], x[kb], 0, 0, 0);
                }
            }
        }
        const bool whole = key0 >= lo_all && key0 + 32 * KB <= hi_all;
        unsigned seen[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) seen[kb] = ~0u;
        if (!whole) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                seen[kb] = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + 32 * kb + 8 * (i / 4) + 4 * h + i % 4;
                    const bool see = key >= lo && key < hi;
                    x[kb][i] = see ? x[kb][i] : -__builtin_inff();
                    seen[kb] |= see ? 1u << i : 0u;
                }
            }
        }
        float top = x[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top - m > slack)) {
            const float next = fmaxf(m, top);
            const float shrink = exp2_fast((m - (next == -__builtin_inff() ? 0.f : next)) * scale);
            m = next;
            l *= shrink;
#pragma unroll
            for (int blk = 0; blk < BLK; ++blk) acc[blk] *= shrink;
        }
        const float off = m == -__builtin_inff() ? 0.f : m * scale;   // a row that has seen nothing yet
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[kb][i] = exp2_fast(fmaf(x[kb][i], scale, -off));
                l += x[kb][i];
            }
        if constexpr (HALF) {
#pragma unroll
            for (int u = 0; u < 2 * KB; ++u) {
                const int kb = u / 2, i0 = 8 * (u % 2);
                f16x8 pr;
#pragma unroll
                for (int i = 0; i < 8; ++i) pr[i] = (_Float16)x[kb][i0 + i];
#pragma unroll
                for (int db = 0; db < BLK; ++db) {
                    const int unit = (2 * db + v_unit) ^ (v_swz(tr_r) >> 1);
                    s16x4 part[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (lds_s16x4 *)(vb_ + v_row + (32 * kb + 8 * (2 * (u % 2) + e)) * PITCH + unit * 32));
                    f16x8 v = __builtin_bit_cast(f16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
                    if (!whole) {
                        Largest16 largest;
                        largest.take(v);
                        if (__any(!largest.finite())) {
                            f16x8 cls, vis;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                cls[i] = class_of(v[i]);
                                v[i] = finite(v[i]) ? v[i] : (_Float16)0.f;
                                vis[i] = (_Float16)((seen[kb] >> (i0 + i) & 1) ? 1.f : 0.f);
                            }
                            const f32x16 c = __builtin_amdgcn_mfma_f32_32x32x16_f16(cls, vis, f32x16{}, 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[db][i] = add_classes(acc[db][i], c[i]);
                        }
                    }
                    acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pr, acc[db], 0, 0, 0);
                }
            }
        } else {
            typedef float vvec __attribute__((ext_vector_type(VW)));
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
#pragma unroll
                    for (int g = 0; g < BLK / VW; ++g) {
                        vvec v = *(__attribute__((address_space(3))) vvec *)(vb_ + v_row + (32 * kb + 8 * (i / 4) + i % 4) * PITCH +
                                                                              g * 32 * VW * 4);
                        bool bad = false;
#pragma unroll
                        for (int e = 0; e < VW; ++e) bad |= !finite((float)v[e]);
                        if (!whole && __any(bad)) {
                            const float vis = (seen[kb] >> i & 1) ? 1.f : 0.f;
#pragma unroll
                            for (int e = 0; e < VW; ++e) {
                                const f32x16 c = __builtin_amdgcn_mfma_f32_32x32x2f32(class_of((float)v[e]), vis, f32x16{}, 0, 0, 0);
                                v[e] = finite((float)v[e]) ? v[e] : 0.f;
#pragma unroll
                                for (int j = 0; j < 16; ++j) acc[g * VW + e][j] = add_classes(acc[g * VW + e][j], c[j]);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < VW; ++e)
                            acc[g * VW + e] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], x[kb][i], acc[g * VW + e], 0, 0, 0);
                    }
                }
        }
    };

    const int start = k0 & ~31;                           // k0 is a multiple of 32 or hi_max (no keys)
    const int steps = k1 > k0 ? (k1 - start + BN - 1) / BN : 0;
    if (steps > 0) {
        Ids ids = ids_of(start);
        copy_step(ids, start, 0);
        ids = ids_of(start + BN);
        for (int it = 0; it < steps; ++it) {
            // this step's copies have arrived, and every wave has read the other buffer
            wait_vmcnt<0>();
            lds_barrier();
            const int kt = start + it * BN;
            if (it + 1 < steps) {
                copy_step(ids, kt + BN, (it + 1) & 1);
                ids = ids_of(kt + 2 * BN);
            }
            compute(kt, it & 1);
        }
    }
    l += __shfl_xor(l, 32);

    if constexpr (WK > 1) {
        // join the key groups: the sums of group g > 0 through LDS, in order
        static_assert(WR * (BLK * 16 + 2) * 64 * 4 <= 4 * TILE, "sums of a key group must fit");
        __attribute__((address_space(3))) float *box = (__attribute__((address_space(3))) float *)(lds_char *)smem +
                                                       wr * (BLK * 16 + 2) * 64 + lane;
#pragma unroll
        for (int g = 1; g < WK; ++g) {
            lds_barrier();
            if (wk == g) {
                box[0] = m;
                box[64] = l;
#pragma unroll
                for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
                    for (int i = 0; i < 16; ++i) box[(2 + blk * 16 + i) * 64] = acc[blk][i];
            }
            lds_barrier();
            if (wk == 0) {
                const float om = box[0], ol = box[64];
                const float next = fmaxf(m, om);
                const float off = next == -__builtin_inff() ? 0.f : next;
                const float mine = exp2_fast((m - off) * scale), theirs = exp2_fast((om - off) * scale);
                m = next;
                l = l * mine + ol * theirs;
#pragma unroll
                for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[blk][i] = acc[blk][i] * mine + box[(2 + blk * 16 + i) * 64] * theirs;
            }
        }
        if (wk != 0) return;
    }

    if (t.r0 + 32 * wr + n > r_last) return;
    // block g VW + e holds dims 32 VW g + VW j + e, j = 8 (i / 4) + 4 h + i % 4: runs of 4 VW dims
    const bool sees = hi > lo;
    const float inv = p.splits == 1 ? 1.f / l : 1.f;
    const long long row = (long long)token * p.q_heads + q_head;
    const long long at = (long long)split * p.batch.tokens * p.q_heads + row;
    T *dst = (T *)p.o.p + (long long)token * p.o.tok + (long long)q_head * p.o.head;
#pragma unroll
    for (int g = 0; g < BLK / VW; ++g)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                const int d = 32 * VW * g + (8 * i4 + 4 * h) * VW + 4 * w;
                float o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = acc[g * VW + (4 * w + e) % VW][4 * i4 + (4 * w + e) / VW];
                if (p.splits == 1) {
                    // a row without a key is 0; one whose logits are all -inf is 0 / 0
                    typedef T quad __attribute__((ext_vector_type(4)));
                    quad out;
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[e] = (T)(sees ? o[e] * inv : 0.f);
                    if constexpr (VEC) {
                        if (d < dim) *(quad *)(dst + d) = out;
                    } else {
                        for (int e = 0; e < 4; ++e)
                            if (d + e < dim) dst[d + e] = out[e];
                    }
                } else {
                    if (d < dim) *(f32x4 *)(p.part + at * p.part_dim + d) = f32x4{o[0], o[1], o[2], o[3]};
                }
            }
    if (p.splits > 1 && h == 0) {
        // a sum that is a NaN stays one in the join (weight exp2(inf - inf));
        // keys seen, but only logits of -inf: 0 / 0 unless another split has more
        p.stat[at * 2] = l != l ? __builtin_inff() : m * scale;
        p.stat[at * 2 + 1] = sees && l == 0.f ? __builtin_nanf("") : l;
    }
}

template <typename T, int DP, bool VEC, int KB>
hipError_t launch_shape(const AttentionParams &p, int tile_rows, int grid, hipStream_t stream)
{
    if (tile_rows == 128) {
        attention_tiles_kernel<T, DP, VEC, 4, 1, KB><<<grid, 256, 0, stream>>>(p);
    } else if constexpr (DP <= 128) {
        attention_tiles_kernel<T, DP, VEC, 2, 2, 1><<<grid, 256, 0, stream>>>(p);
    } else {
        return hipErrorInvalidValue;   // the plan asks for none
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_tiles(const AttentionParams &p, int tile_rows, bool vec, int grid, hipStream_t stream)
{
    constexpr int KB = sizeof(T) == 2 ? 2 : 1;
    if (!vec) {
        return p.dim <= 128 ? launch_shape<T, 128, false, KB>(p, tile_rows, grid, stream)
                            : launch_shape<T, 256, false, 1>(p, tile_rows, grid, stream);
    }
    if (p.dim <= 64) return launch_shape<T, 64, true, KB>(p, tile_rows, grid, stream);
    if (p.dim <= 96) return launch_shape<T, 96, true, KB>(p, tile_rows, grid, stream);
    if (p.dim <= 128) return launch_shape<T, 128, true, KB>(p, tile_rows, grid, stream);
    return launch_shape<T, 256, true, 1>(p, tile_rows, grid, stream);
}

}  // namespace

}  // namespace nnjit
