// Attention over a paged cache for many rows (prompts): tiles of 32 rows a
// wave, keys and values shared through LDS.
//
// The mathematics is that of attention_rows.h: one pass over the keys with a
// running reference and sum; here the matrix cores bound it.  A workgroup has WR x WK
// waves: WR row groups of 32 rows, WK groups that take different keys of a
// step (joined through LDS at the end).  A step takes BN = 32 KB WK keys: K and
// V rows go from their pages to LDS by direct copies, one or two steps ahead of the
// products (one barrier a step).  A lane's copies may come from
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
// The reference of a row moves only when a logit passes it by 2^5 (the
// weights are no less exact for it): the sums are rescaled in the first steps and
// hardly ever again.
//
// fp16 weights are rounded once, to 11 bits (or, below 2^-24 of the row's largest,
// to 2^-35 of it).  The sum that divides takes them unrounded; rounding is
// unbiased, and its share of the result's error is that of the result's own
// rounding to fp16 (2.5 .. 2.9e-4 in all, against 2.1e-4 with exact weights).  (Two
// parts, as in attention_rows.h, are half as many products again: 16 drafted trees of 32 nodes 65 us
// against 56, 64 nodes behind 65536 keys 130 against 100, for 2.1e-4 against 2.7e-4 and 2.6e-4.)
//
// Why 32 rows a wave: K and V of a step are read from LDS once per 32 rows, half
// as often as with 16 x 16 products; the sums and queries of 64 rows would leave
// room for one wave a SIMD only.  Tiles of 128 rows (four row groups) read K
// and V least often; tiles of 64 rows (two row groups times two key groups)
// exist for prompts whose 128-row tiles leave compute units idle.
//
// Measured: 2048 new tokens at the end of 16384, 32 heads of 128 on 8, fp16:
// 527 us, 977 TFLOP/s (a large matrix product: 1210): the clock, which power
// holds at about 1.8 GHz under this load -- a quarter fewer scalar instructions, or
// a step's logits computed one step ahead of its softmax (555 -> 545), change
// next to nothing.  512 tokens at the end of 2048, 32 heads: 37 us, 407 TFLOP/s,
// 31 and 6 for the join of two splits; ragged prompts of up to 777 tokens, 12
// heads of 64: 20 us, the 13 steps of the longest tile, one after the other.
// fp32 in three bf16 parts: four sequences of 256 rows on 256 keys, 16 heads of
// 64: 17 us, 62 TFLOP/s; 2048 tokens alone, 32 heads of 128 on 8: 269 us, 128
// TFLOP/s (a large fp32 matrix product: 153), against 372 on the fp32 matrix
// cores.  (With heads of 128 the queries' parts, the sums and the raw chunks are more
// than the registers of two waves a SIMD: tiles of 128 rows spill 36 of them, 148
// bytes of scratch a lane.)
#pragma once

#include <type_traits>

#include "attention_common.h"

namespace nnjit {

namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// How keys and values reach LDS: ANY element by element, from any address;
// CHUNKS copies of 16 bytes, a look-up a lane; PAGED16 copies whose keys lie in one page
// (pages of a multiple of 16 tokens) and whole head dims (dim == DP), addresses
// by scalar arithmetic.  The look-ups of CHUNKS cost about as many vector
// instructions a step as the softmax.
// SPLIT: fp32 on the bf16 matrix cores (kcommon.h): every chunk is loaded into
// registers a step ahead, split into three bf16 parts and stored to three
// planes, each laid out like fp16 rows; SPLIT_ANY loads element by element.
enum { ANY, CHUNKS, PAGED16, SPLIT, SPLIT_ANY };

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is written on purpose
// copy16_to_lds with a scalar base and a 32-bit offset a lane
__device__ __forceinline__ void copy16_to_lds_from(const void *base, unsigned offset, unsigned lds)
{
    // the same in every lane, and said so: the operands must be scalar registers
    const unsigned long long u = (unsigned long long)base;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)u), hi = __builtin_amdgcn_readfirstlane((unsigned)(u >> 32));
    const unsigned long long s = lo | (unsigned long long)hi << 32;
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(s),
                 "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
}
#pragma clang diagnostic pop

// Larger of the two lanes l and l + 32.
__device__ __forceinline__ float max_of_halves(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = both[0], b = both[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// A row's reference is moved when a logit passes the one that it was taken from by
// 2^kSlack.  fp16 weights are then at most 2^(kLift + kSlack), half of the largest half;
// fp32 references lie that much above their logit, so that weights are at most 1 and
// no value times a weight overflows.  Every move scales all
// sums: 512 tokens at the end of 2048 with logits spread by 2^2.9, 32 heads of 128,
// 37.0 us with a slack of 2, 36.1 with 5, 35.7 with 7 or 8.
constexpr int kSlack = 5, kLift = 10;

// Row r of a tile over the keys k0 .. k1 - 1, by one wave: a lane has dims
// lane, lane + 64, ...; only keys that the row sees are touched.  Correctness, not
// speed: a key after the other, 0.2 (fp32) to 0.35 us (fp16) each.  One value that is
// not finite among 2048 keys of 32 heads of 128 thus takes 512 rows, of which a
// wave's 32 are taken anew, from 0.05 to 24 ms (fp16, a key that some of the rows
// do not see) or from 0.14 to 12 ms (fp32); one such query to 0.06 and 0.8 ms.
template <typename T, int DP, bool TREE>
__device__ __forceinline__ void redo_row(const AttentionParams &p, const RowTile &t, int head, int split, int r, int k0, int k1, int lane)
{
    constexpr int E = (DP + 63) / 64;
    constexpr bool HALF = sizeof(T) == 2;
    const int token = t.q0 + p.group_div.quot(r);
    const int lo = max(TREE ? t.first_cached_of(p, token) : t.first_key(p, r), k0), hi = min(TREE ? t.keys : t.end_key(p, r), k1);
    const int q_head = head * p.group + r - p.group_div.quot(r) * p.group;
    bool sees = !TREE && hi > lo;
    const T *q = (const T *)p.q.p + (long long)token * p.q.tok + (long long)q_head * p.q.head;
    float qv[E], o[E], ref = -__builtin_inff(), l = 0.f;
    for (int e = 0; e < E; ++e) {
        qv[e] = lane + 64 * e < p.dim ? (float)q[lane + 64 * e] : 0.f;
        if (p.negate) qv[e] = -qv[e];
        o[e] = 0.f;
    }
#pragma unroll 1
    for (int key = lo; key < hi; ++key) {
        if constexpr (TREE) {
            if (key >= t.cached && !(t.drafted4(p, token, key) & 1)) continue;
            sees = true;
        }
        const int pi = p.pool.page_size.quot(key), slot = key - pi * (int)p.pool.page_size.d;
        const int page = safe_page(p, t.table[pi]);
        const T *k = (const T *)p.pool.k + (long long)head * p.pool.k_head + page_offset(page, p.pool.k_page, slot, p.pool.k_tok);
        const T *v = (const T *)p.pool.v + (long long)head * p.pool.v_head + page_offset(page, p.pool.v_page, slot, p.pool.v_tok);
        float x = 0.f;
        for (int e = 0; e < E; ++e)
            if (lane + 64 * e < p.dim) x += qv[e] * (float)k[lane + 64 * e];
        for (int i = 1; i < 64; i <<= 1) x += __shfl_xor(x, i);
        const float next = fmaxf(ref, reference<HALF, kLift>(p, x)), off = started(next);
        const float shrink = moved<HALF>(p, ref, off), w = weight<HALF>(p, x, off);
        ref = next;
        l = l * shrink + w;
        for (int e = 0; e < E; ++e)
            if (lane + 64 * e < p.dim) o[e] = o[e] * shrink + w * (float)v[lane + 64 * e];
    }
    const long long at = ((long long)split * p.batch.tokens + token) * p.q_heads + q_head;
    T *dst = (T *)p.o.p + (long long)token * p.o.tok + (long long)q_head * p.o.head;
    for (int e = 0; e < E; ++e) {
        const int d = lane + 64 * e;
        if (p.splits == 1) {
            if (d < p.dim) dst[d] = (T)(sees ? o[e] / l : 0.f);
        } else {
            if (d < p.part_dim) p.part[at * p.part_dim + d] = o[e];
        }
    }
    if (p.splits > 1 && lane == 0) store_stat(p, at, ref, l, sees);
}

// Bytes of a row in LDS, and the waves a SIMD is to hold: two, of two
// workgroups, unless the buffers or the registers of one fill a CU.
template <typename T, int DP, int HOW>
constexpr int row_pitch() { return (DP <= 64 ? 64 : DP <= 128 ? 128 : 256) * (HOW >= SPLIT ? 2 : (int)sizeof(T)); }
// Steps whose copies are in LDS or on their way: three where three still leave
// room for three workgroups a CU (heads of 64 dims in fp16: ragged prompts to 777
// 22.3 -> 20.9 us; with heads of 128 they would leave one: 38 -> 53 where two
// fit).  Look-ups a lane would wait for the copies, so only PAGED16.
template <typename T, int DP, int HOW>
constexpr int stages() { return sizeof(T) == 2 && DP == 64 && HOW == PAGED16 ? 3 : 2; }
template <typename T, int DP, int HOW, int BLOCKS>
constexpr int lds_bytes() { return (HOW >= SPLIT ? 6 : 2 * stages<T, DP, HOW>()) * 32 * BLOCKS * row_pitch<T, DP, HOW>(); }
template <typename T, int DP, int HOW, int BLOCKS>
constexpr int waves_per_simd() { return DP <= 128 && lds_bytes<T, DP, HOW, BLOCKS>() <= 80 * 1024 ? 2 : 1; }

// TREE: drafted trees: a row sees its sequence's cached keys (with a window from
// first_cached() on) and the new tokens that its mask names.  Only steps that hold new tokens
// look at masks.  64 nodes behind 65536 keys, 32 heads of 128 on 8, fp16: 97 to 101 us with the join of 32 splits, 690
// TFLOP/s and 2.7 TB/s of keys and values; 16 sequences of up to 4096 keys with 32 nodes each: 56 us, 3.1 TB/s.
// (Tiles of 256 rows by eight waves with four stages: 103; eight waves on 128 rows, half of the keys
// of a step each, with half of the splits: 113 and 61.)
template <typename T, int DP, int HOW, int WR, int WK, int KB, bool TREE>
__global__ void __launch_bounds__(WR * WK * 64, (waves_per_simd<T, DP, HOW, KB * WK>()))
attention_tiles_kernel(AttentionParams p)
{
    constexpr bool PARTS = HOW >= SPLIT;                  // fp32 in three bf16 parts
    constexpr bool VEC = HOW != ANY && HOW != SPLIT_ANY;
    constexpr bool HALF = sizeof(T) == 2 || PARTS;        // 16-bit rows in LDS
    constexpr int NW = WR * WK;
    constexpr int CH = HALF ? 8 : 4;                      // elements of a chunk in LDS
    constexpr int PITCH = row_pitch<T, DP, HOW>();
    constexpr int CPR = PITCH / 16;                       // chunks of a row
    constexpr int BN = 32 * KB * WK;                      // keys of a step
    constexpr int TILE = BN * PITCH;
    constexpr int NI = BN * CPR / 64 / NW;                // copies of a wave, K and V each
    static_assert(NI * 64 * NW == BN * CPR, "copies must split evenly over waves");
    constexpr int QS = HALF ? DP / 16 : DP / 8;           // chunks of a query row per lane
    constexpr int BLK = DP / 32;                          // output blocks of 32 dims
    constexpr int VW = HALF ? 1 : 4;                      // dims a lane reads side by side
    static_assert(HALF || DP % 128 == 0, "whole runs of four dims");
    typedef T chunk __attribute__((ext_vector_type(CH)));

    // K of every stage, then V; in parts the three planes of K and of V of one step
    __shared__ __attribute__((aligned(1024))) char smem[lds_bytes<T, DP, HOW, KB * WK>()];
    constexpr int ST = stages<T, DP, HOW>();
    auto k_buf = [&](int b) -> lds_char * { return (lds_char *)smem + b * TILE; };
    auto v_buf = [&](int b) -> lds_char * { return (lds_char *)smem + ((PARTS ? 3 : ST) + b) * TILE; };

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
    mark_left_out<NW * 64>(p, t, head, tile, split, 32 * WR);

    const int r_last = t.r0 + t.rows - 1;
    const int lo_min = TREE ? t.first_cached(p, 0) : t.first_key(p, t.r0), hi_max = TREE ? t.keys : t.end_key(p, r_last);
    const long long begin = (lo_min & ~31) + (long long)split * p.split_keys;
    const int k0 = (int)min(begin, (long long)hi_max);
    // (trees: the last split goes to the end, for sequences of more new tokens than max_q)
    const int k1 = TREE && split == p.splits - 1 ? hi_max : (int)min(begin + p.split_keys, (long long)hi_max);
    const int first = max(lo_min, k0);                    // keys first .. k1 - 1 are seen by a row of the tile

    // the wave's rows, and this lane's (rows past the end repeat the last one)
    const int w0 = min(t.r0 + 32 * wr, r_last), w1 = min(t.r0 + 32 * wr + 31, r_last);
    const bool wave_rows = t.r0 + 32 * wr <= r_last;
    const int lo_w = max(TREE ? lo_min : t.first_key(p, w0), k0), hi_w = min(TREE ? t.keys : t.end_key(p, w1), k1);
    const int r = min(t.r0 + 32 * wr + n, r_last);
    const int token = t.q0 + p.group_div.quot(r);
    const int q_head = head * p.group + r - p.group_div.quot(r) * p.group;
    const int lo = max(TREE ? t.first_cached_of(p, token) : t.first_key(p, r), k0), hi = min(TREE ? t.cached : t.end_key(p, r), k1);
    const int dim = p.dim;

    chunk q[PARTS ? 1 : QS];
    Split8 qp[PARTS ? QS : 1];
    bool dirty = false;                                   // see redo_row
    if constexpr (PARTS) {
        const T *src = (const T *)p.q.p + (long long)token * p.q.tok + (long long)q_head * p.q.head;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            f32x8 x = load_eight<VEC>((const float *)src, (2 * s + h) * CH, dim);
            if (p.negate) x = -x;
            float top = 0.f;
            qp[s] = split8(x, top);
            dirty |= !splittable(x);
        }
    } else {
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

    // Copy i of this wave brings KPI keys, key_of[i] the lane's, from the step's
    // first key on.  Page ids are looked up a step before they are used.
    constexpr int KPI = 64 / CPR;
    constexpr int WKEYS = NI * KPI;                       // keys that a wave copies: 8 or 16 in a row
    static_assert(HOW != PAGED16 || 16 % WKEYS == 0, "a wave's keys must lie in one page of 16");
    auto key_of = [&](int i, int ln) { return wave * WKEYS + i * KPI + ln / CPR; };
    auto k_col = [&](int i, int ln) { return ((ln % CPR) ^ k_swz(key_of(i, ln))) * CH; };
    auto v_col = [&](int i, int ln) { return ((ln % CPR) ^ v_swz(key_of(i, ln))) * CH; };
    constexpr int IDS = HOW == PAGED16 ? 1 : NI;
    struct Ids {
        int page[IDS];
    };
    auto ids_of = [&](int kt) {
        Ids ids;
#pragma unroll
        for (int i = 0; i < IDS; ++i) {
            const int at = p.pool.page_size.quot(min(kt + key_of(i, HOW == PAGED16 ? 0 : lane), last_key));
            // (a scalar load: a vector load's value would be waited for together with the copies before it)
            if constexpr (HOW == PAGED16) ids.page[i] = ((const constant_int *)t.table)[__builtin_amdgcn_readfirstlane(at)];
            else ids.page[i] = t.table[at];
        }
        return ids;
    };
    auto copy_rows = [&](auto of_keys, const Ids &ids, int kt, int b) {
        constexpr bool KEYS = decltype(of_keys)::value;
        lds_char *buf = KEYS ? k_buf(b) : v_buf(b);
        const T *base = KEYS ? kp : vp;
        const unsigned page_stride = KEYS ? p.pool.k_page : p.pool.v_page, tok_stride = KEYS ? p.pool.k_tok : p.pool.v_tok;
        const unsigned lds = (unsigned)(uintptr_t)buf + wave * NI * 1024;
        int ln = lane;
        if constexpr (HOW == PAGED16) {
            if (kt >= first && kt + BN <= k1) {
                // every key is there, the wave's lie in one page: a scalar address, lane offsets that never change
                const int key = kt + key_of(0, 0);
                const int slot = key - p.pool.page_size.quot(key) * page_size;
                const int page = safe_page(p, __builtin_amdgcn_readfirstlane(ids.page[0]));
                const T *src = base + page_offset(page, page_stride, slot, tok_stride);
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int col = KEYS ? k_col(i, lane) : v_col(i, lane);   // past dim (DP 96 in rows of 128): never read
                    copy16_to_lds_from(src + i * KPI * tok_stride,
                                       ((unsigned)(lane / CPR) * tok_stride + (col < DP ? col : 0)) * (unsigned)sizeof(T), lds + i * 1024);
                }
                return;
            }
            asm volatile("" : "+v"(ln));   // what the few other steps need is not kept in registers
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int at = kt + key_of(i, ln), col = KEYS ? k_col(i, ln) : v_col(i, ln);
            const int key = min(at, last_key);
            const int slot = key - p.pool.page_size.quot(key) * page_size;
            // PAGED16: keys past the last one are taken from the page of the wave's first (and replaced by zeros)
            const T *src = base + page_offset(safe_page(p, ids.page[HOW == PAGED16 ? 0 : i]), page_stride, slot, tok_stride) + col;
            // keys that no row sees are zeros: what lies in their slots must not be multiplied, not even by 0
            const bool ok = at >= first && at < k1;
            if constexpr (VEC) {
                copy16_to_lds(ok && col < dim ? src : (const T *)p.zero, __builtin_amdgcn_readfirstlane(lds + i * 1024));
            } else {
                chunk x;
                for (int e = 0; e < CH; ++e) x[e] = ok && col + e < dim ? src[e] : (T)0;
                *(__attribute__((address_space(3))) chunk *)(buf + (wave * NI + i) * 1024 + lane * 16) = x;
            }
        }
    };

    // PARTS: the thread's chunks of a step, loaded and, a step later, stored
    struct Raw {
        f32x8 k[PARTS ? NI : 1], v[PARTS ? NI : 1];
    };
    auto load_raw = [&](const Ids &ids, int kt) {
        Raw raw;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int at = kt + key_of(i, lane), col = (lane % CPR) * CH;
            const int key = min(at, last_key);
            const int slot = key - p.pool.page_size.quot(key) * page_size, page = safe_page(p, ids.page[HOW >= SPLIT ? i : 0]);
            // keys that no row sees are zeros
            const int room = at >= first && at < k1 ? dim : 0;
            raw.k[i] = load_eight<VEC>((const float *)kp + page_offset(page, p.pool.k_page, slot, p.pool.k_tok), col, room);
            raw.v[i] = load_eight<VEC>((const float *)vp + page_offset(page, p.pool.v_page, slot, p.pool.v_tok), col, room);
        }
        return raw;
    };
    auto store_raw = [&](const Raw &raw) {
        typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int key = key_of(i, lane), c = lane % CPR;
            dirty |= !splittable(raw.k[i]) || !splittable(raw.v[i]);
            float top = 0.f;
            const Split8 ks = split8(raw.k[i], top), vs = split8(raw.v[i], top);
            lds_char *kd = k_buf(0) + key * PITCH + (c ^ k_swz(key)) * 16, *vd = v_buf(0) + key * PITCH + (c ^ v_swz(key)) * 16;
            *(lds_bf16x8 *)kd = ks.h;
            *(lds_bf16x8 *)(kd + TILE) = ks.m;
            *(lds_bf16x8 *)(kd + 2 * TILE) = ks.l;
            *(lds_bf16x8 *)vd = vs.h;
            *(lds_bf16x8 *)(vd + TILE) = vs.m;
            *(lds_bf16x8 *)(vd + 2 * TILE) = vs.l;
        }
    };

    f32x16 acc[BLK];
#pragma unroll
    for (int b = 0; b < BLK; ++b) acc[b] = f32x16{};
    float ref = -__builtin_inff(), l = 0.f;
    constexpr bool SCALED = sizeof(T) == 2;               // references and weights of fp16
    const float slack = kSlack / p.scale_log2;
    float limit = -__builtin_inff();                      // logits above it move the reference

    // lane parts of the LDS addresses
    const int kw = wk * KB * 32;                          // first key of this wave in a step
    const int k_row = (kw + n) * PITCH;
    const int tr_r = (lane & 15) >> 2;                    // transposing reads: row of the group of four
    const int v_row = HALF ? (kw + 4 * h + tr_r) * PITCH + (lane & 3) * 8 : (kw + 4 * h) * PITCH + n * VW * 4;
    const int v_unit = HALF ? (lane >> 4) & 1 : 0;

    // V of the wave's 32-key block kb: fp16, product u (of two) and block db of 32
    // dims: eight keys of one dim
    auto read_v16 = [&](int b, int kb, int u, int db) {
        const int unit = (2 * db + v_unit) ^ (v_swz(tr_r) >> 1);
        s16x4 part[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4 *)(v_buf(b) + v_row + (32 * kb + 8 * (2 * u + e)) * PITCH + unit * 32));
        return __builtin_bit_cast(f16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // fp32: key i (of 16 a half wave), dims group g: VW dims of one key
    typedef float vvec __attribute__((ext_vector_type(VW)));
    auto read_v32 = [&](int b, int kb, int i, int g) {
        return *(__attribute__((address_space(3))) vvec *)(v_buf(b) + v_row + (32 * kb + 8 * (i / 4) + i % 4) * PITCH + g * 32 * VW * 4);
    };

    // O^T += V^T P^T, P in x.  CHECK: note in `dirty` if any of the values is not finite
    auto add_values = [&](auto check, const f32x16 *x, int b) {
        constexpr bool CHECK = decltype(check)::value;
        Largest16 largest;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            if constexpr (PARTS) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    f32x8 w;
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = x[kb][8 * u + i];
                    float top = 0.f;
                    const Split8 pr = split8(w, top);
                    // two blocks at a time: their products run in turns
                    constexpr int TOGETHER = BLK % 2 == 0 ? 2 : 1;
#pragma unroll
                    for (int d0 = 0; d0 < BLK; d0 += TOGETHER) {
                        bf16x8 v[TOGETHER][3];
#pragma unroll
                        for (int d = 0; d < TOGETHER; ++d)
#pragma unroll
                            for (int part = 0; part < 3; ++part) v[d][part] = __builtin_bit_cast(bf16x8, read_v16(part, kb, u, d0 + d));
                        const bf16x8 w3[3] = {pr.h, pr.m, pr.l};
                        constexpr int V_PART[6] = {0, 2, 1, 0, 1, 0}, W_PART[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
                        for (int i = 0; i < 6; ++i)
#pragma unroll
                            for (int d = 0; d < TOGETHER; ++d) acc[d0 + d] = mma_bf16(v[d][V_PART[i]], w3[W_PART[i]], acc[d0 + d]);
                    }
                }
            } else if constexpr (HALF) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    f16x8 pr;
#pragma unroll
                    for (int i = 0; i < 8; ++i) pr[i] = (_Float16)x[kb][8 * u + i];
#pragma unroll
                    for (int db = 0; db < BLK; ++db) {
                        const f16x8 v = read_v16(b, kb, u, db);
                        if constexpr (CHECK) largest.take(v);
                        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pr, acc[db], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int g = 0; g < BLK / VW; ++g) {
                        const vvec v = read_v32(b, kb, i, g);
#pragma unroll
                        for (int e = 0; e < VW; ++e) {
                            const float value = v[e];
                            if constexpr (CHECK) dirty |= !finite(value);
                            acc[g * VW + e] = __builtin_amdgcn_mfma_f32_32x32x2f32(value, x[kb][i], acc[g * VW + e], 0, 0, 0);
                        }
                    }
            }
        }
        if constexpr (CHECK && HALF && !PARTS) dirty |= !largest.finite();
    };

    // one step of this wave; WHOLE: every row sees every key of it
    auto step = [&](auto is_whole, int key0, int b) {
        constexpr bool WHOLE = decltype(is_whole)::value;
        f32x16 x[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            x[kb] = f32x16{};
            f32x16 low = {};
#pragma unroll
            for (int s = 0; s < QS; ++s) {
                const int c = (2 * s + h) ^ k_swz(n);
                if constexpr (PARTS) {
                    typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
                    const lds_char *at = k_buf(0) + k_row + kb * 32 * PITCH + c * 16;
                    const bf16x8 kh = *(const lds_bf16x8 *)at, km = *(const lds_bf16x8 *)(at + TILE), kl = *(const lds_bf16x8 *)(at + 2 * TILE);
                    // two sums, so that a product does not wait for the one before it
                    x[kb] = mma_bf16(kh, qp[s].m, x[kb]);
                    low = mma_bf16(kh, qp[s].l, low);
                    x[kb] = mma_bf16(km, qp[s].h, x[kb]);
                    low = mma_bf16(kl, qp[s].h, low);
                    x[kb] = mma_bf16(kh, qp[s].h, x[kb]);
                    low = mma_bf16(km, qp[s].m, low);
                    if (s == QS - 1) x[kb] += low;
                } else {
                    const chunk a = *(__attribute__((address_space(3))) chunk *)(k_buf(b) + k_row + kb * 32 * PITCH + c * 16);
                    if constexpr (HALF) {
                        x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q[s], x[kb], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], q[s][i], x[kb], 0, 0, 0);
                    }
                }
            }
        }
        if constexpr (!WHOLE) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                [[maybe_unused]] unsigned drafted = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + 32 * kb + 8 * (i / 4) + 4 * h + i % 4;
                    bool see = key >= lo && key < hi;
                    if constexpr (TREE) {
                        if (i % 4 == 0) drafted = t.drafted4(p, token, key);
                        see |= key >= t.cached && key < k1 && (drafted >> i % 4 & 1);
                    }
                    x[kb][i] = see ? x[kb][i] : -__builtin_inff();
                }
            }
        }
        float top = x[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
        top = max_of_halves(top);
        if (__any(top > limit)) {
            const float room = top + slack;
            const float next = fmaxf(ref, SCALED ? reference<true, kLift>(p, top) : room);
            const float shrink = moved<SCALED>(p, ref, started(next));
            ref = next;
            limit = SCALED ? fmaxf(limit, room) : next;
            l *= shrink;
#pragma unroll
            for (int blk = 0; blk < BLK; ++blk) acc[blk] *= shrink;
        }
        const float off = started(ref);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[kb][i] = weight<SCALED>(p, x[kb][i], off);
                l += x[kb][i];
            }
        add_values(std::bool_constant<!WHOLE>{}, x, b);
    };

    const int start = k0 & ~31;                           // k0 is a multiple of 32 or hi_max (no keys)
    const int steps = k1 > k0 ? (k1 - start + BN - 1) / BN : 0;
    // steps whole_from .. whole_to - 1: every row of the workgroup sees every key.
    // The others, a few at either end, run a loop of their own: one loop with
    // both kinds of step in it would hold the sums in two sets of registers.
    const int lo_max = TREE ? t.first_cached(p, t.new_tokens - 1) : t.first_key(p, r_last), hi_min = min(TREE ? t.cached : t.end_key(p, t.r0), k1);
    const int whole_from = min(max((lo_max - start + BN - 1) / BN, 0), steps);
    const int whole_to = hi_min > start ? max((hi_min - start) / BN, whole_from) : whole_from;
    Ids ids;
    Raw raw;
    if (steps > 0) {
        ids = ids_of(start);
        if constexpr (PARTS) {
            raw = load_raw(ids, start);
        } else {
#pragma unroll
            for (int stage = 0; stage < ST - 1; ++stage) {
                if (stage > 0 && stage >= steps) break;
                if (stage > 0) ids = ids_of(start + stage * BN);
                copy_rows(std::true_type{}, ids, start + stage * BN, stage);
                copy_rows(std::false_type{}, ids, start + stage * BN, stage);
            }
        }
        ids = ids_of(start + (PARTS ? 1 : ST - 1) * BN);
    }
    auto next_step = [&](int it) {
        if constexpr (PARTS) {
            lds_barrier();                                // every wave has read the last step's planes
            store_raw(raw);
            if (it + 1 < steps) {
                raw = load_raw(ids, start + (it + 1) * BN);
                ids = ids_of(start + (it + 2) * BN);
            }
            lds_barrier();
        } else {
            // this step's copies have arrived (a later step's may be on their way), and
            // every wave has read the buffers that the copies below fill
            if (ST == 3 && it + 1 < steps) wait_vmcnt<ST == 3 ? 2 * NI : 0>();
            else wait_vmcnt<0>();
            lds_barrier();
            if (it + ST - 1 < steps) {
                copy_rows(std::true_type{}, ids, start + (it + ST - 1) * BN, (it + ST - 1) % ST);
                copy_rows(std::false_type{}, ids, start + (it + ST - 1) * BN, (it + ST - 1) % ST);
                ids = ids_of(start + (it + ST) * BN);
            }
        }
    };
    for (int it = 0; it < steps;) {
        const int part_to = it < whole_from ? whole_from : steps;
        if (it < whole_from || it >= whole_to) {
            for (; it < part_to; ++it) {
                next_step(it);
                const int key0 = start + it * BN + kw;
                if (wave_rows && key0 < hi_w && key0 + 32 * KB > lo_w) step(std::false_type{}, key0, it % ST);
            }
        }
        for (; it < whole_to; ++it) {
            next_step(it);
            step(std::true_type{}, 0, it % ST);
        }
    }
    l += __shfl_xor(l, 32);
    dirty = PARTS ? __syncthreads_or(dirty) : __any(dirty);   // in parts, any thread may have met the value

    if constexpr (WK > 1) {
        // join the key groups: those of groups 1 .. WK - 1 through LDS, in order
        constexpr int BOX = (BLK * 16 + 3) * 64;          // words a wave
        static_assert(WR * (WK - 1) * BOX * 4 <= (int)sizeof(smem), "sums of the key groups must fit");
        typedef __attribute__((address_space(3))) float lds_float;
        auto box_of = [&](int g) { return (lds_float *)(lds_char *)smem + (wr * (WK - 1) + g - 1) * BOX + lane; };
        lds_barrier();
        if (wk > 0) {
            lds_float *box = box_of(wk);
            box[0] = ref;
            box[64] = l;
            box[128] = dirty ? 1.f : 0.f;
#pragma unroll
            for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
                for (int i = 0; i < 16; ++i) box[(3 + blk * 16 + i) * 64] = acc[blk][i];
        }
        lds_barrier();
        if (wk > 0) return;
#pragma unroll
        for (int g = 1; g < WK; ++g) {
            lds_float *box = box_of(g);
            const float other = box[0], ol = box[64];
            dirty |= box[128] != 0.f;
            const float next = fmaxf(ref, other);
            const float off = started(next);
            const float mine = moved<SCALED>(p, ref, off), theirs = moved<SCALED>(p, other, off);
            ref = next;
            l = l * mine + ol * theirs;
#pragma unroll
            for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[blk][i] = acc[blk][i] * mine + box[(3 + blk * 16 + i) * 64] * theirs;
        }
    }

    if (__any(dirty)) {
        // a step that some of the rows saw only in part held a value that is not
        // finite, and 0 times it has spoilt rows that do not see it; or, in parts,
        // some query, key or value is not the sum of its parts.  Either leaves a NaN
        // or an infinity in the sums of every row that it reaches: those rows are
        // taken anew, key by key
        bool bad = !finite(l);
#pragma unroll
        for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float sum = acc[blk][i];
                bad |= !finite(sum);
            }
        const unsigned long long lanes = __ballot(bad);
        const unsigned rows = (unsigned)(lanes | lanes >> 32);
#pragma unroll 1
        for (int i = 0; i < 32 && t.r0 + 32 * wr + i <= r_last; ++i)
            if (rows >> i & 1) redo_row<T, DP, TREE>(p, t, head, split, t.r0 + 32 * wr + i, k0, k1, lane);
        if (rows >> n & 1) return;
    }
    if (t.r0 + 32 * wr + n > r_last) return;
    // block g VW + e holds dims 32 VW g + VW j + e, j = 8 (i / 4) + 4 h + i % 4: runs of 4 VW dims
    const bool sees = TREE ? t.drafted_any(p, token, k0, k1) : hi > lo;
    const float inv = p.splits == 1 ? 1.f / l : 1.f;
    const long long at = ((long long)split * p.batch.tokens + token) * p.q_heads + q_head;
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
    if (p.splits > 1 && h == 0) store_stat(p, at, ref, l, sees);
}

template <typename T, int DP, int HOW, int KB, bool TREE>
hipError_t launch_shape(const AttentionParams &p, int tile_rows, int grid, hipStream_t stream)
{
    if (tile_rows == 128) {
        attention_tiles_kernel<T, DP, HOW, 4, 1, KB, TREE><<<grid, 256, 0, stream>>>(p);
    } else if constexpr (DP <= 128) {
        attention_tiles_kernel<T, DP, HOW, 2, 2, 1, TREE><<<grid, 256, 0, stream>>>(p);
    } else {
        return hipErrorInvalidValue;   // the plan asks for none
    }
    return hipGetLastError();
}

template <typename T, int DP, int KB, bool TREE>
hipError_t launch_chunks(const AttentionParams &p, int tile_rows, int grid, hipStream_t stream)
{
    // lane offsets of PAGED16 are 32 bits: at most 8 keys and a row
    const bool near = p.pool.k_tok < (1u << 24) && p.pool.v_tok < (1u << 24);
    return p.dim == DP && p.pool.page_size.d % 16 == 0 && near ? launch_shape<T, DP, PAGED16, KB, TREE>(p, tile_rows, grid, stream)
                                                               : launch_shape<T, DP, CHUNKS, KB, TREE>(p, tile_rows, grid, stream);
}

}  // namespace

}  // namespace nnjit
