// Rotary positions and appends to a paged cache.
//
// A turned head row: with c = cos, s = sin of pair i at the row's position,
//   y_a = x_a c - x_b s,   y_b = x_b c + x_a s,
// (a, b) = (i, i + rot / 2) in the half layout, (2 i, 2 i + 1) interleaved;
// dims rot .. dim - 1 pass unchanged.  The transposed turn takes -s: the
// gradient of the turn.  cos and sin come from a table in fp32, computed in
// 64 bits (an angle of position 10^5 taken in fp32 would be off by up to
// 4e-3), so a result is two products and a sum in fp32, rounded once more
// only to a narrower destination.
//
// An append turns the keys of the new rows into their cache slots, copies the
// values there (rounding to the cache's type) and turns the queries of the
// same rows, in one launch: all three lie side by side in what a qkv linear
// gives, and a second and third launch would cost more than the work of a
// decode step.
//
// Bandwidth-bound: every element is read and written once.  A thread keeps
// one place in the row (four pairs, or eight plain elements: two loads of
// four elements, 16 bytes in fp32) and walks over heads of one token, so that
// 16 lanes cover a head of 128 contiguously and cos and sin are read once a
// token.  4096 tokens of 32 heads of 128, fp32 to fp16: 19 us, 5.4 TB/s (a
// large copy: 5.2); ragged prompts of 16 + 32 heads of 64 appended in fp32:
// 11.7 us, 5.0 TB/s; one token, or a decode step's append: 2.2 and 3.0 us on
// the device, a launch.  Loads past the caches gain a tenth where the rows
// come from memory, but lose as much or more where they are still in the last
// level of cache (1000 tokens: 7.1 -> 8.4 us), as what a linear has just
// written is.
#include "kcommon.h"
#include "serving.h"
#include "nnjit.h"

namespace nnjit {

namespace {

template <typename T>
using vec4 = T __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

template <typename S, typename D, bool APPEND, int V>   // V: pairs of a unit (4, or 1 from any address)
__global__ void __launch_bounds__(kThreads)
rotary_kernel(RotaryParams p)
{
    const int t = blockIdx.x;
    int pos = 0;
    D *kdst = nullptr, *vdst = nullptr;
    if constexpr (APPEND) {
        // the sequence that holds row t: the starts up to t, counted 64 at a time
        const int lane = threadIdx.x & 63;
        const PageBatch &b = p.batch;
        if (t < b.q_start[0]) return;
        int seq = 0;
        for (int i = 1; i <= b.sequences; i += 64) {
            const int s = i + lane;
            const unsigned long long before = __ballot(s <= b.sequences && b.q_start[min(s, b.sequences)] <= t);
            seq += __popcll(before);
            if (before != ~0ull) break;
        }
        if (seq >= b.sequences) return;                  // a row behind the last sequence
        const int begin = b.q_start[seq], end = b.q_start[seq + 1];
        pos = b.kv_len[seq] - (end - begin) + (t - begin);
        const int pi = pos < 0 ? -1 : p.pool.page_size.quot(pos);
        if (pi >= 0 && pi < b.table_pages) {
            const int page = b.page_table[(long long)seq * b.ld_table + pi];
            if (page >= 0 && page < p.pool.pages) {
                const int slot = pos - pi * (int)p.pool.page_size.d;
                kdst = (D *)p.pool.k + page_offset(page, p.pool.k_page, slot, p.pool.k_tok);
                vdst = (D *)p.pool.v + page_offset(page, p.pool.v_page, slot, p.pool.v_tok);
            }
        }
    } else {
        pos = p.positions[t];
    }
    pos = min(max(pos, 0), p.table_rows - 1);

    const int turned = p.rot / (2 * V);                              // units that are turned
    const int units = turned + (p.dim - p.rot) / (V == 4 ? 8 : 1);
    const int rows = kThreads / units;                               // heads at a time
    const int u = threadIdx.x % units, r0 = threadIdx.x / units;
    if (r0 >= rows) return;

    // first elements of the unit's two parts, in the row and in the table
    const bool turn = u < turned;
    const int a = turn ? (p.interleaved ? 2 * V * u : V * u) : p.rot + (u - turned) * (V == 4 ? 8 : 1);
    const int b = V == 1 ? (turn ? (p.interleaved ? a + 1 : a + p.rot / 2) : a)
                         : (turn && !p.interleaved ? a + p.rot / 2 : a + 4);
    float c[V], s[V];
    if (turn) {
        const float *row = p.table + (long long)pos * p.rot + V * u;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            c[e] = row[e];
            s[e] = p.sign * row[p.rot / 2 + e];
        }
    }

    auto one = [&](const S *x, D *y, bool do_turn) {
        if constexpr (V == 4) {
            typedef vec4<S> s4;
            typedef vec4<D> d4;
            const s4 xa = *(const s4 *)(x + a), xb = *(const s4 *)(x + b);
            f32x4 fa = __builtin_convertvector(xa, f32x4), fb = __builtin_convertvector(xb, f32x4);
            if (do_turn) {
                if (p.interleaved) {
                    const f32x4 ea = {fa[0], fa[2], fb[0], fb[2]}, eb = {fa[1], fa[3], fb[1], fb[3]};
                    f32x4 ta, tb;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ta[e] = ea[e] * c[e] - eb[e] * s[e];
                        tb[e] = eb[e] * c[e] + ea[e] * s[e];
                    }
                    fa = f32x4{ta[0], tb[0], ta[1], tb[1]};
                    fb = f32x4{ta[2], tb[2], ta[3], tb[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float xa1 = fa[e], xb1 = fb[e];
                        fa[e] = xa1 * c[e] - xb1 * s[e];
                        fb[e] = xb1 * c[e] + xa1 * s[e];
                    }
                }
            }
            *(d4 *)(y + a) = __builtin_convertvector(fa, d4);
            *(d4 *)(y + b) = __builtin_convertvector(fb, d4);
        } else {
            const float fa = (float)x[a], fb = (float)x[b];
            y[a] = (D)(do_turn ? fa * c[0] - fb * s[0] : fa);
            if (do_turn) y[b] = (D)(fb * c[0] + fa * s[0]);
            else if (turn) y[b] = (D)fb;
        }
    };

    const int heads = p.q_heads + 2 * p.kv_heads;
    const int first = blockIdx.y * p.heads_per_block;
    const int last = min(heads, first + p.heads_per_block);
    for (int h = first + r0; h < last; h += rows) {
        if (h < p.q_heads) {
            one((const S *)p.q.p + (long long)t * p.q.tok + (long long)h * p.q.head,
                (D *)p.qo.p + (long long)t * p.qo.tok + (long long)h * p.qo.head, turn);
        } else if constexpr (APPEND) {
            const bool is_v = h >= p.q_heads + p.kv_heads;
            const int kh = h - p.q_heads - (is_v ? p.kv_heads : 0);
            if (!kdst) continue;
            const HeadRows &src = is_v ? p.v : p.k;
            D *dst = is_v ? vdst + (long long)kh * p.pool.v_head : kdst + (long long)kh * p.pool.k_head;
            one((const S *)src.p + (long long)t * src.tok + (long long)kh * src.head, dst, turn && !is_v);
        }
    }
}

// table[p][i] = m cos(p f_i), table[p][rot / 2 + i] = m sin(p f_i), all in 64 bits
// until the last rounding.  f_i = base^(-2 i / rot), scaled (include/nnjit.h).
__global__ void __launch_bounds__(kThreads)
rotary_table_kernel(float *table, int positions, int rot, double base, int scaling, double factor, double original,
                    double fast, double slow, double magnitude)
{
    const long long n = (long long)positions * (rot / 2);
    const long long at = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (at >= n) return;
    const int half = rot / 2;
    const int i = (int)(at % half);
    const long long pos = at / half;
    const double two_pi = 6.283185307179586476925286766559;
    if (scaling == NNJIT_ROTARY_BASE && rot > 2) base *= pow(factor, (double)rot / (rot - 2));
    double f = pow(base, -2.0 * i / rot);
    if (scaling == NNJIT_ROTARY_LINEAR) {
        f /= factor;
    } else if (scaling == NNJIT_ROTARY_TURNS) {
        const double turns = original * f / two_pi;
        const double keep = fmin(fmax((turns - slow) / (fast - slow), 0.0), 1.0);
        f = f * keep + f / factor * (1.0 - keep);
    } else if (scaling == NNJIT_ROTARY_INDEX) {
        // pair index (not rounded) whose frequency turns `n` times over the original positions
        const double lb = 2.0 * log(base);
        const double lo = fmax(floor(rot * log(original / (fast * two_pi)) / lb), 0.0);
        const double hi = fmin(ceil(rot * log(original / (slow * two_pi)) / lb), rot - 1.0);
        const double slowed = fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
        f = f * (1.0 - slowed) + f / factor * slowed;
    }
    double sn, cs;
    sincos((double)pos * f, &sn, &cs);
    table[pos * rot + i] = (float)(magnitude * cs);
    table[pos * rot + half + i] = (float)(magnitude * sn);
}

template <typename S, typename D>
hipError_t launch_as(const RotaryParams &p, bool append, bool vec, dim3 grid, hipStream_t stream)
{
    if (append) {
        if (vec) rotary_kernel<S, D, true, 4><<<grid, kThreads, 0, stream>>>(p);
        else rotary_kernel<S, D, true, 1><<<grid, kThreads, 0, stream>>>(p);
    } else {
        if (vec) rotary_kernel<S, D, false, 4><<<grid, kThreads, 0, stream>>>(p);
        else rotary_kernel<S, D, false, 1><<<grid, kThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary_table(float *table, int positions, int rot, double base, int scaling, double factor,
                               double original, double fast, double slow, double magnitude, hipStream_t stream)
{
    const long long n = (long long)positions * (rot / 2);
    rotary_table_kernel<<<dim3((unsigned)((n + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(
        table, positions, rot, base, scaling, factor, original, fast, slow, magnitude);
    return hipGetLastError();
}

hipError_t launch_rotary(const RotaryParams &in, bool append, int src_dtype, int dst_dtype, bool vec, hipStream_t stream)
{
    RotaryParams p = in;
    const int heads = p.q_heads + 2 * p.kv_heads;
    const int units = vec ? p.dim / 8 : p.rot / 2 + (p.dim - p.rot);
    const int rows = kThreads / units;
    // few tokens: their heads are spread over workgroups until about four
    // workgroups a compute unit are there; many tokens: one workgroup each
    // (one, two, four or eight a compute unit: alike to 0.1 us from 1 to 4096 tokens;
    // sixteen: 11.0 -> 11.9 for 2048 tokens appended)
    const int most = (heads + rows - 1) / rows;
    const int want = (1024 + p.tokens - 1) / p.tokens;
    const int blocks = want < most ? want : most;
    p.heads_per_block = (heads + blocks - 1) / blocks;
    p.heads_per_block = (p.heads_per_block + rows - 1) / rows * rows;
    const dim3 grid((unsigned)p.tokens, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
    if (src_dtype == NNJIT_F32)
        return dst_dtype == NNJIT_F32 ? launch_as<float, float>(p, append, vec, grid, stream)
                                      : launch_as<float, _Float16>(p, append, vec, grid, stream);
    return dst_dtype == NNJIT_F32 ? launch_as<_Float16, float>(p, append, vec, grid, stream)
                                  : launch_as<_Float16, _Float16>(p, append, vec, grid, stream);
}

}  // namespace nnjit
