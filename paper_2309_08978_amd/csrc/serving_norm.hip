// Norms of heads with the turn of their positions in the same pass: appends
// to a paged cache, and the forward and backward pass of training.
//
//   y = R_p (x r w),   r = (mean of x^2 + eps)^(-1/2)
//
// with R_p the turn of rotary.hip.  Backward, with g = R_p^T dy:
//   dx = r (g w - x r mean(g w x r)),   dw = sum over rows of g x r.
// mean(x^2) and mean(g w x) are summed in the same pass over the row.
//
// A group of LPH lanes takes a head row, eight elements a lane -- the two sides
// of four turned pairs, or eight neighbours that are not turned -- so a row is
// loaded once, its sums take log2 LPH exchanges and it is stored from the
// registers that it was loaded to.  Rows of any alignment and dims that are no
// multiple of eight: 64 lanes a head, an element or pair at a time.
//
// Bandwidth-bound once the vector instructions are few: 4096 tokens of 32 heads of 128 in fp16
// forward 13.2 us, 5.1 TB/s, one pass after the other of its kind, and 15.3 between backward passes over other operands;
// backward 19.9, 5.1 (a large copy: 5.0), plus 3.9 to 4.6 for the sum of the partial gradients;
// 2930 rows (and 37 of padding) of 32 query and 8 key and value heads appended, fp32 to fp16: 23.5 us a call, 4.7
// TB/s; one token's append 3.2 on the device.  (With 230 instructions a row of eight elements a lane -- both layouts in one
// kernel, weights and angles by single loads -- forward took 31 us, backward 36.)
//
// The weight's gradient is summed in registers over the rows of a workgroup, then over
// its groups through LDS, then by a second launch over workgroups: in an order that
// sizes, strides and alignment decide.
#include <type_traits>

#include "kcommon.h"
#include "serving.h"
#include "nnjit.h"

namespace nnjit {

namespace {

template <typename T>
using vec4 = T __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// Where a lane's eight elements lie: lo[e] at a(e), hi[e] at b(e), the sides of a
// pair where turned.  HALF, PAIRS (the two layouts): e are neighbours; ANY (either layout, any address): unit
// u + 64 e of a row of pairs and, behind them, single elements (hi[e] is then none).
enum { HALF, PAIRS, ANY };

template <int HOW>
struct Place {
    static constexpr bool VEC = HOW != ANY;
    int u, units, turned, rot, interleaved;
    bool mine;                 // VEC: the row has elements for this lane (else it loads the last ones', and stores none)
    __device__ __forceinline__ Place(const NormParams &p, int lane)
    {
        rot = p.table ? p.rot : 0;
        interleaved = p.interleaved;
        turned = VEC ? rot / 8 : rot / 2;
        units = VEC ? p.dim / 8 : turned + p.dim - rot;
        mine = lane < units;
        u = VEC ? min(lane, units - 1) : lane;
    }
    __device__ __forceinline__ int unit(int e) const { return VEC ? u : u + 64 * e; }
    __device__ __forceinline__ bool has(int e) const { return VEC || unit(e) < units; }
    __device__ __forceinline__ bool turn(int e) const { return unit(e) < turned; }
    __device__ __forceinline__ bool has_hi(int e) const { return VEC || turn(e); }
    // VEC: first elements of the two runs of four; else the elements themselves
    __device__ __forceinline__ int a(int e) const
    {
        if (HOW == HALF) return turn(0) ? 4 * u : 8 * u;                       // (rot = 8 turned)
        if (HOW == PAIRS) return 8 * u;
        const int i = unit(e);
        return turn(e) ? (interleaved ? 2 * i : i) : rot + i - turned;
    }
    __device__ __forceinline__ int b(int e) const
    {
        if (HOW == HALF) return turn(0) ? 4 * u + rot / 2 : 8 * u + 4;
        if (HOW == PAIRS) return 8 * u + 4;
        return interleaved ? a(e) + 1 : a(e) + rot / 2;
    }

    // a row's elements as they lie, so that several rows' loads can be on their way
    template <typename S>
    struct Raw {
        vec4<S> a, b;
    };
    template <typename S>
    __device__ __forceinline__ Raw<S> fetch(const S *x) const
    {
        Raw<S> r;
        if constexpr (VEC) {
            r.a = *(const vec4<S> *)(x + a(0));
            r.b = *(const vec4<S> *)(x + b(0));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                r.a[e] = has(e) ? x[a(e)] : (S)0;
                r.b[e] = has_hi(e) ? x[b(e)] : (S)0;
            }
        }
        return r;
    }
    template <typename S>
    __device__ __forceinline__ void unpack(const Raw<S> &r, float *lo, float *hi) const
    {
        const f32x4 fa = __builtin_convertvector(r.a, f32x4), fb = __builtin_convertvector(r.b, f32x4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = HOW == PAIRS ? (e < 2 ? fa[2 * e & 3] : fb[2 * e & 3]) : fa[e];
            hi[e] = HOW == PAIRS ? (e < 2 ? fa[(2 * e + 1) & 3] : fb[(2 * e + 1) & 3]) : fb[e];
        }
    }
    template <typename S>
    __device__ __forceinline__ void load(const S *x, float *lo, float *hi) const { unpack(fetch(x), lo, hi); }
    template <typename D>
    __device__ __forceinline__ void store(D *y, const float *lo, const float *hi) const
    {
        if constexpr (VEC) {
            const f32x4 fa = HOW == PAIRS ? f32x4{lo[0], hi[0], lo[1], hi[1]} : f32x4{lo[0], lo[1], lo[2], lo[3]};
            const f32x4 fb = HOW == PAIRS ? f32x4{lo[2], hi[2], lo[3], hi[3]} : f32x4{hi[0], hi[1], hi[2], hi[3]};
            if (!mine) return;
            *(vec4<D> *)(y + a(0)) = __builtin_convertvector(fa, vec4<D>);
            *(vec4<D> *)(y + b(0)) = __builtin_convertvector(fb, vec4<D>);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (has(e)) y[a(e)] = (D)lo[e];
                if (has_hi(e)) y[b(e)] = (D)hi[e];
            }
        }
    }
    __device__ __forceinline__ void load_weight(const void *w, long long element, int half, float *lo, float *hi) const
    {
        if (half) load((const _Float16 *)w + element, lo, hi);
        else load((const float *)w + element, lo, hi);
    }
    __device__ __forceinline__ void load_angles(const NormParams &p, int position, float *c, float *s) const
    {
        const float *row = p.table + (long long)min(max(position, 0), p.table_rows - 1) * rot;
        if constexpr (VEC) {
            if (!turn(0)) return;
            const f32x4 fc = *(const f32x4 *)(row + 4 * u), fs = *(const f32x4 *)(row + rot / 2 + 4 * u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                c[e] = fc[e];
                s[e] = fs[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                c[e] = turn(e) ? row[unit(e)] : 1.f;
                s[e] = turn(e) ? row[rot / 2 + unit(e)] : 0.f;
            }
        }
    }
    // lo, hi turned by the angles, or (BACK) by the opposite ones
    template <bool BACK>
    __device__ __forceinline__ void rotate(float *lo, float *hi, const float *c, const float *s) const
    {
        if (VEC && !turn(0)) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!VEC && !turn(e)) continue;
            const float l = lo[e], k = hi[e];
            const float sn = BACK ? -s[e] : s[e];
            lo[e] = fmaf(l, c[e], -(k * sn));
            hi[e] = fmaf(k, c[e], l * sn);
        }
    }
    // a lane's part of a row's sum
    __device__ __forceinline__ float part(float sum) const { return !VEC || mine ? sum : 0.f; }
};

// Sum over the LPH lanes of a group, in all of them.  Up to 16 lanes, a row of
// the wave, by lane permutations of the additions' operands; beyond by exchanges.
template <int HOW>
__device__ __forceinline__ float permuted(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), HOW, 0xf, 0xf, true));
}
template <int LPH>
__device__ __forceinline__ float group_sum(float v)
{
    v += permuted<0xb1>(v);                 // neighbours: lanes 1 0 3 2
    v += permuted<0x4e>(v);                 // lanes 2 3 0 1
    v += permuted<0x141>(v);                // eight lanes mirrored: their halves, alike inside by now
    if constexpr (LPH >= 16) v += permuted<0x140>(v);   // the row mirrored
    if constexpr (LPH >= 32) v += __shfl_xor(v, 16);
    if constexpr (LPH >= 64) v += __shfl_xor(v, 32);
    return v;
}

__device__ __forceinline__ float norm_scale(const NormParams &p, float squares) { return rsqrtf(squares * p.one_by_dim + p.eps); }

// row h of strided ones (strides of rows taken eight elements a lane are below 2^32)
template <bool VEC, typename T>
__device__ __forceinline__ T *row_of(T *base, int h, long long stride)
{
    return base + (VEC ? (unsigned long long)(unsigned)h * (unsigned)stride : (unsigned long long)(h * stride));
}

// A workgroup takes p.tokens_per_block tokens (a power of two), its groups split evenly among
// them, so that a group has a few heads of one token: their loads are on their
// way together, and angles are read once.
template <typename S, typename D, bool APPEND, int HOW, int LPH>
__global__ void __launch_bounds__(kThreads)
norm_rotary_kernel(NormParams p)
{
    constexpr int GROUPS = kThreads / LPH;
    const int groups = GROUPS / p.tokens_per_block;         // of a token
    const int in_block = threadIdx.x / LPH / groups, group = threadIdx.x / LPH % groups;
    const int t = min((int)blockIdx.x * p.tokens_per_block + in_block, p.tokens - 1);
    bool live = (int)blockIdx.x * p.tokens_per_block + in_block < p.tokens;
    constexpr bool VEC = HOW != ANY;
    const Place<HOW> at(p, threadIdx.x % LPH);
    D *kdst = nullptr, *vdst = nullptr;
    if constexpr (APPEND) {
        // (rows that are left alone are read and normed all the same: no load waits for the slot)
        const long long slot = p.slots[t];
        live &= slot >= 0 && slot < (long long)p.pool.pages * p.pool.page_size.d;
        const unsigned page_size = p.pool.page_size.d;
        const int page = live ? (int)(slot / page_size) : 0, in = live ? (int)(slot - (long long)page * page_size) : 0;
        kdst = (D *)p.pool.k + page_offset(page, p.pool.k_page, in, p.pool.k_tok);
        vdst = (D *)p.pool.v + page_offset(page, p.pool.v_page, in, p.pool.v_tok);
    }
    float c[4], s[4], ql[4], qh[4], kl[4], kh[4];
    if (p.table) at.load_angles(p, p.positions[t], c, s);
    const bool one_weight = (!p.q_weight || p.qw_head == 0) && (!p.k_weight || p.kw_head == 0);
    if (one_weight && p.q_weight) at.load_weight(p.q_weight, 0, p.weight_half, ql, qh);
    if (APPEND && one_weight && p.k_weight) at.load_weight(p.k_weight, 0, p.weight_half, kl, kh);

    const int heads = p.q_heads + 2 * p.kv_heads;
    const int first = blockIdx.y * p.heads_per_block, last = min(heads, first + p.heads_per_block);
    // norm and turn of a row, in place; element: of a weight a head
    auto finish = [&](float *lo, float *hi, const void *weight, const float *wl, const float *wh, long long element) {
        if (weight) {
            float squares = 0.f, own_l[4], own_h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) squares += lo[e] * lo[e] + hi[e] * hi[e];
            const float r = norm_scale(p, group_sum<LPH>(at.part(squares)));
            if (!one_weight) at.load_weight(weight, element, p.weight_half, own_l, own_h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = lo[e] * r * (one_weight ? wl[e] : own_l[e]);
                hi[e] = hi[e] * r * (one_weight ? wh[e] : own_h[e]);
            }
        }
        if (p.table) at.template rotate<false>(lo, hi, c, s);
    };

    // rows of a group whose loads are on their way together: of queries, of keys and values
    constexpr int AHEAD = !VEC ? 1 : sizeof(S) == 4 ? 2 : 4, AHEAD_KV = VEC && sizeof(S) == 2 ? 2 : 1;
    typename Place<HOW>::template Raw<S> raw[AHEAD], raw_kv[AHEAD_KV];
    const int kv_last = APPEND ? last - p.q_heads : 0;
    auto fetch_kv = [&](int r0) {
#pragma unroll
        for (int j = 0; j < AHEAD_KV; ++j) {
            const int r = r0 + j * groups;
            if (r >= kv_last) continue;
            const bool is_v = r >= p.kv_heads;
            const S *row = is_v ? (const S *)p.v.p + (long long)t * p.v.tok : (const S *)p.k.p + (long long)t * p.k.tok;
            raw_kv[j] = at.fetch(row_of<VEC>(row, is_v ? r - p.kv_heads : r, is_v ? p.v.head : p.k.head));
        }
    };
    int r0 = max(first - p.q_heads, 0) + group;
    if (APPEND) fetch_kv(r0);

    const S *q_src = (const S *)p.q.p + (long long)t * p.q.tok;
    D *q_dst = (D *)p.qo.p + (long long)t * p.qo.tok;
    const int q_last = min(last, p.q_heads);
    for (int h0 = first + group; h0 < q_last; h0 += AHEAD * groups) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (h0 + j * groups < q_last) raw[j] = at.fetch(row_of<VEC>(q_src, h0 + j * groups, p.q.head));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int h = h0 + j * groups;
            if (h >= q_last) continue;                     // (the same in all lanes of a group, as all below)
            float lo[4], hi[4];
            at.unpack(raw[j], lo, hi);
            finish(lo, hi, p.q_weight, ql, qh, h * p.qw_head);
            if (live) at.store(row_of<VEC>(q_dst, h, p.qo.head), lo, hi);
        }
    }
    if constexpr (APPEND) {
        for (; r0 < kv_last; r0 += AHEAD_KV * groups) {
            if (r0 >= max(first - p.q_heads, 0) + AHEAD_KV * groups) fetch_kv(r0);
#pragma unroll
            for (int j = 0; j < AHEAD_KV; ++j) {
                const int r = r0 + j * groups;
                if (r >= kv_last) continue;
                float lo[4], hi[4];
                at.unpack(raw_kv[j], lo, hi);
                if (r < p.kv_heads) {
                    finish(lo, hi, p.k_weight, kl, kh, r * p.kw_head);
                    if (live) at.store(row_of<VEC>(kdst, r, p.pool.k_head), lo, hi);
                } else {
                    if (live) at.store(row_of<VEC>(vdst, r - p.kv_heads, p.pool.v_head), lo, hi);
                }
            }
        }
    }
}

constexpr int kGradThreads = 512;

// A workgroup takes a run of p.chunk tokens, p.tokens_per_block at a time, its groups split
// among them as in the forward pass.  PER_HEAD: p.heads_per_block heads (from blockIdx.y's first on), each
// group always the same one, so that its sum is that head's.
template <typename X, typename Y, bool PER_HEAD, int HOW, int LPH>
__global__ void __launch_bounds__(kGradThreads)
norm_rotary_grad_kernel(NormParams p)
{
    constexpr int GROUPS = kGradThreads / LPH;
    __shared__ __attribute__((aligned(16))) float sums[GROUPS][LPH * 8];
    const int lane = threadIdx.x % LPH, groups = GROUPS / p.tokens_per_block;       // of a token
    const int in_block = threadIdx.x / LPH / groups, group = threadIdx.x / LPH % groups;
    constexpr bool VEC = HOW != ANY;
    const Place<HOW> at(p, lane);
    const int h_first = PER_HEAD ? blockIdx.y * p.heads_per_block : 0;
    const int h_last = PER_HEAD ? min(h_first + p.heads_per_block, p.q_heads) : p.q_heads;
    float wl[4], wh[4], dl[4] = {}, dh[4] = {};
    const int w_head = PER_HEAD ? min(h_first + group, h_last - 1) : 0;
    at.load_weight(p.q_weight, w_head * p.qw_head, p.weight_half, wl, wh);

    // a row: its part of dw, and dx
    auto row = [&](const typename Place<HOW>::template Raw<X> &x, const typename Place<HOW>::template Raw<Y> &y, const float *c, const float *s, X *dx) {
        float xl[4], xh[4], gl[4], gh[4], squares = 0.f, dots = 0.f;
        at.unpack(x, xl, xh);
        at.unpack(y, gl, gh);
        if (p.table) at.template rotate<true>(gl, gh, c, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            squares += xl[e] * xl[e] + xh[e] * xh[e];
            dots += gl[e] * wl[e] * xl[e] + gh[e] * wh[e] * xh[e];
        }
        const float r = norm_scale(p, group_sum<LPH>(at.part(squares))), m = group_sum<LPH>(at.part(dots)) * r * p.one_by_dim;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ul = xl[e] * r, uh = xh[e] * r;
            dl[e] += gl[e] * ul;
            dh[e] += gh[e] * uh;
            gl[e] = r * (gl[e] * wl[e] - ul * m);
            gh[e] = r * (gh[e] * wh[e] - uh * m);
        }
        if (p.qo.p) at.store(dx, gl, gh);
    };
    auto x_row = [&](int t) { return (const X *)p.q.p + (long long)t * p.q.tok; };
    auto y_row = [&](int t) { return (const Y *)p.dy.p + (long long)t * p.dy.tok; };
    auto dx_row = [&](int t) { return (X *)p.qo.p + (long long)t * p.qo.tok; };

    const int first = blockIdx.x * p.chunk, last = min(p.tokens, first + p.chunk);
    if constexpr (PER_HEAD) {
        // a group's head is always the same: tokens are what it has loads ahead of
        constexpr int AHEAD = VEC ? 3 : 1;
        const int h = h_first + group;
        for (int t0 = first + in_block; t0 < last && h < h_last; t0 += AHEAD * p.tokens_per_block) {      // (the same in all lanes of a group)
            typename Place<HOW>::template Raw<X> x[AHEAD];
            typename Place<HOW>::template Raw<Y> y[AHEAD];
            float c[AHEAD][4], s[AHEAD][4];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int t = min(t0 + j * p.tokens_per_block, last - 1);
                x[j] = at.fetch(row_of<VEC>(x_row(t), h, p.q.head));
                y[j] = at.fetch(row_of<VEC>(y_row(t), h, p.dy.head));
                if (p.table) at.load_angles(p, p.positions[t], c[j], s[j]);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int t = t0 + j * p.tokens_per_block;
                if (t < last) row(x[j], y[j], c[j], s[j], row_of<VEC>(dx_row(t), h, p.qo.head));
            }
        }
    } else {
        constexpr int AHEAD = VEC ? 4 : 1;
        for (int t = first + in_block; t < last; t += p.tokens_per_block) {
            float c[4], s[4];
            if (p.table) at.load_angles(p, p.positions[t], c, s);
            for (int h0 = group; h0 < p.q_heads; h0 += AHEAD * groups) {
                typename Place<HOW>::template Raw<X> x[AHEAD];
                typename Place<HOW>::template Raw<Y> y[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const int h = h0 + j * groups;
                    if (h >= p.q_heads) continue;
                    x[j] = at.fetch(row_of<VEC>(x_row(t), h, p.q.head));
                    y[j] = at.fetch(row_of<VEC>(y_row(t), h, p.dy.head));
                }
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const int h = h0 + j * groups;
                    if (h < p.q_heads) row(x[j], y[j], c, s, row_of<VEC>(dx_row(t), h, p.qo.head));
                }
            }
        }
    }
    if (!p.dw) return;
    at.store(sums[threadIdx.x / LPH], dl, dh);
    __syncthreads();
    // per head: group g of every token is head h_first + g
    const int out = PER_HEAD ? h_last - h_first : 1;
    for (int i = threadIdx.x; i < out * p.dim; i += kGradThreads) {
        const int g0 = PER_HEAD ? i / p.dim : 0, d = i - g0 * p.dim;
        float sum = 0.f;
        for (int g = g0; g < GROUPS; g += PER_HEAD ? groups : 1) sum += sums[g][d];
        (gridDim.x == 1 ? p.dw : p.part)[((long long)blockIdx.x * (PER_HEAD ? p.q_heads : 1) + h_first + g0) * p.dim + d] = sum;
    }
}

// dw[i] = sum over groups of part[group][i], i < n: 32 columns a workgroup, 32 slices of the groups.
__global__ void __launch_bounds__(1024)
sum_parts_kernel(const float *part, float *dw, int groups, long long n)
{
    __shared__ float sums[32][33];
    const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const long long i = (long long)blockIdx.x * 32 + col;
    float sum = 0.f;
    if (i < n) {
#pragma unroll 8
        for (int g = slice; g < groups; g += 32) sum += part[g * n + i];
    }
    sums[slice][col] = sum;
    __syncthreads();
    if (slice == 0 && i < n) {
        float total = 0.f;
#pragma unroll
        for (int s = 0; s < 32; ++s) total += sums[s][col];
        dw[i] = total;
    }
}

int lanes_per_head(int dim, bool vec) { return !vec ? 64 : dim <= 64 ? 8 : dim <= 128 ? 16 : 32; }

// launch(how, lanes) with both as constants
template <typename F>
void pick(const NormParams &p, bool vec, F launch)
{
    using std::integral_constant;
    const int lanes = lanes_per_head(p.dim, vec);
    auto of = [&](auto how) {
        if (lanes == 8) launch(how, integral_constant<int, 8>{});
        else if (lanes == 16) launch(how, integral_constant<int, 16>{});
        else launch(how, integral_constant<int, 32>{});
    };
    if (!vec) launch(integral_constant<int, ANY>{}, integral_constant<int, 64>{});
    else if (p.interleaved) of(integral_constant<int, PAIRS>{});
    else of(integral_constant<int, HALF>{});
}

template <typename S, typename D, bool APPEND>
hipError_t launch_as(const NormParams &p, bool vec, dim3 grid, hipStream_t stream)
{
    pick(p, vec, [&](auto how, auto lanes) { norm_rotary_kernel<S, D, APPEND, how(), lanes()><<<grid, kThreads, 0, stream>>>(p); });
    return hipGetLastError();
}

template <typename S, typename D>
hipError_t launch_typed(const NormParams &p, bool append, bool vec, dim3 grid, hipStream_t stream)
{
    return append ? launch_as<S, D, true>(p, vec, grid, stream) : launch_as<S, D, false>(p, vec, grid, stream);
}

template <typename X, typename Y, bool PER_HEAD>
hipError_t launch_grad_as(const NormParams &p, bool vec, dim3 grid, hipStream_t stream)
{
    pick(p, vec, [&](auto how, auto lanes) { norm_rotary_grad_kernel<X, Y, PER_HEAD, how(), lanes()><<<grid, kGradThreads, 0, stream>>>(p); });
    return hipGetLastError();
}

template <typename X, typename Y>
hipError_t launch_grad_typed(const NormParams &p, bool vec, int groups, hipStream_t stream)
{
    const unsigned blocks = (unsigned)((p.q_heads + p.heads_per_block - 1) / p.heads_per_block);
    return p.qw_head > 0 ? launch_grad_as<X, Y, true>(p, vec, dim3((unsigned)groups, blocks), stream)
                         : launch_grad_as<X, Y, false>(p, vec, dim3((unsigned)groups), stream);
}

// Tokens that the groups of a workgroup are split among, so that a group has about `rows` heads.
int tokens_per_block(int groups, int heads, int rows)
{
    int t = 1;
    while (2 * t <= groups && groups / (2 * t) * rows >= heads) t *= 2;
    return t;
}

// ... per head: a group a head, if there are so many groups
int tokens_per_block_of_heads(int groups, int heads)
{
    int t = 1;
    while (2 * t <= groups && groups / (2 * t) >= heads) t *= 2;
    return t;
}

}  // namespace

hipError_t launch_norm_rotary(const NormParams &in, bool append, int src_dtype, int dst_dtype, bool vec, hipStream_t stream)
{
    NormParams p = in;
    p.one_by_dim = 1.f / (float)p.dim;
    const int heads = p.q_heads + 2 * p.kv_heads, groups = kThreads / lanes_per_head(p.dim, vec);
    // few tokens: their heads are spread over workgroups until about four a compute unit are there
    const int most = (heads + groups - 1) / groups, want = (1024 + p.tokens - 1) / p.tokens, blocks = want < most ? want : most;
    p.heads_per_block = (heads + blocks - 1) / blocks;
    p.heads_per_block = (p.heads_per_block + groups - 1) / groups * groups;
    // (4096 tokens of 32 heads of 128: in fp16 13.5 us with two heads a group, 13.1 with four, 12.8 with eight; in fp32 28.2, 30.6, 32.7)
    p.tokens_per_block = blocks == 1 && p.tokens >= 1024 ? tokens_per_block(groups, append ? p.q_heads > 2 * p.kv_heads ? p.q_heads : 2 * p.kv_heads : heads, src_dtype == NNJIT_F32 ? 2 : 4) : 1;
    const dim3 grid((unsigned)((p.tokens + p.tokens_per_block - 1) / p.tokens_per_block), (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
    if (src_dtype == NNJIT_F32)
        return dst_dtype == NNJIT_F32 ? launch_typed<float, float>(p, append, vec, grid, stream)
                                      : launch_typed<float, _Float16>(p, append, vec, grid, stream);
    return dst_dtype == NNJIT_F32 ? launch_typed<_Float16, float>(p, append, vec, grid, stream)
                                  : launch_typed<_Float16, _Float16>(p, append, vec, grid, stream);
}

int norm_grad_groups(int64_t tokens, int64_t heads, int dim, bool per_head, bool vec, int cus)
{
    const int groups = kGradThreads / lanes_per_head(dim, vec);
    const int64_t at_once = per_head ? tokens_per_block_of_heads(groups, (int)heads) : tokens_per_block(groups, (int)heads, 4);
    const int64_t blocks = per_head ? (heads * at_once + groups - 1) / groups : 1;           // of heads
    // (up to two runs by a lone workgroup, which needs no second launch: 8 tokens of 32 heads 7.2 us, with one 10; but
    // 20 tokens, five runs, 14.7 alone and 10.2 by five)
    const int64_t runs = (tokens + at_once - 1) / at_once, want = runs <= 2 ? 1 : runs;
    // Two workgroups a compute unit; per head, where each adds heads * dim partial sums to write and read again, only if that
    // leaves runs of eight or more (32 heads of 128 in fp16: 500 tokens 11.3 us by 256, by 500 16.6; 4096 tokens 34.0 and 30.5)
    const int64_t wanted = per_head && runs < 16ll * cus ? cus : 2ll * cus, most = (wanted + blocks - 1) / blocks;
    return (int)(want < 1 ? 1 : want < most ? want : most);      // (no tokens: one adds up nothing)
}

hipError_t launch_norm_rotary_grad(const NormParams &in, int x_dtype, int dy_dtype, bool vec, int groups, hipStream_t stream)
{
    NormParams p = in;
    p.one_by_dim = 1.f / (float)p.dim;
    const int at_once = kGradThreads / lanes_per_head(p.dim, vec);
    p.tokens_per_block = p.qw_head > 0 ? tokens_per_block_of_heads(at_once, p.q_heads) : tokens_per_block(at_once, p.q_heads, 4);
    p.heads_per_block = at_once / p.tokens_per_block;
    p.chunk = (p.tokens + groups - 1) / groups;
    hipError_t e;
    if (x_dtype == NNJIT_F32)
        e = dy_dtype == NNJIT_F32 ? launch_grad_typed<float, float>(p, vec, groups, stream) : launch_grad_typed<float, _Float16>(p, vec, groups, stream);
    else
        e = dy_dtype == NNJIT_F32 ? launch_grad_typed<_Float16, float>(p, vec, groups, stream)
                                  : launch_grad_typed<_Float16, _Float16>(p, vec, groups, stream);
    if (e != hipSuccess || !p.dw || groups == 1) return e;
    const long long n = (long long)p.dim * (p.qw_head > 0 ? p.q_heads : 1);
    sum_parts_kernel<<<dim3((unsigned)((n + 31) / 32)), 1024, 0, stream>>>(p.part, p.dw, groups, n);
    return hipGetLastError();
}

}  // namespace nnjit
