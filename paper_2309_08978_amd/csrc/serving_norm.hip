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
// The weight's gradient is summed in registers over the rows of a workgroup, then over
// its groups through LDS, then by a second launch over workgroups: in an order
// that the sizes alone decide.
#include "kcommon.h"
#include "serving.h"
#include "nnjit.h"

namespace nnjit {

namespace {

template <typename T>
using vec4 = T __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// Where a lane's eight elements lie: lo[e] at a(e), hi[e] at b(e), the sides of a
// pair where turned.  VEC: e neighbours; else unit u + 64 e of a row of pairs and, behind
// them, single elements (hi[e] is then none).
template <bool VEC>
struct Place {
    int u, units, turned, rot, dim, interleaved;
    __device__ __forceinline__ Place(const NormParams &p, int lane)
    {
        u = lane;
        rot = p.table ? p.rot : 0;
        dim = p.dim;
        interleaved = p.interleaved;
        turned = VEC ? rot / 8 : rot / 2;
        units = VEC ? dim / 8 : turned + dim - rot;
    }
    __device__ __forceinline__ int unit(int e) const { return VEC ? u : u + 64 * e; }
    __device__ __forceinline__ bool has(int e) const { return unit(e) < units; }
    __device__ __forceinline__ bool turn(int e) const { return unit(e) < turned; }
    __device__ __forceinline__ bool has_hi(int e) const { return VEC ? has(e) : turn(e); }
    // VEC: first elements of the two runs of four; else the elements themselves
    __device__ __forceinline__ int a(int e) const
    {
        if (VEC) return turn(0) ? (interleaved ? 8 * u : 4 * u) : 8 * u;       // (rot = 8 turned)
        const int i = unit(e);
        return turn(e) ? (interleaved ? 2 * i : i) : rot + i - turned;
    }
    __device__ __forceinline__ int b(int e) const
    {
        if (VEC) return turn(0) && !interleaved ? 4 * u + rot / 2 : 8 * u + 4;
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
        Raw<S> r = {};
        if constexpr (VEC) {
            if (has(0)) {
                r.a = *(const vec4<S> *)(x + a(0));
                r.b = *(const vec4<S> *)(x + b(0));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (has(e)) r.a[e] = x[a(e)];
                if (has_hi(e)) r.b[e] = x[b(e)];
            }
        }
        return r;
    }
    template <typename S>
    __device__ __forceinline__ void unpack(const Raw<S> &r, float *lo, float *hi) const
    {
        const f32x4 fa = __builtin_convertvector(r.a, f32x4), fb = __builtin_convertvector(r.b, f32x4);
        const bool mixed = VEC && interleaved && turn(0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = mixed ? (e < 2 ? fa[2 * e] : fb[2 * e - 4]) : fa[e];
            hi[e] = mixed ? (e < 2 ? fa[2 * e + 1] : fb[2 * e - 3]) : fb[e];
        }
    }
    template <typename S>
    __device__ __forceinline__ void load(const S *x, float *lo, float *hi) const { unpack(fetch(x), lo, hi); }
    template <typename D>
    __device__ __forceinline__ void store(D *y, const float *lo, const float *hi) const
    {
        if constexpr (VEC) {
            if (!has(0)) return;
            const bool mixed = interleaved && turn(0);
            const f32x4 fa = mixed ? f32x4{lo[0], hi[0], lo[1], hi[1]} : f32x4{lo[0], lo[1], lo[2], lo[3]};
            const f32x4 fb = mixed ? f32x4{lo[2], hi[2], lo[3], hi[3]} : f32x4{hi[0], hi[1], hi[2], hi[3]};
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
    __device__ __forceinline__ void load_weight(const void *w, int half, float *lo, float *hi) const
    {
        if (half) load((const _Float16 *)w, lo, hi);
        else load((const float *)w, lo, hi);
    }
    __device__ __forceinline__ void load_angles(const NormParams &p, int position, float *c, float *s) const
    {
        const float *row = p.table + (long long)min(max(position, 0), p.table_rows - 1) * rot;
        if constexpr (VEC) {
            f32x4 fc = {1.f, 1.f, 1.f, 1.f}, fs = {};
            if (turn(0)) {
                fc = *(const f32x4 *)(row + 4 * u);
                fs = *(const f32x4 *)(row + rot / 2 + 4 * u);
            }
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

__device__ __forceinline__ float norm_scale(const NormParams &p, float squares) { return rsqrtf(squares / (float)p.dim + p.eps); }

template <typename S, typename D, bool APPEND, bool VEC, int LPH>
__global__ void __launch_bounds__(kThreads)
norm_rotary_kernel(NormParams p)
{
    constexpr int GROUPS = kThreads / LPH;
    const int t = blockIdx.x, group = threadIdx.x / LPH;
    const Place<VEC> at(p, threadIdx.x % LPH);
    D *kdst = nullptr, *vdst = nullptr;
    if constexpr (APPEND) {
        const long long slot = p.slots[t];
        if (slot < 0 || slot >= (long long)p.pool.pages * p.pool.page_size.d) return;
        const unsigned page_size = p.pool.page_size.d;
        const int page = (int)(slot / page_size), in = (int)(slot - (long long)page * page_size);
        kdst = (D *)p.pool.k + page_offset(page, p.pool.k_page, in, p.pool.k_tok);
        vdst = (D *)p.pool.v + page_offset(page, p.pool.v_page, in, p.pool.v_tok);
    }
    float c[4], s[4], ql[4], qh[4], kl[4], kh[4];
    if (p.table) at.load_angles(p, p.positions[t], c, s);
    const bool one_weight = (!p.q_weight || p.qw_head == 0) && (!p.k_weight || p.kw_head == 0);
    if (one_weight && p.q_weight) at.load_weight(p.q_weight, p.weight_half, ql, qh);
    if (APPEND && one_weight && p.k_weight) at.load_weight(p.k_weight, p.weight_half, kl, kh);

    const int heads = p.q_heads + 2 * p.kv_heads;
    const int first = blockIdx.y * p.heads_per_block, last = min(heads, first + p.heads_per_block);
    // rows of a group whose loads are on their way together
    constexpr int AHEAD = VEC ? 4 : 1;
    for (int h0 = first + group; h0 < last; h0 += AHEAD * GROUPS) {
        typename Place<VEC>::template Raw<S> raw[AHEAD];
        D *dst[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int h = h0 + j * GROUPS;
            dst[j] = nullptr;
            if (h >= last) continue;
            const S *src;
            if (!APPEND || h < p.q_heads) {
                src = (const S *)p.q.p + (long long)t * p.q.tok + (long long)h * p.q.head;
                dst[j] = (D *)p.qo.p + (long long)t * p.qo.tok + (long long)h * p.qo.head;
            } else {
                const bool is_v = h >= p.q_heads + p.kv_heads;
                const int key_head = h - p.q_heads - (is_v ? p.kv_heads : 0);
                const HeadRows &rows = is_v ? p.v : p.k;
                src = (const S *)rows.p + (long long)t * rows.tok + (long long)key_head * rows.head;
                dst[j] = is_v ? vdst + (long long)key_head * p.pool.v_head : kdst + (long long)key_head * p.pool.k_head;
            }
            raw[j] = at.fetch(src);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int h = h0 + j * GROUPS;
            if (h >= last) continue;                       // (the same in all lanes of a group, as all below)
            const bool is_q = !APPEND || h < p.q_heads, is_v = APPEND && h >= p.q_heads + p.kv_heads;
            float lo[4], hi[4];
            at.unpack(raw[j], lo, hi);
            if (is_q ? p.q_weight != nullptr : !is_v && p.k_weight) {
                float wl[4], wh[4], squares = 0.f;
                if (one_weight) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        wl[e] = is_q ? ql[e] : kl[e];
                        wh[e] = is_q ? qh[e] : kh[e];
                    }
                } else {
                    const long long element = is_q ? h * p.qw_head : (h - p.q_heads) * p.kw_head;
                    at.load_weight((const char *)(is_q ? p.q_weight : p.k_weight) + element * (p.weight_half ? 2 : 4), p.weight_half, wl, wh);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) squares += lo[e] * lo[e] + hi[e] * hi[e];
                const float r = norm_scale(p, group_sum<LPH>(squares));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    lo[e] = lo[e] * r * wl[e];
                    hi[e] = hi[e] * r * wh[e];
                }
            }
            if (p.table && !is_v) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!at.turn(e)) continue;
                    const float l = lo[e], k = hi[e];
                    lo[e] = l * c[e] - k * s[e];
                    hi[e] = k * c[e] + l * s[e];
                }
            }
            at.store(dst[j], lo, hi);
        }
    }
}

// PER_HEAD: blockIdx.y is a head, rows are its tokens; else rows are all heads of all tokens.
template <typename X, typename Y, bool PER_HEAD, bool VEC, int LPH>
__global__ void __launch_bounds__(kThreads)
norm_rotary_grad_kernel(NormParams p, FastDiv heads)
{
    constexpr int GROUPS = kThreads / LPH;
    __shared__ __attribute__((aligned(16))) float sums[GROUPS][LPH * 8];
    const int group = threadIdx.x / LPH, lane = threadIdx.x % LPH;
    const Place<VEC> at(p, lane);
    const long long all = PER_HEAD ? p.tokens : (long long)p.tokens * p.q_heads;
    const long long first = (long long)blockIdx.x * p.chunk, last = min(all, first + p.chunk);
    float wl[4], wh[4], dl[4] = {}, dh[4] = {};
    if constexpr (PER_HEAD) at.load_weight((const char *)p.q_weight + blockIdx.y * p.qw_head * (p.weight_half ? 2 : 4), p.weight_half, wl, wh);
    else at.load_weight(p.q_weight, p.weight_half, wl, wh);
    constexpr int AHEAD = VEC ? 2 : 1;
    float c[4], s[4];
    int angles_of = -1;
    for (long long i0 = first + group; i0 < last; i0 += AHEAD * GROUPS) {
        typename Place<VEC>::template Raw<X> x[AHEAD];
        typename Place<VEC>::template Raw<Y> y[AHEAD];
        int tok[AHEAD], head[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const long long i = i0 + j * GROUPS;
            if (i >= last) continue;
            tok[j] = PER_HEAD ? (int)i : heads.quot((int)i);
            head[j] = PER_HEAD ? blockIdx.y : (int)i - tok[j] * p.q_heads;
            x[j] = at.fetch((const X *)p.q.p + (long long)tok[j] * p.q.tok + (long long)head[j] * p.q.head);
            y[j] = at.fetch((const Y *)p.dy.p + (long long)tok[j] * p.dy.tok + (long long)head[j] * p.dy.head);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (i0 + j * GROUPS >= last) continue;
            const int t = tok[j], h = head[j];
            float xl[4], xh[4], gl[4], gh[4], squares = 0.f, dots = 0.f;
            at.unpack(x[j], xl, xh);
            at.unpack(y[j], gl, gh);
            if (p.table) {
                if (t != angles_of) {
                    at.load_angles(p, p.positions[t], c, s);
                    angles_of = t;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!at.turn(e)) continue;
                    const float l = gl[e], k = gh[e];
                    gl[e] = l * c[e] + k * s[e];
                    gh[e] = k * c[e] - l * s[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                squares += xl[e] * xl[e] + xh[e] * xh[e];
                dots += gl[e] * wl[e] * xl[e] + gh[e] * wh[e] * xh[e];
            }
            const float r = norm_scale(p, group_sum<LPH>(squares)), m = group_sum<LPH>(dots) * r / (float)p.dim;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float ul = xl[e] * r, uh = xh[e] * r;
                dl[e] += gl[e] * ul;
                dh[e] += gh[e] * uh;
                gl[e] = r * (gl[e] * wl[e] - ul * m);
                gh[e] = r * (gh[e] * wh[e] - uh * m);
            }
            if (p.qo.p) at.store((X *)p.qo.p + (long long)t * p.qo.tok + (long long)h * p.qo.head, gl, gh);
        }
    }
    if (!p.dw) return;
    at.store(sums[group], dl, dh);
    __syncthreads();
    float *part = p.part + ((long long)blockIdx.x * (PER_HEAD ? p.q_heads : 1) + (PER_HEAD ? blockIdx.y : 0)) * p.dim;
    for (int i = threadIdx.x; i < p.dim; i += kThreads) {
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) sum += sums[g][i];
        part[i] = sum;
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
#pragma unroll 4
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

template <typename S, typename D, bool APPEND>
hipError_t launch_as(const NormParams &p, bool vec, dim3 grid, hipStream_t stream)
{
    switch (lanes_per_head(p.dim, vec)) {
    case 8: norm_rotary_kernel<S, D, APPEND, true, 8><<<grid, kThreads, 0, stream>>>(p); break;
    case 16: norm_rotary_kernel<S, D, APPEND, true, 16><<<grid, kThreads, 0, stream>>>(p); break;
    case 32: norm_rotary_kernel<S, D, APPEND, true, 32><<<grid, kThreads, 0, stream>>>(p); break;
    default: norm_rotary_kernel<S, D, APPEND, false, 64><<<grid, kThreads, 0, stream>>>(p);
    }
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
    const FastDiv heads((unsigned)p.q_heads);
    switch (lanes_per_head(p.dim, vec)) {
    case 8: norm_rotary_grad_kernel<X, Y, PER_HEAD, true, 8><<<grid, kThreads, 0, stream>>>(p, heads); break;
    case 16: norm_rotary_grad_kernel<X, Y, PER_HEAD, true, 16><<<grid, kThreads, 0, stream>>>(p, heads); break;
    case 32: norm_rotary_grad_kernel<X, Y, PER_HEAD, true, 32><<<grid, kThreads, 0, stream>>>(p, heads); break;
    default: norm_rotary_grad_kernel<X, Y, PER_HEAD, false, 64><<<grid, kThreads, 0, stream>>>(p, heads);
    }
    return hipGetLastError();
}

template <typename X, typename Y>
hipError_t launch_grad_typed(const NormParams &p, bool vec, int groups, hipStream_t stream)
{
    return p.qw_head > 0 ? launch_grad_as<X, Y, true>(p, vec, dim3((unsigned)groups, (unsigned)p.q_heads), stream)
                         : launch_grad_as<X, Y, false>(p, vec, dim3((unsigned)groups), stream);
}

}  // namespace

hipError_t launch_norm_rotary(const NormParams &in, bool append, int src_dtype, int dst_dtype, bool vec, hipStream_t stream)
{
    NormParams p = in;
    const int heads = p.q_heads + 2 * p.kv_heads, rows = kThreads / lanes_per_head(p.dim, vec);
    // few tokens: their heads are spread over workgroups until about four a compute unit are there
    const int most = (heads + rows - 1) / rows, want = (1024 + p.tokens - 1) / p.tokens, blocks = want < most ? want : most;
    p.heads_per_block = (heads + blocks - 1) / blocks;
    p.heads_per_block = (p.heads_per_block + rows - 1) / rows * rows;
    const dim3 grid((unsigned)p.tokens, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
    if (src_dtype == NNJIT_F32)
        return dst_dtype == NNJIT_F32 ? launch_typed<float, float>(p, append, vec, grid, stream)
                                      : launch_typed<float, _Float16>(p, append, vec, grid, stream);
    return dst_dtype == NNJIT_F32 ? launch_typed<_Float16, float>(p, append, vec, grid, stream)
                                  : launch_typed<_Float16, _Float16>(p, append, vec, grid, stream);
}

int norm_grad_groups(int64_t tokens, int64_t heads, int dim, bool per_head, bool vec, int cus)
{
    const int64_t rows = per_head ? tokens : tokens * heads, at_once = kThreads / lanes_per_head(dim, vec);
    const int64_t want = (rows + at_once - 1) / at_once, most = per_head ? (4 * cus + heads - 1) / heads : 4 * cus;
    return (int)(want < 1 ? 1 : want < most ? want : most);      // (no rows: one adds up nothing)
}

hipError_t launch_norm_rotary_grad(const NormParams &in, int x_dtype, int dy_dtype, bool vec, int groups, hipStream_t stream)
{
    NormParams p = in;
    const long long rows = p.qw_head > 0 ? p.tokens : (long long)p.tokens * p.q_heads;
    p.chunk = (int)((rows + groups - 1) / groups);
    hipError_t e;
    if (x_dtype == NNJIT_F32)
        e = dy_dtype == NNJIT_F32 ? launch_grad_typed<float, float>(p, vec, groups, stream) : launch_grad_typed<float, _Float16>(p, vec, groups, stream);
    else
        e = dy_dtype == NNJIT_F32 ? launch_grad_typed<_Float16, float>(p, vec, groups, stream)
                                  : launch_grad_typed<_Float16, _Float16>(p, vec, groups, stream);
    if (e != hipSuccess || !p.dw) return e;
    const long long n = (long long)p.dim * (p.qw_head > 0 ? p.q_heads : 1);
    sum_parts_kernel<<<dim3((unsigned)((n + 31) / 32)), 1024, 0, stream>>>(p.part, p.dw, groups, n);
    return hipGetLastError();
}

}  // namespace nnjit
