// Rules for logits: penalties for tokens that are there already, biases of
// single tokens, masks of allowed ones.
//
//   z = x;  z = x > 0 ? x / rho : x rho   where the token is in the history
//   z -= phi c + (pi if c > 0)            c: how often it is there behind the prompt
//   z += beta;  -inf where the mask has no bit
//
// A workgroup takes kSegment neighbouring tokens of a row: it counts those of the
// history that fall into them (integer sums in LDS, so their order does not matter),
// notes for each token the last bias entry, and goes over the logits once.  The
// history is read once a segment, from the caches.
#include "kcommon.h"
#include "serving.h"
#include "nnjit.h"

namespace nnjit {

namespace {

constexpr int kThreads = 256;
constexpr unsigned kInPrompt = 1u << 31;      // of a count: the token is in the prompt

template <typename T>
using vec4 = T __attribute__((ext_vector_type(4)));

template <typename S, typename D, bool VEC, int QUADS>   // QUADS: groups of four tokens a thread
__global__ void __launch_bounds__(kThreads)
adjust_logits_kernel(LogitParams p, int segments)
{
    constexpr int SEGMENT = kThreads * 4 * QUADS;
    __shared__ __attribute__((aligned(16))) unsigned counts[SEGMENT];
    __shared__ __attribute__((aligned(16))) int last_bias[SEGMENT];
    const int row = blockIdx.x / segments, v0 = (blockIdx.x - row * segments) * SEGMENT, tid = threadIdx.x;
    const S *x = (const S *)p.x + (long long)row * p.ldx + v0;
    D *y = (D *)p.y + (long long)row * p.ldy + v0;
    const int here = min(p.vocab - v0, SEGMENT);

    float z[QUADS][4];
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int v = (q * kThreads + tid) * 4;
        if (VEC && v + 4 <= here) {
            const f32x4 f = __builtin_convertvector(*(const vec4<S> *)(x + v), f32x4);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[q][e] = f[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) z[q][e] = v + e < here ? (float)x[v + e] : 0.f;
        }
    }

    for (int i = tid; i < SEGMENT; i += kThreads) {
        counts[i] = 0;
        last_bias[i] = 0;
    }
    __syncthreads();
    if (p.history) {
        const int length = p.length ? min(max(p.length[row], 0), p.history_len) : p.history_len;
        const int prompt = p.prompt ? p.prompt[row] : 0;
        const int *tokens = p.history + (long long)row * p.ld_history;
#pragma unroll 4
        for (int i = tid; i < length; i += kThreads) {
            const unsigned v = (unsigned)tokens[i] - (unsigned)v0;   // (a negative token lies above every segment)
            if (v >= (unsigned)here) continue;
            if (i < prompt) atomicOr(&counts[v], kInPrompt);
            else atomicAdd(&counts[v], 1u);
        }
    }
    if (p.bias_token) {
        const int *tokens = p.bias_token + (long long)row * p.ld_bias;
        for (int i = tid; i < p.bias_len; i += kThreads) {
            const unsigned v = (unsigned)tokens[i] - (unsigned)v0;
            if (v < (unsigned)here) atomicMax(&last_bias[v], i + 1);
        }
    }
    __syncthreads();

    const float rho = p.repetition ? p.repetition[row] : 1.f, pi = p.presence ? p.presence[row] : 0.f;
    const float phi = p.frequency ? p.frequency[row] : 0.f;
    const float *bias = p.bias_value + (p.bias_token ? (long long)row * p.ld_bias : 0);
    const unsigned *mask = nullptr;
    if (p.mask) {
        const int m = p.mask_row ? p.mask_row[row] : row;
        if (m >= 0) mask = p.mask + (long long)min(m, p.mask_rows - 1) * p.ld_mask;
    }
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int v = (q * kThreads + tid) * 4;
        if (v >= here) continue;
        const unsigned allowed = mask ? mask[(v0 + v) >> 5] >> (v & 31) : 15u;
        vec4<D> out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned seen = counts[v + e], c = seen & ~kInPrompt;
            float f = z[q][e];
            if (p.repetition && seen) f = f > 0.f ? f / rho : f * rho;
            if (c > 0) f = f - phi * (float)c - pi;
            const int entry = last_bias[v + e];
            if (entry) f += bias[entry - 1];
            out[e] = (D)(allowed >> e & 1 ? f : -__builtin_inff());
        }
        if (VEC && v + 4 <= here) {
            *(vec4<D> *)(y + v) = out;
        } else {
            for (int e = 0; e < 4 && v + e < here; ++e) y[v + e] = out[e];
        }
    }
}

template <typename S, typename D, int QUADS>
hipError_t launch_quads(const LogitParams &p, bool vec, hipStream_t stream)
{
    const int segments = (p.vocab + kThreads * 4 * QUADS - 1) / (kThreads * 4 * QUADS);
    const unsigned grid = (unsigned)p.rows * (unsigned)segments;
    if (vec) adjust_logits_kernel<S, D, true, QUADS><<<grid, kThreads, 0, stream>>>(p, segments);
    else adjust_logits_kernel<S, D, false, QUADS><<<grid, kThreads, 0, stream>>>(p, segments);
    return hipGetLastError();
}

template <typename S, typename D>
hipError_t launch_as(const LogitParams &p, bool vec, int cus, hipStream_t stream)
{
    // small calls: more workgroups, of fewer tokens
    const long long groups = (long long)p.rows * ((p.vocab + kThreads * 16 - 1) / (kThreads * 16));
    return groups < 2 * cus ? launch_quads<S, D, 1>(p, vec, stream) : launch_quads<S, D, 4>(p, vec, stream);
}

}  // namespace

hipError_t launch_adjust_logits(const LogitParams &p, int x_dtype, int y_dtype, bool vec, int cus, hipStream_t stream)
{
    if (x_dtype == NNJIT_F32)
        return y_dtype == NNJIT_F32 ? launch_as<float, float>(p, vec, cus, stream) : launch_as<float, _Float16>(p, vec, cus, stream);
    return y_dtype == NNJIT_F32 ? launch_as<_Float16, float>(p, vec, cus, stream) : launch_as<_Float16, _Float16>(p, vec, cus, stream);
}

}  // namespace nnjit
