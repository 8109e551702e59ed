// Rules for logits: penalties for tokens that are there already, biases of
// single tokens, masks of allowed ones.
//
//   z = x;  z = x > 0 ? x / rho : x rho   where the token is in the history
//   z -= phi c + (pi if c > 0)            c: how often it is there behind the prompt
//   z += beta;  -inf where the mask has no bit
//
// A workgroup takes a segment of neighbouring tokens of a row: it counts those of the
// history that fall into it (integer sums in LDS, so their order does not matter),
// notes for each token the last bias entry, and goes over the logits once; they and the
// first of the history are asked for before all that.  The history is read once a
// segment, from the caches.
//
// Bandwidth-bound for many rows: 64 rows of 128000 fp32 logits, histories of up to 4000
// tokens, 100 biases a row, masks: 14.5 us, 4.6 TB/s (without biases and masks 13.1); one row of 32000 with a history of
// 1000: 3.8 us on the device.
#include "kcommon.h"
#include "serving.h"
#include "nnjit.h"

namespace nnjit {

namespace {

// What LDS holds of a token: bit 31: it is in the prompt; then its count; then the
// last bias entry, from 1 on.  NARROW: in one word, for histories below 2^15 tokens and
// biases of less than 2^16 entries, so that twice as many workgroups fit a compute unit; else in two.
template <bool NARROW>
struct Noted {
    static constexpr unsigned kPrompt = 1u << 31, kOne = NARROW ? 1u << 16 : 1u;
    static constexpr int kWords = NARROW ? 1 : 2;
    __device__ static __forceinline__ unsigned count(unsigned w) { return (w & ~kPrompt) >> (NARROW ? 16 : 0); }
    __device__ static __forceinline__ bool seen(unsigned w) { return w >= kOne; }
};

template <typename T>
using vec4 = T __attribute__((ext_vector_type(4)));

template <typename S, typename D, bool VEC, bool NARROW, int THREADS, int QUADS>   // QUADS: groups of four tokens a thread
__global__ void __launch_bounds__(THREADS)
adjust_logits_kernel(LogitParams p, int segments, int segment)
{
    typedef Noted<NARROW> N;
    constexpr int SEGMENT = THREADS * 4 * QUADS, AHEAD = 4096 / THREADS;
    __shared__ __attribute__((aligned(16))) unsigned noted[N::kWords * SEGMENT];
    unsigned *entries = noted + (N::kWords - 1) * SEGMENT;             // last bias entries
    const int row = blockIdx.x / segments, v0 = (blockIdx.x - row * segments) * segment, tid = threadIdx.x;
    const S *x = (const S *)p.x + (long long)row * p.ldx + v0;
    D *y = (D *)p.y + (long long)row * p.ldy + v0;
    const int here = min(p.vocab - v0, segment);                       // (one or more)

    const int length = p.length ? min(max(p.length[row], 0), p.history_len) : p.history_len;
    const int prompt = p.prompt ? p.prompt[row] : 0;
    const int *bias_tokens = p.bias_token + (p.bias_token ? (long long)row * p.ld_bias : 0);
    int first_bias = p.bias_token && tid < p.bias_len ? bias_tokens[tid] : -1;
    const int *tokens = p.history + (p.history ? (long long)row * p.ld_history : 0);
    int first[AHEAD];
    if (p.history) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) first[k] = k * THREADS + tid < p.history_len ? tokens[k * THREADS + tid] : -1;
    }
    vec4<S> raw[QUADS];
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int v = (q * THREADS + tid) * 4;
        raw[q] = vec4<S>{};
        if (VEC && v + 4 <= here) {
            raw[q] = *(const vec4<S> *)(x + v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (v + e < here) raw[q][e] = x[v + e];
        }
    }
    const float rho = p.repetition ? p.repetition[row] : 1.f, pi = p.presence ? p.presence[row] : 0.f;
    const float phi = p.frequency ? p.frequency[row] : 0.f;
    const float *bias = p.bias_value + (p.bias_token ? (long long)row * p.ld_bias : 0);
    const unsigned *mask = nullptr;
    if (p.mask) {
        const int m = p.mask_row ? p.mask_row[row] : row;
        if (m >= 0) mask = p.mask + (long long)min(m, p.mask_rows - 1) * p.ld_mask;
    }
    unsigned allowed[QUADS];
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int v = (q * THREADS + tid) * 4;
        allowed[q] = mask && v < here ? mask[(v0 + v) >> 5] >> (v & 31) : 15u;
    }

    for (int i = tid; i < N::kWords * SEGMENT / 4; i += THREADS) ((u32x4 *)noted)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    if (p.bias_token) {
        // (unsigned: the last step of lists of almost 2^31 entries passes 31 bits)
        for (unsigned i = tid; i < (unsigned)p.bias_len; i += THREADS) {
            const unsigned v = (unsigned)(i == (unsigned)tid ? first_bias : bias_tokens[i]) - (unsigned)v0;   // (a negative token lies above every segment)
            if (v < (unsigned)here) atomicMax(&entries[v], i + 1u);
        }
        if (NARROW) __syncthreads();                                   // (counts lie above the entries)
    }
    if (p.history) {
        auto note = [&](int i, int token) {
            const unsigned v = (unsigned)token - (unsigned)v0;
            if (i >= length || v >= (unsigned)here) return;
            if (i < prompt) atomicOr(&noted[v], N::kPrompt);
            else atomicAdd(&noted[v], N::kOne);
        };
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) note(k * THREADS + tid, first[k]);
#pragma unroll 4
        for (unsigned i = AHEAD * THREADS + tid; i < (unsigned)length; i += THREADS) note((int)i, tokens[i]);
    }
    __syncthreads();

#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int v = (q * THREADS + tid) * 4;
        if (v >= here) continue;
        const u32x4 four = *(const u32x4 *)&noted[v];
        u32x4 entry = NARROW ? four & 0xffffu : *(const u32x4 *)&entries[v];
        vec4<D> out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float f = (float)raw[q][e];
            if (four[e] | entry[e]) {                                  // few waves have such a token
                const unsigned c = N::count(four[e]), at = entry[e];
                if (p.repetition && N::seen(four[e])) f = f > 0.f ? f / rho : f * rho;
                if (c > 0) f = f - phi * (float)c - pi;
                if (at) f += bias[at - 1];
            }
            out[e] = (D)(allowed[q] >> e & 1 ? f : -__builtin_inff());
        }
        if (VEC && v + 4 <= here) {
            *(vec4<D> *)(y + v) = out;
        } else {
            for (int e = 0; e < 4 && v + e < here; ++e) y[v + e] = out[e];
        }
    }
}

template <typename S, typename D, bool NARROW, int THREADS, int QUADS>
hipError_t launch_as(const LogitParams &p, bool vec, hipStream_t stream)
{
    const int segments = (p.vocab + THREADS * 4 * QUADS - 1) / (THREADS * 4 * QUADS);
    // equal ones, of whole cache lines, SEGMENT or less, so that the last holds something: 256 rows of 50000 in fp16 20.5 us, with a
    // short last one 22.8, 300 of 20000 in fp32 16.9 and 20.2
    const int segment = ((p.vocab + segments - 1) / segments + 63) / 64 * 64;
    const unsigned grid = (unsigned)p.rows * (unsigned)segments;
    if (vec) adjust_logits_kernel<S, D, true, NARROW, THREADS, QUADS><<<grid, THREADS, 0, stream>>>(p, segments, segment);
    else adjust_logits_kernel<S, D, false, NARROW, THREADS, QUADS><<<grid, THREADS, 0, stream>>>(p, segments, segment);
    return hipGetLastError();
}

template <typename S, typename D>
hipError_t launch_typed(const LogitParams &p, bool vec, int cus, hipStream_t stream)
{
    const LogitPlan plan = logit_plan(p.rows, p.vocab, p.history_len, p.bias_len, cus);
    if (plan.threads == 512) return launch_as<S, D, true, 512, 1>(p, vec, stream);
    if (plan.quads == 4) return launch_as<S, D, true, 1024, 4>(p, vec, stream);
    if (plan.quads == 2) return plan.narrow ? launch_as<S, D, true, 1024, 2>(p, vec, stream) : launch_as<S, D, false, 1024, 2>(p, vec, stream);
    return plan.narrow ? launch_as<S, D, true, 1024, 1>(p, vec, stream) : launch_as<S, D, false, 1024, 1>(p, vec, stream);
}

}  // namespace

// Long segments read the history seldom, short ones spread a call over more compute units; many threads read it in
// fewer steps and start later.  By 512 threads of 4 tokens, 1024 of 4, of 8 and of 16, histories of 4000, in us:
//   1 row of 32000 in fp32        3.9   4.3   5.2   7.0   (histories of 16000: 7.0   6.1   7.0   9.0)
//   8 rows of 128000 in fp32      4.9   4.8   5.5   7.0
//   32 rows of 128000 in fp16    11.0  10.5   8.2   8.6
//   64 rows of 128000 in fp16    18.1  18.0  13.5  12.7
// Two words a token: 16 leave one workgroup a compute unit: 64 rows, histories of 33000 28.8 with 8, 32.6 with 16.
LogitPlan logit_plan(int64_t rows, int64_t vocab, int64_t history_len, int64_t bias_len, int cus)
{
    const int narrow = history_len < 1 << 15 && bias_len < 1 << 16;
    auto groups = [&](int64_t segment) { return rows * ((vocab + segment - 1) / segment); };
    if (narrow && history_len <= 4096 && groups(2048) <= cus) return LogitPlan{512, 1, narrow};
    if (groups(4096) <= cus) return LogitPlan{1024, 1, narrow};
    // (with 16 two fit a compute unit at once: not for a few that are left over: 300 rows of 20000 in fp16 15.6, with 8 14.6)
    const int64_t longest = groups(16384), over = longest % (2 * cus);
    if (narrow && (over == 0 || 2 * over >= 3 * cus || longest >= 8ll * cus)) return LogitPlan{1024, 4, narrow};
    return LogitPlan{1024, 2, narrow};
}

hipError_t launch_adjust_logits(const LogitParams &p, int x_dtype, int y_dtype, bool vec, int cus, hipStream_t stream)
{
    if (x_dtype == NNJIT_F32)
        return y_dtype == NNJIT_F32 ? launch_typed<float, float>(p, vec, cus, stream) : launch_typed<float, _Float16>(p, vec, cus, stream);
    return y_dtype == NNJIT_F32 ? launch_typed<_Float16, float>(p, vec, cus, stream) : launch_typed<_Float16, _Float16>(p, vec, cus, stream);
}

}  // namespace nnjit
