// Attention over a paged cache: the instances of attention_rows.h for plain
// and causal rows, the join of splits, the plan that picks kernel and splits.
#include <algorithm>
#include <cmath>

#include "attention_rows.h"
#include "nnjit.h"

namespace nnjit {

namespace {

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
// Trees: few rows over many keys.  Workgroups count in whole rounds for both types, and
// splits that fill the chip's workgroups once to four times are tried as well (64 nodes behind 65536 keys: 26 splits
// of 128 rows 109 us, 32 splits, two workgroups a CU, 97).  Fitted to 300 shapes of 17 .. 1024 rows, 150
// .. 65536 keys, 1 .. 32 sequences; on 150 others within 3.4% of the best choice on the geometric mean, where the
// constants above are within 5.7%.
constexpr StepCost kTreeF16[] = {{16, 128, 1.06, -0.12, 0.82, 2.07}, {64, 64, 0.38, 1.23, 0.38, 0.58}, {128, 64, 0.5, 2.05, 0.47, 0.84}};
constexpr StepCost kTreeF32[] = {{16, 64, 0.78, 1.2, 0.55, 1.31}, {64, 64, 0.4, 4.2, -0.78, 5.9}, {128, 64, -0.3, 7.6, 0.7, 4.46}};
// The second launch of a split, the share of its partial sums' traffic, a later start of tall tiles, and what
// sequences of different lengths cost.
struct SplitCost {
    double join, part, tall, spread;
};
constexpr SplitCost kPromptSplit = {3.8, 1, 1.5, 1.15}, kTreeSplit = {4.9, 1.32, 2.5, 1.02};

// The kernel and the splits of the keys that these estimates call cheapest.
// Tall tiles read keys and values least often but leave CUs idle where rows are
// few (512 new tokens on 3584 cached, 32 heads of 128, in us: 128 rows unsplit 93,
// 64 rows 82, in two splits 59, 128 rows in four 55; 777 alone: 25, 23, 40, 42);
// up to 128 rows of up to 128 keys the 16-row kernel starts soonest (7 against 8);
// a split costs a second launch and writes and reads the partial sums (512 new
// tokens alone: 16 unsplit, 28 in two).
AttentionPlan many_rows_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t rows,
                             int64_t max_kv, int64_t window, bool tree, int cus)
{
    const SplitCost &of = tree ? kTreeSplit : kPromptSplit;
    const StepCost (&steps)[3] = dtype == NNJIT_F16 ? (tree ? kTreeF16 : kStepF16) : (tree ? kTreeF32 : kStepF32);
    const int64_t group = q_heads / kv_heads, lanes = (int64_t)kv_heads * sequences;
    const int elt = dtype == NNJIT_F16 ? 2 : 4;
    const double d = dim / 128.0, part_us = (double)tokens * q_heads * dim * 8 / 3.3e6;   // partial sums of a split, written and read
    AttentionPlan best{};
    double least = 0;
    for (const StepCost &c : steps) {
        if (c.tile_rows == 64 && dim > 128) continue;      // not built: registers
        const int64_t row_tiles = (rows + c.tile_rows - 1) / c.tile_rows;
        const int64_t span = seen_span(max_kv, window, c.tile_rows, group);
        const int64_t filled = tree ? cus / (row_tiles * lanes) : 0;      // splits that give every CU a workgroup
        int64_t want = 1, fill = filled;
        while (want <= 256) {
            // the next number of splits: of the row 1, 2, 3, 4, 6, 8, 12, ..., and one to four times `filled` between them
            const bool between = fill > 0 && fill <= 4 * filled && fill < want;
            const int64_t tried = between ? fill : want;
            if (between || fill == want) fill += filled;
            if (!between) want = want < 4 ? want + 1 : want * 3 / 2 - want * 3 / 2 % 2;
            const int64_t per = (span + tried - 1) / tried;
            const int64_t split_keys = std::max<int64_t>((per + 31) / 32 * 32, 32);
            const int64_t splits = std::max<int64_t>((span + split_keys - 1) / split_keys, 1);
            const double o = (double)row_tiles * lanes * splits / cus;
            // keys and values come once from memory for all row tiles; one workgroup a CU does
            // not draw its full rate, a few CUs with one more take longer, and so do
            // sequences of different lengths unless there are many workgroups
            const double even = o < 4 ? std::ceil(o) : o;
            double bytes_us = 2.0 * c.keys * dim * elt * (even / row_tiles) * 256 / (5.5e6 * std::min(1.0, 0.9 + 0.05 * o));
            if (sequences > 1 && o < 8) bytes_us *= of.spread;
            // fp32 products fill the matrix cores of a CU: its second workgroup takes as long again
            const double share = elt == 4 && c.tile_rows > 16 ? std::ceil(o) : tree ? even : o;
            const double step = std::max({c.a0 + c.a1 * d, (c.b0 + c.b1 * d) * share, bytes_us});
            const double cost = ((split_keys < span ? split_keys : span) + c.keys - 1) / c.keys * step + (splits > 1 ? of.join + splits * part_us * of.part : 0) +
                                (c.tile_rows == 16 ? 0 : of.tall);   // a later start: copies, then products
            if (best.tile_rows == 0 || cost < least) {
                least = cost;
                best.tile_rows = c.tile_rows;
                best.row_tiles = (int)row_tiles;
                best.splits = (int)splits;
                best.split_keys = (int)split_keys;
                best.waves = 4;
            }
            if (splits < tried || o > 16) break;           // more splits than keys, or than the chip holds
        }
    }
    return best;
}

AttentionPlan plan_of(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t max_q, int64_t max_kv,
                      int64_t window, bool tree, int cus)
{
    const int64_t group = q_heads / kv_heads, rows = max_q * group;
    AttentionPlan plan = rows <= 16 ? few_rows_plan(dtype, tokens, sequences, q_heads, kv_heads, dim, seen_span(max_kv, window, 16, group), cus)
                                    : many_rows_plan(dtype, tokens, sequences, q_heads, kv_heads, dim, rows, max_kv, window, tree, cus);
    plan.ws_floats = plan.splits > 1 ? plan.splits * tokens * q_heads * ((dim + 3) / 4 * 4 + 2) : 0;
    return plan;
}

}  // namespace

AttentionPlan attention_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t max_q,
                             int64_t max_kv, int causal, int64_t window, int cus)
{
    return plan_of(dtype, tokens, sequences, q_heads, kv_heads, dim, max_q, max_kv, causal ? window : 0, false, cus);
}

AttentionPlan tree_plan(int dtype, int64_t tokens, int64_t sequences, int q_heads, int kv_heads, int dim, int64_t max_q, int64_t max_kv,
                        int64_t window, int cus)
{
    return plan_of(dtype, tokens, sequences, q_heads, kv_heads, dim, max_q, max_kv, window, true, cus);
}

hipError_t launch_attention(AttentionParams p, const AttentionPlan &plan, int dtype, bool vec, hipStream_t stream)
{
    p.row_tiles = plan.row_tiles;
    p.splits = plan.splits;
    p.split_keys = plan.split_keys;
    p.may_leave_out = plan.splits > 1 && (int64_t)plan.row_tiles * plan.tile_rows < (int64_t)p.batch.tokens * p.group;
    const int grid = plan.row_tiles * plan.splits * (p.q_heads / p.group) * p.batch.sequences;
    hipError_t e;
    if (p.mask && plan.tile_rows == 16)
        e = launch_tree_rows(p, dtype, vec, plan.waves, grid, stream);
    else if (p.mask)
        e = dtype == NNJIT_F16 ? launch_tree_tiles_f16(p, plan.tile_rows, vec, grid, stream) : launch_tree_tiles_f32(p, plan.tile_rows, vec, grid, stream);
    else if (dtype == NNJIT_F16)
        e = plan.tile_rows == 16 ? launch_typed<_Float16, false>(p, vec, plan.waves, grid, stream) : launch_attention_tiles_f16(p, plan.tile_rows, vec, grid, stream);
    else
        e = plan.tile_rows == 16 ? launch_typed<float, false>(p, vec, plan.waves, grid, stream) : launch_attention_tiles_f32(p, plan.tile_rows, vec, grid, stream);
    if (e != hipSuccess || plan.splits == 1) return e;
    return dtype == NNJIT_F16 ? launch_join<_Float16>(p, stream) : launch_join<float>(p, stream);
}

}  // namespace nnjit
