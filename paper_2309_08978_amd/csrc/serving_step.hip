// The arrays of one step of a served batch, from the requests' lengths.
//
// All of it is prefix sums over the sequences and look-ups in them: with
//   old = ceil(held / P), need = ceil((keep + added) / P)
// sequence b gives back old - need pages or takes need - old.  Taken page i
// (counted over the batch) is entry top - 1 - i of the stack that the given back
// ones lie on top of, top = count + given back: above `count` that is given
// back page top - 1 - i - count itself, read from where it still stands in the
// page table.  So every entry of table, stack and slots follows from the prefix
// sums and from entries that no one writes in this step, and workgroups need
// not wait for each other: each takes the sums anew (a few kilobytes of lengths)
// and then its share of the rows and pages.
//
// Only where lengths or count are replaced in place would a workgroup that starts
// late read what an early one has written: one workgroup does such a step alone,
// writing them last, or a second launch does.
//
// A tree row's ancestors are found by walking up the parents, of which a workgroup holds
// its rows' and those as far before them as a mask reaches in LDS.
//
// All latency: lengths, sums, then page table and stack, one after the other.  Eight
// sequences that decode a token each: 4.2 us on the device (a call: 5.4); 256 requests that come, go and
// shrink, with trees of up to 48 tokens (7181 rows): a call every 7.1, 7.6 on the device under a
// profiler.  (With the sums behind a barrier each, lengths read again for every page and all
// workgroups seeing to pages and rows: 9.5 a call.)
#include "serving.h"

namespace nnjit {

namespace {

enum { kMissing = 1, kLengths = 2, kRows = 4, kPool = 8 };

// Three sums over the threads before this one, and over all; and what any thread has in `bad`.  One barrier.
template <int THREADS>
__device__ __forceinline__ void sums_before(long long (&v)[3], long long (&all)[3], int &bad, long long (*waves)[THREADS / 64], int *flags)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        long long run = v[k];
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const long long up = __shfl_up(run, i);
            if (lane >= i) run += up;
        }
        if (lane == 63) waves[k][wave] = run;
        v[k] = run - v[k];
    }
    const int any = (__ballot(bad & kLengths) ? kLengths : 0) | (__ballot(bad & kRows) ? kRows : 0);
    if (lane == 0) flags[wave] = any;
    __syncthreads();
    bad = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) bad |= flags[w];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        all[k] = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) v[k] += waves[k][w];
            all[k] += waves[k][w];
        }
    }
}

// The last b with sums[b] <= i, 0 <= i < sums[n].
__device__ __forceinline__ int holder(const int *sums, int n, int i)
{
    int lo = 0, hi = n;                       // sums[lo] <= i < sums[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// THREADS PER sequences at most.  LATER: lengths and count are left to a second
// launch, FINISH, which writes nothing else.
template <int THREADS, int PER, bool LATER, bool FINISH>
__global__ void __launch_bounds__(THREADS)
paged_step_kernel(StepParams p)
{
    constexpr int N = THREADS * PER, REACH = 32 * kStepWords;
    __shared__ int start[N + 1], back[N + 1], more[N + 1], old_pages[N];
    __shared__ long long waves[3][THREADS / 64];
    __shared__ int flags[THREADS / 64];
    __shared__ int parents[REACH + THREADS];

    const int tid = threadIdx.x, n = p.sequences;
    const int page_size = p.page_size.d;
    const long long room = min((long long)p.table_pages * page_size, kMaxKeys);
    auto pages_of = [&](int tokens) { return p.page_size.quot(tokens + page_size - 1); };

    int rows_of[PER], delta[PER], old_of[PER], bad = 0;
    long long sums[3] = {0, 0, 0}, all[3];                   // rows, pages given back, pages taken
    const int count = p.count[0];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int b = tid * PER + e;
        rows_of[e] = delta[e] = old_of[e] = 0;
        if (b >= n) continue;
        const int held = p.held[b], keep = p.keep ? p.keep[b] : held, added = p.added[b];
        if (held < 0 || keep < 0 || keep > held || added < 0 || held > room || (long long)keep + added > room) {
            bad |= kLengths;
            continue;
        }
        if (p.parent && added > 32 * p.mask_words) bad |= kRows;
        rows_of[e] = added;
        old_of[e] = pages_of(held);
        delta[e] = pages_of(keep + added) - old_of[e];
        sums[0] += added;
        sums[1] += max(-delta[e], 0);
        sums[2] += max(delta[e], 0);
    }
    sums_before<THREADS>(sums, all, bad, waves, flags);
    const long long all_rows = all[0], all_given = all[1], all_taken = all[2];
    if (all_rows > p.tokens) bad |= kRows;
    if (count < 0 || count > p.capacity || count + all_given > p.capacity) bad |= kPool;
    const long long missing = bad & (kLengths | kPool) ? 0 : max(all_taken - all_given - count, 0ll);
    if (missing > 0) bad |= kMissing;
    const int top = bad ? count : count + (int)all_given, left = bad ? count : top - (int)all_taken;
    const int pages = bad ? 0 : (int)all_taken, pushes = max(left - count, 0);

    if constexpr (!FINISH) {
        int at[3] = {(int)sums[0], (int)sums[1], (int)sums[2]};
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int b = tid * PER + e;
            start[b] = bad ? 0 : at[0];
            back[b] = at[1];
            more[b] = at[2];
            old_pages[b] = old_of[e];
            at[0] += rows_of[e];
            at[1] += max(-delta[e], 0);
            at[2] += max(delta[e], 0);
        }
        if (tid == THREADS - 1) {
            start[N] = bad ? 0 : at[0];
            back[N] = at[1];
            more[N] = at[2];
        }
        __syncthreads();

        auto given_back = [&](int i) {
            const int b = holder(back, n, i);                            // its last pages, up to old_pages[b]
            return p.page_table[(long long)b * p.ld_table + old_pages[b] - (back[b + 1] - i)];
        };
        auto page_taken = [&](int i) {
            const int entry = top - 1 - i;
            return entry >= count ? given_back(entry - count) : p.free_pages[entry];
        };

        // rows are the first workgroups' share, pages the others' (a lone workgroup does both)
        const int row_groups = gridDim.x > 1 ? gridDim.x - p.page_groups : 1, page_groups = gridDim.x > 1 ? p.page_groups : 1;
        const bool has_rows = (int)blockIdx.x < row_groups, has_pages = gridDim.x == 1 || !has_rows;
        const int page_stride = page_groups * THREADS;
        const int page_first = has_pages ? (gridDim.x > 1 ? (int)blockIdx.x - row_groups : 0) * THREADS + tid : 0x7fffffff;
        for (int b = page_first; b <= n; b += page_stride) p.q_start[b] = start[b];
        // (unsigned: a step behind the last of almost 2^31 pages passes 31 bits)
        for (unsigned at = page_first; at < (unsigned)pages; at += page_stride) {
            const int i = at, b = holder(more, n, i);
            p.page_table[(long long)b * p.ld_table + old_pages[b] + i - more[b]] = page_taken(i);
        }
        for (unsigned at = page_first; at < (unsigned)pushes; at += page_stride) p.free_pages[count + at] = given_back(at);
        if (blockIdx.x == 0 && tid < 4)
            p.status[tid] = tid == 0 ? bad : tid == 1 ? (int)min(missing, 0x7fffffffll) : tid == 2 ? (bad ? 0 : (int)all_rows) : left;

        const int end = start[n];
        for (int base = has_rows ? blockIdx.x * THREADS : p.tokens; base < p.tokens; base += row_groups * THREADS) {
            const int t = base + tid;
            if (p.parent) {
                __syncthreads();
                for (int i = REACH - 32 * p.mask_words + tid; i < REACH + THREADS; i += THREADS) {
                    const int row = base - REACH + i;
                    parents[i] = row >= 0 && row < end ? p.parent[row] : -1;
                }
                __syncthreads();
            }
            if (t >= p.tokens) continue;
            int position = 0;
            long long slot = -1;
            unsigned *mask_row = p.mask ? p.mask + (long long)t * p.ld_mask : nullptr;
            if (t < end) {
                const int b = holder(start, n, t), keep = p.keep ? p.keep[b] : p.held[b];
                const int place = keep + t - start[b], at_page = p.page_size.quot(place), old = old_pages[b];
                const int page = at_page < old ? p.page_table[(long long)b * p.ld_table + at_page] : page_taken(more[b] + at_page - old);
                if (page >= 0) slot = (long long)page * page_size + place - at_page * page_size;
                position = place;
                if (p.parent) {
                    const int *own = parents + REACH - (base - start[b]);          // own[i]: parent of the sequence's node i
                    int node = t - start[b], word = p.mask_words - 1, depth = 0;
                    unsigned bits = 0;
                    while (true) {
                        for (; word > node >> 5; --word) {
                            mask_row[word] = bits;
                            bits = 0;
                        }
                        bits |= 1u << (node & 31);
                        const int up = own[node];
                        if (up < 0 || up >= node) break;
                        node = up;
                        ++depth;
                    }
                    for (; word >= 0; --word) {
                        mask_row[word] = bits;
                        bits = 0;
                    }
                    position = keep + depth;
                } else if (mask_row) {
                    // no trees: the chain, as far as the words go
                    const int node = t - start[b];
                    for (int w = 0; w < p.mask_words; ++w) {
                        const int last_bit = node - 32 * w;               // of this word
                        mask_row[w] = last_bit < 0 ? 0u : last_bit >= 31 ? ~0u : (2u << last_bit) - 1u;
                    }
                }
            } else if (mask_row) {
                for (int w = 0; w < p.mask_words; ++w) mask_row[w] = 0;
            }
            if (p.positions) p.positions[t] = position;
            if (p.slots) p.slots[t] = slot;
        }
        __syncthreads();
    }
    if constexpr (!LATER) {
        for (int b = blockIdx.x * THREADS + tid; b < n; b += gridDim.x * THREADS) {
            const int held = p.held[b];
            p.kv_len[b] = bad ? held : (p.keep ? p.keep[b] : held) + p.added[b];
        }
        if (blockIdx.x == 0 && tid == 0) p.count_out[0] = left;
    }
}

template <int THREADS, int PER>
hipError_t launch_as(const StepParams &p, hipStream_t stream)
{
    const bool in_place = p.kv_len == p.held || p.kv_len == p.keep || p.count_out == p.count;
    StepParams q = p;
    const int most = 512, want = (p.tokens + THREADS - 1) / THREADS, rows = want < 1 ? 1 : want < most ? want : most;
    q.page_groups = rows > 1 ? (rows + 3) / 4 : 0;
    const int groups = rows + q.page_groups;
    if (in_place && groups > 1) {
        paged_step_kernel<THREADS, PER, true, false><<<groups, THREADS, 0, stream>>>(q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        paged_step_kernel<THREADS, PER, false, true><<<1, THREADS, 0, stream>>>(q);
    } else {
        paged_step_kernel<THREADS, PER, false, false><<<groups, THREADS, 0, stream>>>(q);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_step(const StepParams &p, hipStream_t stream)
{
    if (p.sequences <= 256) return launch_as<256, 1>(p, stream);
    if (p.sequences <= 1024) return launch_as<256, 4>(p, stream);
    return launch_as<1024, kStepSequences / 1024>(p, stream);
}

}  // namespace nnjit
