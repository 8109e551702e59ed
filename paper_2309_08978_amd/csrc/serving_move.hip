// The keys and values of accepted nodes of drafted trees go to the places behind
// the cached ones.
//
// Node path[i] of the new tokens moves to new token i's place, i <= path[i].  A
// thread takes one piece (16 bytes, where alignment allows) of one head's key or value row
// and moves it for every i, sixteen loads before their stores: no thread
// touches another's piece, and since later i read at or behind themselves,
// stores of earlier ones never reach what is still to be read.
#include "attention_common.h"

namespace nnjit {

namespace {

constexpr int kThreads = 256, kAhead = 16;

template <typename U>
__global__ void __launch_bounds__(kThreads)
kv_move_kernel(MoveParams p, int elem_bytes)
{
    const int b = blockIdx.x;
    // (what says where things go is the same for all threads: scalar loads)
    const constant_int *path = (const constant_int *)(p.path + (long long)b * p.ld_path);
    int ahead[kAhead];                                               // asked for before what says how many of them count
#pragma unroll
    for (int e = 0; e < kAhead; ++e) ahead[e] = path[min(e, p.path_len - 1)];
    const PageBatch &batch = p.batch;
    const int q0 = min(max(batch.q_start[b], 0), batch.tokens);
    const int added = min(max(batch.q_start[b + 1] - q0, 0), batch.tokens - q0);
    const long long room = min((long long)batch.table_pages * p.pool.page_size.d, kMaxKeys);
    const long long past = (long long)batch.kv_len[b] - added;      // place of the sequence's new token 0
    const int count = min(max(p.accepted[b], 0), p.path_len);
    const constant_int *table = (const constant_int *)(batch.page_table + (long long)b * batch.ld_table);

    const int pieces = p.row_bytes / (int)sizeof(U);                 // of a head's row
    const int piece = blockIdx.y * kThreads + threadIdx.x;
    if (piece >= 2 * p.kv_heads * pieces) return;
    const bool value = piece >= p.kv_heads * pieces;
    const int in = value ? piece - p.kv_heads * pieces : piece, head = in / pieces;
    char *base = (char *)(value ? p.pool.v : p.pool.k) + (value ? p.pool.v_head : p.pool.k_head) * head * elem_bytes +
                 (long long)(in - head * pieces) * sizeof(U);
    const unsigned page_stride = value ? p.pool.v_page : p.pool.k_page, slot_stride = value ? p.pool.v_tok : p.pool.k_tok;

    // the piece of new token i; NULL where the cache has no such place
    auto page_at = [&](int i) {
        const long long place = past + i;
        return place < 0 || place >= room ? -1 : table[p.pool.page_size.quot((int)place)];
    };
    auto piece_at = [&](int i, int page) -> U * {
        if (page < 0 || page >= p.pool.pages) return nullptr;
        const int place = (int)(past + i), slot = place - p.pool.page_size.quot(place) * (int)p.pool.page_size.d;
        return (U *)(base + page_offset(page, page_stride, slot, slot_stride) * elem_bytes);
    };
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        U kept[kAhead], *to[kAhead];
        int from[kAhead], src_page[kAhead], dst_page[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int i = i0 + e;
            if (i0 > 0) ahead[e] = path[min(i, p.path_len - 1)];
            // (an entry at its own place is there already)
            from[e] = i < count && ahead[e] > i && ahead[e] < added ? ahead[e] : -1;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            src_page[e] = from[e] < 0 ? -1 : page_at(from[e]);
            dst_page[e] = from[e] < 0 ? -1 : page_at(i0 + e);
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const U *src = piece_at(from[e], src_page[e]);
            to[e] = src ? piece_at(i0 + e, dst_page[e]) : nullptr;
            if (to[e]) kept[e] = *src;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (to[e]) *to[e] = kept[e];
    }
}

typedef unsigned move4 __attribute__((ext_vector_type(4)));
typedef unsigned move2 __attribute__((ext_vector_type(2)));

}  // namespace

hipError_t launch_kv_move(const MoveParams &p, int elem_bytes, int unit, hipStream_t stream)
{
    const long long threads = 2ll * p.kv_heads * (p.row_bytes / unit);
    const dim3 grid((unsigned)p.batch.sequences, (unsigned)((threads + kThreads - 1) / kThreads));
    if (unit == 16) kv_move_kernel<move4><<<grid, kThreads, 0, stream>>>(p, elem_bytes);
    else if (unit == 8) kv_move_kernel<move2><<<grid, kThreads, 0, stream>>>(p, elem_bytes);
    else if (unit == 4) kv_move_kernel<unsigned><<<grid, kThreads, 0, stream>>>(p, elem_bytes);
    else kv_move_kernel<unsigned short><<<grid, kThreads, 0, stream>>>(p, elem_bytes);
    return hipGetLastError();
}

}  // namespace nnjit
