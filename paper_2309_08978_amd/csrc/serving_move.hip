// The keys and values of accepted nodes of drafted trees go to the places behind
// the cached ones.
//
// Node path[i] of the new tokens moves to new token i's place, i <= path[i].  A
// workgroup takes kPieces pieces (16 bytes, where alignment allows) of a sequence's key and value
// rows and moves them for all i, a thread a piece and entry, kEntries entries at a time: everything is loaded,
// then, behind a barrier, stored.  No workgroup touches another's pieces, and since later i
// read at or behind themselves, stores of earlier ones never reach what is still to be read.
// All latency: lengths and path, then the page table, then the rows.  (A thread for all
// entries of a piece, eight or sixteen loads ahead, took 4.2 to 7.8 us on the device for six entries of four sequences.)
#include "serving.h"

namespace nnjit {

namespace {

constexpr int kPieces = 16, kEntries = 16;

template <typename U>
__global__ void __launch_bounds__(kPieces * kEntries)
kv_move_kernel(MoveParams p, int elem_bytes)
{
    const int b = blockIdx.x, i0 = threadIdx.x / kPieces;
    const int *path = p.path + (long long)b * p.ld_path;
    int from = i0 < p.path_len ? path[i0] : -1;                      // asked for before what says whether it counts
    const PageBatch &batch = p.batch;
    const int q0 = min(max(batch.q_start[b], 0), batch.tokens);
    const int added = min(max(batch.q_start[b + 1] - q0, 0), batch.tokens - q0);
    const long long room = min((long long)batch.table_pages * p.pool.page_size.d, kMaxKeys);
    // place of the sequence's new token 0: from the starts as they stand, as appends and attention take it, though the
    // batch may hold fewer rows
    const long long past = (long long)batch.kv_len[b] - ((long long)batch.q_start[b + 1] - q0);
    const int count = min(min(max(p.accepted[b], 0), p.path_len), added);     // (entries read behind their own place: none from `added` on)
    const int *table = batch.page_table + (long long)b * batch.ld_table;

    const int pieces = p.row_bytes / (int)sizeof(U);                 // of a head's row
    const int piece = blockIdx.y * kPieces + threadIdx.x % kPieces;
    const bool mine = piece < 2 * p.kv_heads * pieces;
    const bool value = piece >= p.kv_heads * pieces;
    const int in = value ? piece - p.kv_heads * pieces : piece, head = in / pieces;
    char *base = (char *)(value ? p.pool.v : p.pool.k) + (value ? p.pool.v_head : p.pool.k_head) * head * elem_bytes +
                 (long long)(in - head * pieces) * sizeof(U);
    const unsigned page_stride = value ? p.pool.v_page : p.pool.k_page, slot_stride = value ? p.pool.v_tok : p.pool.k_tok;

    // (unsigned: the last step of almost 2^31 entries passes 31 bits)
    for (unsigned first = 0; first < (unsigned)count; first += kEntries) {
        const unsigned i = first + i0;
        if (first > 0) from = i < (unsigned)p.path_len ? path[i] : -1;
        // (an entry at its own place is there already)
        const long long src = past + from, dst = past + i;
        bool moves = mine && i < (unsigned)count && from > (int)i && from < added && dst >= 0 && src < room;
        U kept = {};
        U *to = nullptr;
        if (moves) {
            const int at_src = p.pool.page_size.quot((int)src), at_dst = p.pool.page_size.quot((int)dst);
            const int src_page = table[at_src], dst_page = table[at_dst];
            moves = src_page >= 0 && src_page < p.pool.pages && dst_page >= 0 && dst_page < p.pool.pages;
            if (moves) {
                const int size = p.pool.page_size.d;
                kept = *(const U *)(base + page_offset(src_page, page_stride, (int)src - at_src * size, slot_stride) * elem_bytes);
                to = (U *)(base + page_offset(dst_page, page_stride, (int)dst - at_dst * size, slot_stride) * elem_bytes);
            }
        }
        __syncthreads();
        if (moves) *to = kept;
        __syncthreads();
    }
}

typedef unsigned move4 __attribute__((ext_vector_type(4)));
typedef unsigned move2 __attribute__((ext_vector_type(2)));

}  // namespace

hipError_t launch_kv_move(const MoveParams &p, int elem_bytes, int unit, hipStream_t stream)
{
    const long long all = 2ll * p.kv_heads * (p.row_bytes / unit);
    const dim3 grid((unsigned)p.batch.sequences, (unsigned)((all + kPieces - 1) / kPieces));
    constexpr int threads = kPieces * kEntries;
    if (unit == 16) kv_move_kernel<move4><<<grid, threads, 0, stream>>>(p, elem_bytes);
    else if (unit == 8) kv_move_kernel<move2><<<grid, threads, 0, stream>>>(p, elem_bytes);
    else if (unit == 4) kv_move_kernel<unsigned><<<grid, threads, 0, stream>>>(p, elem_bytes);
    else kv_move_kernel<unsigned short><<<grid, threads, 0, stream>>>(p, elem_bytes);
    return hipGetLastError();
}

}  // namespace nnjit
