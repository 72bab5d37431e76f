// kv_copy: tokens' keys and values copied within the page pools.
//
// A token is two sets of kv_heads rows of head_dim values, so a copy moves
// pieces of up to 16 bytes, each read once and written once; what bounds it is
// the memory (6 forks of up to 4093 tokens, 163 MB both ways, 42 us: 3.9 TB/s, and 27
// us of what the caches still hold), or for the few tokens of a tree the chain of accesses
// before the first piece (counts, path, tables: 64 trees 4.9 us).
#include <algorithm>

#include "draft.h"

namespace ilpm {
namespace {

// Bytes of a token that a copy moves, from its place in a pool; -1: no place.
__device__ inline int64_t slot_of(const CopyArgs &a, const int32_t *table, int64_t stride, int max_pages, int seq, int64_t token)
{
    if (token < 0 || token >= (int64_t)max_pages * a.page_size) return -1;
    const int at = (int)(token / a.page_size);
    const int page = table[(int64_t)seq * stride + at];
    if (page < 0 || page >= a.n_pages) return -1;
    return (int64_t)page * a.page_size + (token - (int64_t)at * a.page_size);
}

// A token of row `seq` and where it goes, as slots over all pages; -1 where it
// is not copied (nor is one onto itself).
struct Move {
    int64_t from, to;
};

__device__ inline Move move_of(const CopyArgs &a, int seq, int64_t from, int64_t to)
{
    Move m;
    m.from = slot_of(a, a.src_table, a.src_table_stride, a.src_max_pages, seq, from);
    m.to = slot_of(a, a.dst_table, a.dst_table_stride, a.dst_max_pages, seq, to);
    if (m.from < 0 || m.to < 0 || m.from == m.to) m.from = m.to = -1;
    return m;
}

// Of token i of a path.
__device__ inline Move move_of_path(const CopyArgs &a, int seq, int i)
{
    if (i >= min(a.counts[seq], a.max_count)) return Move{-1, -1};
    const int step = a.path[(int64_t)seq * a.path_stride + i];
    if (step < 0) return Move{-1, -1};
    return move_of(a, seq, (int64_t)a.src_start[seq] + step, (int64_t)a.dst_start[seq] + i);
}

// The byte offset in a pool of a slot over all pages.
__device__ inline int64_t at_slot(const CopyArgs &a, int64_t slot, int64_t page_bytes, int64_t slot_bytes)
{
    const int64_t page = slot / a.page_size;
    return page * page_bytes + (slot - page * a.page_size) * slot_bytes;
}

struct Place {
    int64_t k_from, k_to, v_from, v_to;
};

__device__ inline Place place_of(const CopyArgs &a, Move m)
{
    if (m.from < 0) return Place{-1, -1, -1, -1};
    return Place{at_slot(a, m.from, a.k_page, a.k_slot), at_slot(a, m.to, a.k_page, a.k_slot),
                 at_slot(a, m.from, a.v_page, a.v_slot), at_slot(a, m.to, a.v_page, a.v_slot)};
}

// Pieces need the alignment of an element only.
template <int P> using Piece = Pack<unsigned short, P / 2>;

// With a path: a thread takes one piece of all of the row's tokens, and reads
// them all before it writes the first.  No other thread touches these bytes.
template <int P, int N> __global__ __launch_bounds__(256) void copy_path(CopyArgs a)
{
    __shared__ Place places[N];
    const int seq = blockIdx.y, tid = threadIdx.x;
    if (tid < N) places[tid] = place_of(a, move_of_path(a, seq, tid));
    __syncthreads();
    const int per_head = a.row_bytes / P, per = a.kv_heads * per_head;
    int i = (int)(blockIdx.x * 256 + tid);
    if (i >= 2 * per) return;
    const bool value = i >= per;
    if (value) i -= per;
    const int h = i / per_head, e = (i - h * per_head) * P;
    char *pool = value ? (char *)a.v + (int64_t)h * a.v_head + e : (char *)a.k + (int64_t)h * a.k_head + e;
    Piece<P> got[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int64_t from = value ? places[n].v_from : places[n].k_from;
        if (from >= 0) got[n] = load_loose<unsigned short, P / 2>((const unsigned short *)(pool + from));
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int64_t to = value ? places[n].v_to : places[n].k_to;
        if (to >= 0) store_loose<unsigned short, P / 2>((unsigned short *)(pool + to), got[n]);
    }
}

// Of a workgroup at a time.  (With 8 and 32, whose stores wait for fewer and for more others:
// 6 forks of 4000 tokens of 8 bf16 heads of 128 51.4 us, 48.2 and 47.7; 64 of 700 of 2 heads of 64
// 19.1, 15.9 and 18.7; 64 of 40 of 8 of 128 7.7, 6.6 and 10.7; 1 of 16000 of 8 f32 heads 60.3, 58.8
// and 62.8.)
constexpr int kTokens = 16;

// Without one: a thread takes one piece of kTokens tokens, and reads them all before
// it writes the first, so that as many reads are on their way.  (Stores are not: each is
// behind a condition, and waits for the one before it.)
template <int P> __global__ __launch_bounds__(256) void copy_rows(CopyArgs a)
{
    __shared__ Place places[kTokens];
    const int seq = blockIdx.y, tid = threadIdx.x, per_head = a.row_bytes / P, per = a.kv_heads * per_head;
    // Tokens that have places in both tables: no more than the grid was made for, whatever counts and starts are.
    const int64_t from = a.src_start[seq], to = a.dst_start[seq];
    const int64_t begin = max((int64_t)0, -min(from, to));
    const int64_t end = min((int64_t)min(a.counts[seq], a.max_count),
                            min((int64_t)a.src_max_pages * a.page_size - from, (int64_t)a.dst_max_pages * a.page_size - to));
    for (int64_t first = begin + (int64_t)blockIdx.x * kTokens; first < end; first += (int64_t)gridDim.x * kTokens) {
        if (tid < kTokens) places[tid] = place_of(a, first + tid < end ? move_of(a, seq, from + first + tid, to + first + tid) : Move{-1, -1});
        __syncthreads();
        for (int i0 = tid; i0 < 2 * per; i0 += 256) {
            const bool value = i0 >= per;
            const int i = value ? i0 - per : i0, h = i / per_head, e = (i - h * per_head) * P;
            char *pool = value ? (char *)a.v + (int64_t)h * a.v_head + e : (char *)a.k + (int64_t)h * a.k_head + e;
            Piece<P> got[kTokens];
#pragma unroll
            for (int n = 0; n < kTokens; ++n) {
                const int64_t from = value ? places[n].v_from : places[n].k_from;
                if (from >= 0) got[n] = load_loose<unsigned short, P / 2>((const unsigned short *)(pool + from));
            }
#pragma unroll
            for (int n = 0; n < kTokens; ++n) {
                const int64_t to = value ? places[n].v_to : places[n].k_to;
                if (to >= 0) store_loose<unsigned short, P / 2>((unsigned short *)(pool + to), got[n]);
            }
        }
        __syncthreads();  // the places have been read
    }
}

template <int P> hipError_t launch(const CopyArgs &a, hipStream_t stream)
{
    if (!a.path) {
        // (A workgroup for every kTokens that there may be: those beyond the counts end at once.)
        const int64_t most = std::min<int64_t>(a.max_count, (int64_t)std::min(a.src_max_pages, a.dst_max_pages) * a.page_size);
        const int64_t groups = std::min<int64_t>((most + kTokens - 1) / kTokens, 1 << 16);
        hipLaunchKernelGGL((copy_rows<P>), dim3((unsigned)groups, a.n_seqs), dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)((2ll * a.kv_heads * (a.row_bytes / P) + 255) / 256), a.n_seqs);
    if (a.max_count <= 8) hipLaunchKernelGGL((copy_path<P, 8>), grid, dim3(256), 0, stream, a);
    else if (a.max_count <= 16) hipLaunchKernelGGL((copy_path<P, 16>), grid, dim3(256), 0, stream, a);
    else if (P == 16 || a.max_count <= 32) hipLaunchKernelGGL((copy_path<P, 32>), grid, dim3(256), 0, stream, a);
    else if constexpr (P < 16) hipLaunchKernelGGL((copy_path<P, 64>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t copy_launch(const CopyArgs &a, hipStream_t stream)
{
    // (Of 64 tokens pieces of 8 bytes, so that all fit the registers: paths of 64 nodes in any order, 64 and 1
    // sequences of 8 bf16 heads of 128, 15.4 and 12.8 us, with pieces of 16 bytes 15.8 and 13.2; of 32 nodes both 9.1.)
    if (a.row_bytes % 16 == 0 && !(a.path && a.max_count > 32)) return launch<16>(a, stream);
    if (a.row_bytes % 8 == 0) return launch<8>(a, stream);
    if (a.row_bytes % 4 == 0) return launch<4>(a, stream);
    return launch<2>(a, stream);
}

}  // namespace ilpm
