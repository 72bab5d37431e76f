// verify_drafts: which nodes of a tree of drafted tokens are kept, and the next
// token, from the target's probabilities and given random numbers.
//
// The walk from the root needs a few values of the rows only; a whole row is read
// where it ends, to draw from what is left of it.  With draft rows that is, after
// m refused children of a node, max(a p - b q, 0) with a and b numbers: from
// w' = max(w / Z - q, 0) follow a' = a / Z and b' = b / Z + 1.  So a row is never
// stored, and w of any token is known from a and b.
//
// Sums are 64 bits: a row of 2^17 values in 32 would move the places where one
// token ends and the next begins by more than many a token's share.
#include <algorithm>

#include "draft.h"

namespace ilpm {
namespace {

// A probability as it counts: nothing that is not above 0, nothing beyond fp32.
template <typename T> __device__ inline float prob(T v)
{
    const float f = (float)v;
    return f > 0.f ? fminf(f, 3.402823466e38f) : 0.f;
}

__device__ inline double left_of(double a, double b, float p, float q)
{
    const double w = a * (double)p - b * (double)q;
    return w > 0. ? w : 0.;
}

constexpr int kThreads = 256;

// The sum over the workgroup, in all threads.
__device__ inline double sum_all(double v, double *lds)
{
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <typename T> __device__ inline const T *row_of(const void *base, int64_t seq_stride, int64_t node_stride, int seq, int node)
{
    return (const T *)base + (int64_t)seq * seq_stride + (int64_t)node * node_stride;
}

// A workgroup walks one sequence's tree, all of its threads alike; they are
// needed only where a node has several children and draft rows, for the sums
// after a refusal.
template <typename T> __global__ __launch_bounds__(kThreads) void verify_walk(VerifyArgs a)
{
    __shared__ double lds[4];
    const ilpm_verify_args &v = a.v;
    const int seq = blockIdx.x, lane = threadIdx.x & 63, n = v.n_nodes;
    const int64_t at = (int64_t)seq * n;
    // Lane i holds node i, and its probabilities below its parent.
    int parent = -2, token = -1;
    float u = 0.f, p = 0.f, q = 0.f;
    if (lane < n) {
        parent = v.parents[at + lane];
        token = v.tokens[at + lane];
        u = v.uniforms[at + lane];
        const bool known = token >= 0 && token < v.vocab;
        if (!known) token = -1;
        if (known && parent >= 0 && parent < lane) {
            p = prob(row_of<T>(v.target, v.target_seq_stride, v.target_node_stride, seq, parent)[token]);
            if (v.draft) q = prob(row_of<T>(v.draft, v.draft_seq_stride, v.draft_node_stride, seq, parent)[token]);
        }
    }
    const bool real = __builtin_amdgcn_readlane(parent, 0) == -1;
    int cur = 0, count = 1;
    int mine = -1;  // path[lane]
    double wa = 1., wb = 0., z = 1.;
    unsigned long long gone = 0;  // refused children of the current node
    unsigned long long kids = __builtin_amdgcn_ballot_w64(parent == 0 && lane > 0 && token >= 0);
    if (lane == 0) mine = 0;
    while (real && kids) {
        const int c = __builtin_ctzll(kids);
        kids &= kids - 1;
        const int x = __builtin_amdgcn_readlane(token, c);
        const double uc = (double)__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u), c));
        const float pc = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), c));
        const float qc = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, q), c));
        bool keep;
        double w;
        if (v.draft) {
            w = left_of(wa, wb, pc, qc);
            keep = z > 0. && uc * (double)qc * z < w;
        } else {
            // (A token that was refused before has nothing left.)
            const bool again = __builtin_amdgcn_ballot_w64(((gone >> lane) & 1) && token == x) != 0;
            w = again ? 0. : (double)pc;
            keep = z > 0. && uc * z < w;
        }
        if (keep) {
            cur = c;
            if (lane == count) mine = c;
            ++count;
            wa = z = 1.;
            wb = 0.;
            gone = 0;
            kids = __builtin_amdgcn_ballot_w64(parent == c && lane > c && token >= 0);
        } else if (!(z > 0.)) {
            continue;
        } else if (v.draft) {
            wa /= z;
            wb = wb / z + 1.;
            if (kids) {
                const T *pr = row_of<T>(v.target, v.target_seq_stride, v.target_node_stride, seq, cur);
                const T *qr = row_of<T>(v.draft, v.draft_seq_stride, v.draft_node_stride, seq, cur);
                double s = 0.;
                for (int i = threadIdx.x; i < v.vocab; i += kThreads) s += left_of(wa, wb, prob(pr[i]), prob(qr[i]));
                z = sum_all(s, lds);
            }
        } else {
            z -= w;
            gone |= 1ull << c;
        }
    }
    if (threadIdx.x < n) v.path[at + lane] = real ? mine : -1;
    if (threadIdx.x == 0) v.counts[seq] = real ? count : 0;
    VerifyEnd &end = a.ends[seq];
    if (threadIdx.x == 0) {
        end.node = real ? cur : -1;
        end.a = wa;
        end.b = wb;
        end.n_gone = __builtin_popcountll(gone);
    }
    if (threadIdx.x < 64 && ((gone >> lane) & 1)) end.gone[__builtin_popcountll(gone & ((1ull << lane) - 1))] = token;
}

// What is left of a row at its end's node, element by element.
template <typename T> struct Rest {
    const T *p, *q;
    double a, b;
    const unsigned *hole;  // a bit for each element of the chunk
    int first;
    __device__ double left(int i) const
    {
        const float pi = prob(p[i]);
        if (q) return left_of(a, b, pi, prob(q[i]));
        return (hole[(i - first) >> 5] >> ((i - first) & 31)) & 1 ? 0. : (double)pi;
    }
};

template <typename T> __device__ inline Rest<T> rest_of(const VerifyArgs &a, int seq, const VerifyEnd &end, int chunk, unsigned *hole)
{
    const ilpm_verify_args &v = a.v;
    const int first = chunk * kVerifyChunk;
    if (threadIdx.x < kVerifyChunk / 32) hole[threadIdx.x] = 0;
    __syncthreads();
    if ((int)threadIdx.x < end.n_gone) {
        const int i = end.gone[threadIdx.x] - first;
        if (i >= 0 && i < kVerifyChunk) atomicOr(&hole[i >> 5], 1u << (i & 31));
    }
    __syncthreads();
    Rest<T> r;
    r.p = row_of<T>(v.target, v.target_seq_stride, v.target_node_stride, seq, end.node);
    r.q = v.draft ? row_of<T>(v.draft, v.draft_seq_stride, v.draft_node_stride, seq, end.node) : nullptr;
    r.a = end.a;
    r.b = end.b;
    r.hole = hole;
    r.first = first;
    return r;
}

template <typename T> __global__ __launch_bounds__(kThreads) void verify_sums(VerifyArgs a)
{
    __shared__ double lds[4];
    __shared__ unsigned hole[kVerifyChunk / 32];
    const int seq = blockIdx.y, chunk = blockIdx.x;
    const VerifyEnd &end = a.ends[seq];
    if (end.node < 0) return;
    const Rest<T> r = rest_of<T>(a, seq, end, chunk, hole);
    const int last = (int)min((int64_t)a.v.vocab, (int64_t)r.first + kVerifyChunk);
    double left = 0., all = 0.;
    for (int i = r.first + (int)threadIdx.x; i < last; i += kThreads) {
        left += r.left(i);
        all += (double)prob(r.p[i]);
    }
    left = sum_all(left, lds);
    all = sum_all(all, lds);
    if (threadIdx.x == 0) a.sums[(int64_t)seq * a.chunks + chunk] = VerifySum{left, all};
}

// Sums up to and with each thread's value.
__device__ inline double scan_all(double v, double *lds, double *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    const double s0 = lds[0], s1 = s0 + lds[1], s2 = s1 + lds[2];
    *total = s2 + lds[3];
    return v + (wave == 0 ? 0. : wave == 1 ? s0 : wave == 2 ? s1 : s2);
}

template <typename T> __global__ __launch_bounds__(kThreads) void verify_pick(VerifyArgs a)
{
    __shared__ double lds[4], before;
    __shared__ unsigned hole[kVerifyChunk / 32];
    __shared__ int found, positive;
    const ilpm_verify_args &v = a.v;
    const int seq = blockIdx.x, tid = threadIdx.x;
    const VerifyEnd &end = a.ends[seq];
    if (end.node < 0) {
        if (tid == 0) v.next_tokens[seq] = -1;
        return;
    }
    const VerifySum *sums = a.sums + (int64_t)seq * a.chunks;
    double left = 0., all = 0., part;
    for (int c0 = 0; c0 < a.chunks; c0 += kThreads) {
        const VerifySum s = c0 + tid < a.chunks ? sums[c0 + tid] : VerifySum{0., 0.};
        scan_all(s.left, lds, &part);
        left += part;
        scan_all(s.all, lds, &part);
        all += part;
    }
    const bool whole = !(left > 0.);  // nothing is left: the row itself
    const double total = whole ? all : left;
    if (!(total > 0.)) {
        if (tid == 0) v.next_tokens[seq] = -1;
        return;
    }
    const double want = (double)v.uniforms[(int64_t)seq * v.n_nodes] * total;
    if (tid == 0) found = INT_MAX, positive = -1;
    // The first chunk whose sum passes `want`, else the last one that has any.
    double carry = 0.;
    for (int c0 = 0; c0 < a.chunks; c0 += kThreads) {
        const VerifySum s = c0 + tid < a.chunks ? sums[c0 + tid] : VerifySum{0., 0.};
        const double own = whole ? s.all : s.left;
        const double up_to = carry + scan_all(own, lds, &part);
        if (own > 0.) {
            if (up_to > want) atomicMin(&found, c0 + tid);
            atomicMax(&positive, c0 + tid);
        }
        __syncthreads();
        if (found == c0 + tid || (found == INT_MAX && positive == c0 + tid)) before = up_to - own;
        __syncthreads();
        if (found != INT_MAX) break;
        carry += part;
    }
    const int chunk = found != INT_MAX ? found : positive;
    const double rest_want = want - before;
    __syncthreads();
    if (tid == 0) found = INT_MAX, positive = -1;
    const Rest<T> r = rest_of<T>(a, seq, end, chunk, hole);
    const int last = (int)min((int64_t)v.vocab, (int64_t)r.first + kVerifyChunk);
    carry = 0.;
    for (int i0 = r.first; i0 < last; i0 += kThreads) {
        const int i = i0 + tid;
        const double w = i < last ? (whole ? (double)prob(r.p[i]) : r.left(i)) : 0.;
        const double up_to = carry + scan_all(w, lds, &part);
        if (w > 0.) {
            if (up_to > rest_want) atomicMin(&found, i);
            atomicMax(&positive, i);
        }
        carry += part;
    }
    __syncthreads();
    if (tid == 0) v.next_tokens[seq] = found != INT_MAX ? found : positive;
}

template <typename T> hipError_t launch(const VerifyArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((verify_walk<T>), dim3(a.v.n_seqs), dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL((verify_sums<T>), dim3(a.chunks, a.v.n_seqs), dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL((verify_pick<T>), dim3(a.v.n_seqs), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

size_t ends_bytes(int n_seqs) { return ((size_t)n_seqs * sizeof(VerifyEnd) + 15) / 16 * 16; }

}  // namespace

size_t verify_plan(VerifyArgs *a)
{
    a->chunks = (int)(((int64_t)a->v.vocab + kVerifyChunk - 1) / kVerifyChunk);
    return ends_bytes(a->v.n_seqs) + (size_t)a->v.n_seqs * (size_t)a->chunks * sizeof(VerifySum);
}

void verify_workspace(VerifyArgs *a, void *ws)
{
    a->ends = (VerifyEnd *)ws;
    a->sums = (VerifySum *)((char *)ws + ends_bytes(a->v.n_seqs));
}

hipError_t verify_launch(const VerifyArgs &a, hipStream_t stream)
{
    if (a.v.dtype == ILPM_F32) return launch<float>(a, stream);
    if (a.v.dtype == ILPM_F16) return launch<_Float16>(a, stream);
    return launch<__bf16>(a, stream);
}

}  // namespace ilpm
