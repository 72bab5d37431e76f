// attn_tree: attention of drafted nodes over a paged cache and the nodes above
// them.
#include <climits>

#include "draft.h"

namespace ilpm {
namespace {

// The nodes that each node sees (itself and those above it), as bits; 0: no
// node.  Lane i holds node i.  Whoever is above whom is followed by doubling.
__device__ inline unsigned long long seen_nodes(int parent, int lane, int n)
{
    bool ok = lane < n && parent >= -1 && parent < lane;
    int up = ok ? parent : -1;
    unsigned lo = lane < 32 ? 1u << lane : 0, hi = lane >= 32 ? 1u << (lane - 32) : 0;
#pragma unroll 1
    for (int d = 1; d < 64; d <<= 1) {
        const int from = up < 0 ? lane : up;
        const unsigned l = __shfl(lo, from), h = __shfl(hi, from);
        const int u = __shfl(up, from), k = __shfl((int)ok, from);
        lo |= l;
        hi |= h;
        ok = ok && k;
        up = up < 0 ? -1 : u;
    }
    return ok ? (unsigned long long)hi << 32 | lo : 0ull;
}

__device__ inline float read_any(const void *p, int64_t i, int dtype)
{
    if (dtype == ILPM_F32) return ((const float *)p)[i];
    if (dtype == ILPM_F16) return (float)((const _Float16 *)p)[i];
    return (float)((const __bf16 *)p)[i];
}
__device__ inline void write_any(void *p, int64_t i, int dtype, float v)
{
    if (dtype == ILPM_F32) ((float *)p)[i] = v;
    else if (dtype == ILPM_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// One workgroup for a head of a node, a key a thread and step.
__global__ __launch_bounds__(256) void tree_plain(TreeArgs t, int cache_dtype)
{
    __shared__ float query[256], probs[256], red[4];
    __shared__ int64_t rows[256];
    const AttnArgs &a = t.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int head = blockIdx.x % a.q_heads, row = blockIdx.x / a.q_heads, seq = row / t.n_nodes, node = row - seq * t.n_nodes;
    const int kvh = head / a.group;
    const unsigned long long bits = seen_nodes(lane < t.n_nodes ? t.parents[(int64_t)seq * t.n_nodes + lane] : -2, lane, t.n_nodes);
    const int my_depth = __builtin_popcountll(bits) - 1;
    const unsigned long long above = __shfl(bits, node);
    const int depth = __shfl(my_depth, node);
    const int64_t length = max(a.lengths[seq], 0), place = length + depth;
    for (int d = tid; d < a.dim; d += 256) query[d] = read_any(a.q, (int64_t)row * a.q_row + (int64_t)head * a.q_head + d, a.q_dtype);
    __syncthreads();
    float m = -INFINITY, l = 0.f, o = 0.f;
    const int64_t end = above ? min((int64_t)a.capacity, length + t.n_nodes) : 0;
    for (int64_t k0 = 0; k0 < end; k0 += 256) {
        const int64_t key = k0 + tid;
        bool seen = key < end;
        int64_t at = key;
        const int n = (int)min(max(key - length, (int64_t)0), (int64_t)63), dn = __shfl(my_depth, n);  // (lanes' nodes differ: all take part)
        if (seen && key >= length) {
            seen = (above >> (key - length)) & 1;
            at = length + dn;
        }
        if (a.window > 0 && at <= place - a.window && at >= t.sinks) seen = false;
        float x = -INFINITY;
        int64_t page = -1, slot = 0;
        if (seen) {
            const int p = (int)(key / a.page_size);
            slot = key - (int64_t)p * a.page_size;
            page = a.table[(int64_t)seq * a.table_stride + p];
            if (page < 0 || page >= a.n_pages) seen = false;
            if (a.mask && (key >= a.mask_len || !a.mask[(int64_t)seq * a.mask_stride + key])) seen = false;
        }
        if (seen) {
            const int64_t at_k = page * a.k_page + slot * a.k_slot + (int64_t)kvh * a.k_head;
            float s = 0.f;
            for (int d = 0; d < a.dim; ++d) s += query[d] * read_any(a.k, at_k + d, cache_dtype);
            x = s * a.scale;
            if (a.softcap > 0.f) x = a.softcap * tanhf(x / a.softcap);
        }
        float top = x;
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        __syncthreads();
        if (lane == 0) red[wave] = top;
        __syncthreads();
        const float now = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float base = now == -INFINITY ? 0.f : now, alpha = expf(m - base);
        m = now;
        const float p = seen ? expf(x - base) : 0.f;
        probs[tid] = p;
        rows[tid] = seen ? page * a.v_page + slot * a.v_slot + (int64_t)kvh * a.v_head : -1;
        float sum = p;
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        __syncthreads();
        if (lane == 0) red[wave] = sum;
        __syncthreads();
        l = l * alpha + (red[0] + red[1]) + (red[2] + red[3]);
        o *= alpha;
        if (tid < a.dim)
            for (int j = 0; j < 256; ++j)
                if (rows[j] >= 0) o += probs[j] * read_any(a.v, rows[j] + tid, cache_dtype);
        __syncthreads();
    }
    if (tid < a.dim) write_any(a.out, (int64_t)row * a.o_row + (int64_t)head * a.o_head + tid, a.q_dtype, l == 0.f ? 0.f : o / l);
    if (tid == 0 && a.lse) a.lse[(int64_t)row * a.q_heads + head] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

size_t tree_plan(TreeArgs *, int, bool, int) { return 0; }
void tree_workspace(TreeArgs *, void *) {}

hipError_t tree_launch(const TreeArgs &t, int cache_dtype, hipStream_t stream)
{
    hipLaunchKernelGGL(tree_plain, dim3((unsigned)(t.a.n_seqs * t.n_nodes * t.a.q_heads)), dim3(256), 0, stream, t, cache_dtype);
    return hipGetLastError();
}

}  // namespace ilpm
