// attn_decode: attention of one new token a sequence over a paged cache,
//   x_j = scale <q, k_j>,  out = sum e^(x_j - m) v_j / sum e^(x_j - m),  m = max x_j,
// in one pass over the keys with the running maximum and sum of the softmax,
// split over the length and joined.
//
// Both products run on the fp32 matrix cores (v_mfma_f32_16x16x4_f32) for every
// cache type: 16 keys x 16 query heads of one key head.  The first gives the
// scores transposed, S[key][head] = sum_d K[key][d] Q[head][d], so that lane
// (n, g) = (lane % 16, lane / 16) holds keys 4g..4g+3 of head n.  That is the
// layout in which the second one wants its operand, O[d][head] = sum_key
// V[key][d] P[key][head], with keys 4g + r as the contraction of instruction
// r: the probabilities never leave their lane, the statistics of a head are
// one value per lane, and a lane's V operand is V[4g + r][d], an element of a
// row that it loads as it lies in memory.
#include "decode.h"

#include <algorithm>

namespace ilpm {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kSeg = 512;        // keys whose places a workgroup holds in LDS
constexpr int kHeads = 16;       // query heads of a workgroup
constexpr int kMaxSplits = 256;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ inline float load_f32(const void *p, int64_t i, int dtype)
{
    if (dtype == ILPM_F32) return ((const float *)p)[i];
    if (dtype == ILPM_F16) return (float)((const _Float16 *)p)[i];
    return (float)((const __bf16 *)p)[i];
}

__device__ inline void store_f32(void *p, int64_t i, int dtype, float v)
{
    if (dtype == ILPM_F32) ((float *)p)[i] = v;
    else if (dtype == ILPM_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// The keys of a sequence that the window leaves: [first, end).
__device__ inline void visible_range(const AttnArgs &a, int seq, int *first, int *end)
{
    const int n = min(max(a.lengths[seq], 0), a.capacity);
    *end = n;
    // (The window counts from the sequence's own length, also where the table ends before it.)
    *first = a.window > 0 ? (int)min((int64_t)n, max((int64_t)a.lengths[seq] - a.window, (int64_t)0)) : 0;
}

// Splits that a sequence's visible keys fill.
__device__ inline int splits_of(const AttnArgs &a, int keys)
{
    return min((keys + a.chunk - 1) / a.chunk, a.splits);
}

// N elements of a row from element d on, where `vec` in one access; elements
// from `dim` on are 0.
template <typename T, int N, bool ALIGNED> __device__ inline void load_row(const T *row, int d, int dim, T (&to)[N])
{
    if constexpr (ALIGNED) {
        Pack<T, N> p = {};
        if (d < dim) p = *reinterpret_cast<const Pack<T, N> *>(row + d);
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = p.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = d + i < dim ? row[d + i] : (T)0.f;
    }
}

// DC: the head size's class (64, 128 or 256).  ALIGNED: rows are multiples of
// 16 bytes on 16-byte boundaries.
template <typename TC, int DC, bool ALIGNED> __global__ __launch_bounds__(256) void attn_split(AttnArgs a)
{
    constexpr int KV = 16 / (int)sizeof(TC);                  // elements of a K load
    constexpr int NK = DC / (4 * KV);                         // K loads of a lane
    constexpr int VV = KV < DC / 16 ? KV : DC / 16;           // elements of a V load
    constexpr int NV = DC / (16 * VV);                        // V loads of a lane and key
    __shared__ int64_t koff[kSeg], voff[kSeg];                // places of the segment's keys, -1 where not seen
    __shared__ float sm[4][kHeads], sl[4][kHeads];
    __shared__ float so[2][64][NV * VV * 4 + 1];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n16 = lane & 15, g = lane >> 4;
    const int blocks = (a.group + kHeads - 1) / kHeads;       // of a key head's query heads
    int64_t id = blockIdx.x;
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int hb = (int)(id % blocks);
    id /= blocks;
    const int kvh = (int)(id % a.kv_heads), seq = (int)(id / a.kv_heads);
    const int in_group = hb * kHeads + n16;                   // this lane's query head
    const bool has_head = in_group < a.group;
    const int head = kvh * a.group + in_group;

    int first, end;
    visible_range(a, seq, &first, &end);
    const int ns = splits_of(a, end - first);
    if (split >= max(ns, 1)) return;
    const int k0 = first + split * a.chunk;
    const int k1 = split == a.splits - 1 ? end : min(k0 + a.chunk, end);

    float q[NK][KV];
#pragma unroll
    for (int c = 0; c < NK; ++c)
#pragma unroll
        for (int j = 0; j < KV; ++j) {
            const int d = (g + 4 * c) * KV + j;
            q[c][j] = has_head && d < a.dim
                          ? load_f32(a.q, (int64_t)seq * a.q_row + (int64_t)head * a.q_head + d, a.q_dtype)
                          : 0.f;
        }

    floatx4 o[NV * VV];
#pragma unroll
    for (int i = 0; i < NV * VV; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const TC *kh = (const TC *)a.k + (int64_t)kvh * a.k_head;
    const TC *vh = (const TC *)a.v + (int64_t)kvh * a.v_head;
    const float scale2 = a.softcap > 0.f ? a.scale / a.softcap : a.scale * kLog2e;
    const float cap2 = a.softcap * kLog2e;

    for (int seg = k0; seg < k1; seg += kSeg) {
        const int count = min(kSeg, k1 - seg);
        __syncthreads();
        for (int i = threadIdx.x; i < kSeg; i += 256) {
            const int key = seg + i;
            int64_t ko = -1, vo = -1;
            if (i < count && (!a.mask || (key < a.mask_len && a.mask[(int64_t)seq * a.mask_stride + key]))) {
                const int at = key / a.page_size, slot = key - at * a.page_size;
                const int page = a.table[(int64_t)seq * a.table_stride + at];
                if (page >= 0 && page < a.n_pages) {
                    ko = (int64_t)page * a.k_page + (int64_t)slot * a.k_slot;
                    vo = (int64_t)page * a.v_page + (int64_t)slot * a.v_slot;
                }
            }
            koff[i] = ko;
            voff[i] = vo;
        }
        __syncthreads();
        for (int t = wave * 16; t < count; t += 64) {
            // K row of key n16, V rows of keys 4g + r; a key not seen reads the
            // pool's first row, and none of it is used.
            TC kr[NK][KV], vr[4][NV][VV];
            const TC *krow = kh + max(koff[t + n16], (int64_t)0);
#pragma unroll
            for (int c = 0; c < NK; ++c) load_row<TC, KV, ALIGNED>(krow, (g + 4 * c) * KV, a.dim, kr[c]);
            bool seen[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t vo = voff[t + 4 * g + r];
                seen[r] = vo >= 0;
                const TC *vrow = vh + max(vo, (int64_t)0);
#pragma unroll
                for (int c = 0; c < NV; ++c) load_row<TC, VV, ALIGNED>(vrow, (n16 + 16 * c) * VV, a.dim, vr[r][c]);
            }
            floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NK; ++c)
#pragma unroll
                for (int j = 0; j < KV; ++j)
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32((float)kr[c][j], q[c][j], s, 0, 0, 0);
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float x = s[r] * scale2;
                if (a.softcap > 0.f) x = cap2 * tanhf(x);
                s[r] = seen[r] ? x : -INFINITY;
                top = fmaxf(top, s[r]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top);
            const float base = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m - base);
            m = m_new;
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] - base);
            l = l * alpha + ((p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
            for (int i = 0; i < NV * VV; ++i) o[i] *= alpha;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int j = 0; j < VV; ++j)
                        o[c * VV + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(seen[r] ? (float)vr[r][c][j] : 0.f, p[r],
                                                                            o[c * VV + j], 0, 0, 0);
        }
    }

    // Join the four waves: l first over the lanes of a head, then all to their
    // common maximum.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        sm[wave][n16] = m;
        sl[wave][n16] = l;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(sm[0][n16], sm[1][n16]), fmaxf(sm[2][n16], sm[3][n16]));
    const float base = top == -INFINITY ? 0.f : top;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) l += sl[w][n16] * __builtin_amdgcn_exp2f(sm[w][n16] - base);
    const float f = __builtin_amdgcn_exp2f(m - base);
#pragma unroll
    for (int i = 0; i < NV * VV; ++i) o[i] *= f;
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int i = 0; i < NV * VV; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) so[wave - half][lane][i * 4 + r] = o[i][r];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int i = 0; i < NV * VV; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] += so[wave][lane][i * 4 + r];
        }
    }
    if (wave != 0 || !has_head) return;
    const bool whole = ns <= 1;
    const int64_t row = (int64_t)seq * a.q_heads + head;
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    float *part = whole ? nullptr : a.part_o + (row * a.splits + split) * a.dim;
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VV; ++j) {
                const int d = (4 * g + r + 16 * c) * VV + j;
                if (d >= a.dim) continue;
                const float v = o[c * VV + j][r] * inv;
                if (whole) store_f32(a.out, (int64_t)seq * a.o_row + (int64_t)head * a.o_head + d, a.q_dtype, v);
                else part[d] = v;
            }
    if (g == 0) {
        if (whole) {
            if (a.lse) a.lse[row] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
        } else {
            float *ml = a.part_ml + (row * a.splits + split) * 2;
            ml[0] = top;
            ml[1] = l;
        }
    }
}

// Joins the splits of a row (a sequence's query head), in their order.
__global__ __launch_bounds__(256) void attn_join(AttnArgs a)
{
    __shared__ float w[kMaxSplits];
    const int64_t row = blockIdx.x;
    const int seq = (int)(row / a.q_heads), head = (int)(row % a.q_heads);
    int first, end;
    visible_range(a, seq, &first, &end);
    const int ns = splits_of(a, end - first);
    if (ns <= 1) return;
    const float *ml = a.part_ml + row * a.splits * 2;
    float top = -INFINITY;
    for (int i = 0; i < ns; ++i) top = fmaxf(top, ml[2 * i]);
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    for (int i = 0; i < ns; ++i) l += ml[2 * i + 1] * __builtin_amdgcn_exp2f(ml[2 * i] - base);
    for (int i = threadIdx.x; i < ns; i += 256) w[i] = __builtin_amdgcn_exp2f(ml[2 * i] - base);
    __syncthreads();
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float *part = a.part_o + row * a.splits * a.dim;
    for (int d = threadIdx.x; d < a.dim; d += 256) {
        float v = 0.f;
        for (int i = 0; i < ns; ++i) v += part[(int64_t)i * a.dim + d] * w[i];
        store_f32(a.out, (int64_t)seq * a.o_row + (int64_t)head * a.o_head + d, a.q_dtype, v * inv);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

int blocks_of(const AttnArgs &a) { return a.kv_heads * ceil_div(a.group, kHeads); }

template <typename TC, int DC> hipError_t launch(const AttnArgs &a, bool aligned, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.n_seqs * blocks_of(a) * a.splits));
    if (aligned) hipLaunchKernelGGL((attn_split<TC, DC, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((attn_split<TC, DC, false>), grid, dim3(256), 0, stream, a);
    if (a.splits > 1)
        hipLaunchKernelGGL(attn_join, dim3((unsigned)((int64_t)a.n_seqs * a.q_heads)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <typename TC> hipError_t launch_dim(const AttnArgs &a, hipStream_t stream)
{
    const int64_t step = 16 / (int64_t)sizeof(TC);
    const bool aligned = a.dim % step == 0 && ((uintptr_t)a.k | (uintptr_t)a.v) % 16 == 0 &&
                         (a.k_page | a.k_slot | a.k_head | a.v_page | a.v_slot | a.v_head) % step == 0;
    if (a.dim <= 64) return launch<TC, 64>(a, aligned, stream);
    if (a.dim <= 128) return launch<TC, 128>(a, aligned, stream);
    return launch<TC, 256>(a, aligned, stream);
}

}  // namespace

size_t attn_plan(AttnArgs *a, int max_len)
{
    const int64_t units = (int64_t)a->n_seqs * blocks_of(*a);
    const int64_t keys = std::max(1, std::min(max_len, a->window > 0 ? a->window : max_len));
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>({2048 / std::max<int64_t>(units, 1), (keys + 127) / 128,
                                                                 (int64_t)kMaxSplits}));
    const int64_t per = (keys + want - 1) / want;
    a->chunk = (int)std::min<int64_t>((per + 63) / 64 * 64, 0x7fffffc0);
    a->splits = (int)((keys + a->chunk - 1) / a->chunk);
    if (a->splits <= 1) return 0;
    return sizeof(float) * (size_t)a->n_seqs * a->q_heads * a->splits * (size_t)(a->dim + 2);
}

hipError_t attn_launch(const AttnArgs &a, int cache_dtype, hipStream_t stream)
{
    if (cache_dtype == ILPM_F32) return launch_dim<float>(a, stream);
    if (cache_dtype == ILPM_F16) return launch_dim<_Float16>(a, stream);
    return launch_dim<__bf16>(a, stream);
}

}  // namespace ilpm
