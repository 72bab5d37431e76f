// attn_decode: how a call is shared out over the card, and the join of units
// that span workgroups (the kernel over the keys is in decode_attn.h).
#include <algorithm>
#include <climits>

#include "decode.h"

namespace ilpm {

#define ILPM_ATTN_KERNELS(name)                                      \
    hipError_t attn_split_##name(const AttnArgs &a, hipStream_t stream); \
    int attn_card_##name(int dim);
ILPM_ATTN_KERNELS(f32)
ILPM_ATTN_KERNELS(f16)
ILPM_ATTN_KERNELS(f16_q32)
ILPM_ATTN_KERNELS(bf16)
ILPM_ATTN_KERNELS(bf16_q32)
#undef ILPM_ATTN_KERNELS

namespace {

constexpr int kMaxParts = 4 * kAttnCus;  // of a unit: workgroups of a call
constexpr float kLn2 = 0.69314718055994530942f;

__device__ inline void store_f32(void *p, int64_t i, int dtype, float v)
{
    if (dtype == ILPM_F32) ((float *)p)[i] = v;
    else if (dtype == ILPM_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// Joins the parts of the unit that workgroup blockIdx.x of attn_split began
// without ending it, for its head blockIdx.y: part 0 is that workgroup's, the
// others are those of the workgroups after it.  Group p of T threads adds
// parts p, p + 256 / T, ... in their order, V values a thread, then the groups'
// sums are added in theirs.
template <int V, int T> __global__ __launch_bounds__(256) void attn_join(AttnArgs a)
{
    constexpr int G = 256 / T;
    __shared__ float red[4], w[kMaxParts];
    __shared__ Pack<float, V> sum[G][T];
    const AttnPart u = a.parts[blockIdx.x];
    if (u.seq < 0) return;
    const int kvh = u.unit / a.blocks, in_group = (u.unit - kvh * a.blocks) * kAttnHeads + (int)blockIdx.y;
    if (in_group >= a.group) return;
    const int head = kvh * a.group + in_group, tid = threadIdx.x;
    auto slot = [&](int i) { return ((((int64_t)blockIdx.x + i) * 2 + (i == 0)) * a.part_heads + blockIdx.y); };
    float top = -INFINITY;
    for (int i = tid; i < u.count; i += 256) {
        w[i] = a.part_ml[slot(i) * 2];
        top = fmaxf(top, w[i]);
    }
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    for (int i = tid; i < u.count; i += 256) {
        w[i] = __builtin_amdgcn_exp2f(w[i] - base);
        l += a.part_ml[slot(i) * 2 + 1] * w[i];
    }
    for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = l;
    const int group = tid / T, d = tid % T * V;
    Pack<float, V> v = {};
    if (d < a.dim) {
#pragma unroll 8
        for (int i = group; i < u.count; i += G) {
            const Pack<float, V> p = *reinterpret_cast<const Pack<float, V> *>(a.part_o + slot(i) * a.dim + d);
#pragma unroll
            for (int k = 0; k < V; ++k) v.v[k] += p.v[k] * w[i];
        }
    }
    sum[group][tid % T] = v;
    __syncthreads();
    l = (red[0] + red[1]) + (red[2] + red[3]);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (tid < a.dim) {
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) x += sum[g][tid / V].v[tid % V];
        store_f32(a.out, (int64_t)u.seq * a.o_row + (int64_t)head * a.o_head + tid, a.q_dtype, x * inv);
    }
    if (tid == 0 && a.lse) a.lse[(int64_t)u.seq * a.q_heads + head] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

// Sequences that cannot have more than kWholeTiles tiles go a unit to a
// workgroup; else as many workgroups share all tiles as the card holds, or as
// there are smallest shares.
size_t attn_plan(AttnArgs *a, int cache_dtype, bool q32, int max_len)
{
    a->blocks = ceil_div(a->group, kAttnHeads);
    const int64_t units = (int64_t)a->n_seqs * a->kv_heads * a->blocks;
    const int64_t keys = a->window > 0 ? std::min(max_len, a->window) : max_len, tiles = std::max<int64_t>(1, (keys + 15) / 16);
    // (Tiles are counted in 32 bits.  Where a table could name more, there are units enough without a split.)
    const int64_t most = (((int64_t)a->capacity + 15) / 16 + kUnitCost) * units;
    a->split = tiles > kWholeTiles && units > 0 && (most < INT_MAX || units == 1);
    if (!a->split) {
        a->grid = (int)units;
        return 0;
    }
    const int card = cache_dtype == ILPM_F32   ? attn_card_f32(a->dim)
                     : cache_dtype == ILPM_F16 ? (q32 ? attn_card_f16_q32(a->dim) : attn_card_f16(a->dim))
                                               : (q32 ? attn_card_bf16_q32(a->dim) : attn_card_bf16(a->dim));
    a->grid = (int)std::min<int64_t>({card, kMaxParts, units * ((tiles + kUnitCost + kMinShare - 1) / kMinShare)});
    a->part_heads = std::min(a->group, kAttnHeads);
    return (size_t)a->grid * (sizeof(AttnPart) + 2 * a->part_heads * (size_t)(a->dim + 2) * sizeof(float));
}

void attn_workspace(AttnArgs *a, void *ws)
{
    a->parts = (AttnPart *)ws;
    a->part_o = (float *)(a->parts + a->grid);  // (16-byte aligned, as AttnPart has 16 bytes)
    a->part_ml = a->part_o + (size_t)a->grid * 2 * a->part_heads * a->dim;
}

hipError_t attn_launch(const AttnArgs &a, int cache_dtype, hipStream_t stream)
{
    const bool q32 = a.q_dtype == ILPM_F32;
    const hipError_t e = cache_dtype == ILPM_F32   ? attn_split_f32(a, stream)
                         : cache_dtype == ILPM_F16 ? (q32 ? attn_split_f16_q32(a, stream) : attn_split_f16(a, stream))
                                                   : (q32 ? attn_split_bf16_q32(a, stream) : attn_split_bf16(a, stream));
    if (e != hipSuccess || !a.split) return e;
    const dim3 grid(a.grid, a.part_heads);
    if (a.dim % 4) hipLaunchKernelGGL((attn_join<1, 256>), grid, dim3(256), 0, stream, a);
    else if (a.dim <= 64) hipLaunchKernelGGL((attn_join<4, 16>), grid, dim3(256), 0, stream, a);
    else if (a.dim <= 128) hipLaunchKernelGGL((attn_join<4, 32>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((attn_join<4, 64>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ilpm
