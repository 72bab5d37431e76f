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

constexpr float kLn2 = 0.69314718055994530942f;

__device__ inline void store_f32(void *p, int64_t i, int dtype, float v)
{
    if (dtype == ILPM_F32) ((float *)p)[i] = v;
    else if (dtype == ILPM_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// Joins the parts of the unit that workgroup blockIdx.x of attn_split began
// without ending it, for its head blockIdx.y: part 0 is that workgroup's, the
// others are those of the workgroups after it.  Thread (p, d) adds parts p, p +
// 8, ... of value d in their order, then the eight sums are added in theirs.
__global__ __launch_bounds__(256) void attn_join(AttnArgs a)
{
    __shared__ float red[4];
    __shared__ float sum[8][256];
    const AttnPart u = a.parts[blockIdx.x];
    if (u.seq < 0) return;
    const int kvh = u.unit / a.blocks, in_group = (u.unit - kvh * a.blocks) * kAttnHeads + (int)blockIdx.y;
    if (in_group >= a.group) return;
    const int head = kvh * a.group + in_group, tid = threadIdx.x;
    auto slot = [&](int i) { return ((((int64_t)blockIdx.x + i) * 2 + (i == 0)) * a.part_heads + blockIdx.y); };
    float top = -INFINITY;
    for (int i = tid; i < u.count; i += 256) top = fmaxf(top, a.part_ml[slot(i) * 2]);
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    for (int i = tid; i < u.count; i += 256) l += a.part_ml[slot(i) * 2 + 1] * __builtin_amdgcn_exp2f(a.part_ml[slot(i) * 2] - base);
    for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = l;
    const int part = tid >> 5;
    float v[8] = {};
#pragma unroll 4
    for (int i = part; i < u.count; i += 8) {
        const float w = __builtin_amdgcn_exp2f(a.part_ml[slot(i) * 2] - base);
        const float *po = a.part_o + slot(i) * a.dim;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int d = (tid & 31) + 32 * k;
            if (d < a.dim) v[k] += po[d] * w;
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[part][(tid & 31) + 32 * k] = v[k];
    __syncthreads();
    l = (red[0] + red[1]) + (red[2] + red[3]);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (tid < a.dim) {
        const float x = ((sum[0][tid] + sum[1][tid]) + (sum[2][tid] + sum[3][tid])) + ((sum[4][tid] + sum[5][tid]) + (sum[6][tid] + sum[7][tid]));
        store_f32(a.out, (int64_t)u.seq * a.o_row + (int64_t)head * a.o_head + tid, a.q_dtype, x * inv);
    }
    if (tid == 0 && a.lse) a.lse[(int64_t)u.seq * a.q_heads + head] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

// Sequences that cannot have more keys than two smallest shares go a unit to a
// workgroup; else as many workgroups share all tiles as the card holds, or as
// there are smallest shares.
size_t attn_plan(AttnArgs *a, int cache_dtype, bool q32, int max_len)
{
    a->blocks = ceil_div(a->group, kAttnHeads);
    const int64_t units = (int64_t)a->n_seqs * a->kv_heads * a->blocks;
    const int64_t keys = a->window > 0 ? std::min(max_len, a->window) : max_len, tiles = std::max<int64_t>(1, (keys + 15) / 16);
    // (Tiles are counted in 32 bits.  Where a table could name more, there are units enough without a split.)
    const int64_t most = ((int64_t)a->capacity + 15) / 16 * units;
    a->split = tiles > 2 * kMinShare && units > 0 && (most < INT_MAX || units == 1);
    if (!a->split) {
        a->grid = (int)units;
        return 0;
    }
    const int card = cache_dtype == ILPM_F32   ? attn_card_f32(a->dim)
                     : cache_dtype == ILPM_F16 ? (q32 ? attn_card_f16_q32(a->dim) : attn_card_f16(a->dim))
                                               : (q32 ? attn_card_bf16_q32(a->dim) : attn_card_bf16(a->dim));
    a->grid = (int)std::min<int64_t>(card, (units * tiles + kMinShare - 1) / kMinShare);
    a->part_heads = std::min(a->group, kAttnHeads);
    return (size_t)a->grid * (sizeof(AttnPart) + 2 * a->part_heads * (size_t)(a->dim + 2) * sizeof(float));
}

void attn_workspace(AttnArgs *a, void *ws)
{
    a->parts = (AttnPart *)ws;
    a->part_o = (float *)(a->parts + a->grid);
    a->part_ml = a->part_o + (size_t)a->grid * 2 * a->part_heads * a->dim;
}

hipError_t attn_launch(const AttnArgs &a, int cache_dtype, hipStream_t stream)
{
    const bool q32 = a.q_dtype == ILPM_F32;
    const hipError_t e = cache_dtype == ILPM_F32   ? attn_split_f32(a, stream)
                         : cache_dtype == ILPM_F16 ? (q32 ? attn_split_f16_q32(a, stream) : attn_split_f16(a, stream))
                                                   : (q32 ? attn_split_bf16_q32(a, stream) : attn_split_bf16(a, stream));
    if (e != hipSuccess || !a.split) return e;
    hipLaunchKernelGGL(attn_join, dim3(a.grid, a.part_heads), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ilpm
