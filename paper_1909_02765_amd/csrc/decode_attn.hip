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

// Joins the parts of the unit at place blockIdx.x, for its head blockIdx.y and
// 64 values of it, blockIdx.z: those of the workgroup that began the unit and of
// the ones after it.  Group p of the threads adds parts p, p + G, ... in their
// order, V values a thread, then the groups' sums are added in theirs.  What bounds
// it is a chain of accesses that wait for each other, so the first parts are read
// before their weights are known, and it launches little that finds no work (8
// units of 16 heads of 256 6.6 -> 4.0 us).
template <int V> __global__ __launch_bounds__(256) void attn_join(AttnArgs a)
{
    constexpr int T = 64 / V, G = 256 / T, AHEAD = 4, OWN = kMaxParts / 256;
    __shared__ float red[2][4], w[kMaxParts];
    __shared__ Pack<float, V> sum[G][T];
    const AttnPart u = a.parts[blockIdx.x];
    if (u.count == 0) return;
    const int kvh = u.unit / a.blocks, in_group = (u.unit - kvh * a.blocks) * kAttnHeads + (int)blockIdx.y;
    if (in_group >= a.group) return;
    const int head = kvh * a.group + in_group, tid = threadIdx.x;
    auto slot = [&](int i) { return ((((int64_t)u.first + i) * 2 + (i == 0)) * a.part_heads + blockIdx.y); };
    const int group = tid / T, d = (int)blockIdx.z * 64 + tid % T * V;
    auto part = [&](int i) {
        Pack<float, V> p = {};
        if (i < u.count && d < a.dim) p = load_pack<float, V>(a.part_o + slot(i) * a.dim + d);
        return p;
    };
    float m[OWN], l[OWN], top = -INFINITY, total = 0.f;
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int i = tid + k * 256;
        m[k] = i < u.count ? a.part_ml[slot(i) * 2] : -INFINITY;
        l[k] = i < u.count ? a.part_ml[slot(i) * 2 + 1] : 0.f;
    }
    Pack<float, V> ahead[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ahead[k] = part(group + k * G);
#pragma unroll
    for (int k = 0; k < OWN; ++k) top = fmaxf(top, m[k]);
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) red[0][tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const float f = __builtin_amdgcn_exp2f(m[k] - base);
        total += l[k] * f;
        if (tid + k * 256 < u.count) w[tid + k * 256] = f;
    }
    for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
    if ((tid & 63) == 0) red[1][tid >> 6] = total;
    __syncthreads();
    Pack<float, V> v = {};
    auto add = [&](const Pack<float, V> &p, int i) {
        if (i >= u.count) return;
#pragma unroll
        for (int k = 0; k < V; ++k) v.v[k] += p.v[k] * w[i];
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) add(ahead[k], group + k * G);
#pragma unroll 4
    for (int i = group + AHEAD * G; i < u.count; i += G) add(part(i), i);
    sum[group][tid % T] = v;
    __syncthreads();
    total = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int e = (int)blockIdx.z * 64 + tid;
    if (tid < 64 && e < a.dim) {
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) x += sum[g][tid / V].v[tid % V];
        store_f32(a.out, (int64_t)u.seq * a.o_row + (int64_t)head * a.o_head + e, a.q_dtype, x * inv);
    }
    if (e == 0 && a.lse) a.lse[(int64_t)u.seq * a.q_heads + head] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

}  // namespace

// Either a unit goes to a workgroup, or as many workgroups as the card holds (or
// as there are smallest shares) share all tiles.  The first takes about 5 us and
// `round` for every four tiles of the longest sequence; the second 12 us for its
// two kernels and one more for every 36 units (fitted to 64 calls of 17 to 64 tiles
// and 60 to 1425 units: 1386 units of 48 tiles, f16 heads of 80, 114 us shared and
// 66 by units; 65 such units under f32 queries 15 and 20).  Beyond 64 tiles units
// differ too much in length (207 of up to 321 tiles 56 us shared and 134 by units).
// The fit has no calls of fewer than 60 units, and those are shared beyond 16 tiles: 8
// and 32 units of bf16 heads of 128 take 9.7 and 10.0 us shared at 19 tiles (8.0 and 8.1
// by units), 9.8 and 10.7 at 29 (10.1 and 10.2), 9.8 and 11.0 at 44 (12.7 and 12.8), 8
// units of f32 ones 10.8 at 17 tiles (12.6).
size_t attn_plan(AttnArgs *a, int cache_dtype, bool q32, int max_len)
{
    a->blocks = ceil_div(a->group, kAttnHeads);
    const int64_t units = (int64_t)a->n_seqs * a->kv_heads * a->blocks;
    const int64_t keys = a->window > 0 ? std::min(max_len, a->window) : max_len, tiles = std::max<int64_t>(1, (keys + 15) / 16);
    // (Tiles are counted in 32 bits.  Where a table could name more, there are units enough without a split.)
    const int64_t most = (((int64_t)a->capacity + 15) / 16 + kUnitCost) * units;
    const double round = cache_dtype == ILPM_F32 ? 0.2 + a->dim / 55. : 0.7 + a->dim / 250. + (q32 ? 0.35 : 0.);
    const bool by_units = tiles <= kWholeTiles || (tiles <= 4 * kWholeTiles && units >= 60 && 5. + (double)tiles / 4. * round <= 12. + (double)units / 36.);
    a->split = !by_units && units > 0 && (most < INT_MAX || units == 1);
    if (!a->split) {
        a->grid = (int)units;
        return 0;
    }
    const int card = cache_dtype == ILPM_F32   ? attn_card_f32(a->dim)
                     : cache_dtype == ILPM_F16 ? (q32 ? attn_card_f16_q32(a->dim) : attn_card_f16(a->dim))
                                               : (q32 ? attn_card_bf16_q32(a->dim) : attn_card_bf16(a->dim));
    // (Shares of few tiles are better off larger: 8 key heads of 2445 x 10 f16 keys of
    // 80 15.2 us on 768 workgroups, 14.3 on 512.)
    int grid = card;
    while (grid > 2 * kAttnCus && units * tiles < 18 * (int64_t)grid) grid -= kAttnCus;
    a->grid = (int)std::min<int64_t>({grid, kMaxParts, units * ((tiles + kUnitCost + kMinShare - 1) / kMinShare)});
    a->part_heads = std::min(a->group, kAttnHeads);
    a->part_of_unit = units <= a->grid;
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
    const dim3 grid(a.part_of_unit ? a.n_seqs * a.kv_heads * a.blocks : a.grid, a.part_heads, ceil_div(a.dim, 64));
    if (a.dim % 4) hipLaunchKernelGGL((attn_join<1>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((attn_join<4>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ilpm
