// attn_decode: how a call is split over the sequences' lengths, and the join of
// the splits (the kernel over the keys is in decode_attn.h).
#include "decode_attn.h"

#include <algorithm>

namespace ilpm {

hipError_t attn_split_f32(const AttnArgs &a, hipStream_t stream);
hipError_t attn_split_f16(const AttnArgs &a, hipStream_t stream);
hipError_t attn_split_f16_q32(const AttnArgs &a, hipStream_t stream);
hipError_t attn_split_bf16(const AttnArgs &a, hipStream_t stream);
hipError_t attn_split_bf16_q32(const AttnArgs &a, hipStream_t stream);

namespace {

constexpr int kMaxSplits = 256;

// Joins the splits of a row (a sequence's query head): thread (p, d) adds
// splits p, p + 8, ... of values 4d.. in their order, then the eight sums are
// added in theirs.
__global__ __launch_bounds__(256) void attn_join(AttnArgs a)
{
    __shared__ float w[kMaxSplits], red[4];
    __shared__ float sum[8][256];
    const int64_t row = blockIdx.x;
    const int seq = (int)(row / a.q_heads), head = (int)(row % a.q_heads), tid = threadIdx.x;
    int first, end;
    visible_range(a, seq, &first, &end);
    const int ns = splits_of(a, end - first);
    if (ns <= 1) return;
    const float *ml = a.part_ml + row * a.splits * 2;
    const float m = tid < ns ? ml[2 * tid] : -INFINITY;
    float l = tid < ns ? ml[2 * tid + 1] : 0.f;
    float top = m;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float base = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m - base);
    w[tid] = f;
    l *= f;
    for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = l;
    __syncthreads();
    l = (red[0] + red[1]) + (red[2] + red[3]);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int part = tid >> 5;
    const float *po = a.part_o + row * a.splits * a.dim;
    for (int d = tid & 31; d < a.dim; d += 32) {
        float v = 0.f;
#pragma unroll 8
        for (int i = part; i < ns; i += 8) v += po[(int64_t)i * a.dim + d] * w[i];
        sum[part][d] = v;
    }
    __syncthreads();
    for (int d = tid; d < a.dim; d += 256) {
        const float v = ((sum[0][d] + sum[1][d]) + (sum[2][d] + sum[3][d])) + ((sum[4][d] + sum[5][d]) + (sum[6][d] + sum[7][d]));
        store_f32(a.out, (int64_t)seq * a.o_row + (int64_t)head * a.o_head + d, a.q_dtype, v * inv);
    }
    if (tid == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

size_t attn_plan(AttnArgs *a, int max_len)
{
    const int64_t units = (int64_t)a->n_seqs * a->kv_heads * ceil_div(a->group, kHeads);
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
    const bool q32 = a.q_dtype == ILPM_F32;
    const hipError_t e = cache_dtype == ILPM_F32   ? attn_split_f32(a, stream)
                         : cache_dtype == ILPM_F16 ? (q32 ? attn_split_f16_q32(a, stream) : attn_split_f16(a, stream))
                                                   : (q32 ? attn_split_bf16_q32(a, stream) : attn_split_bf16(a, stream));
    if (e != hipSuccess || a.splits <= 1) return e;
    hipLaunchKernelGGL(attn_join, dim3((unsigned)((int64_t)a.n_seqs * a.q_heads)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ilpm
