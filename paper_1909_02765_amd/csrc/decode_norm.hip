// residual_norm: r = x + scale * gate * post(y), z = pre(r), a row per token.
#include "decode.h"

namespace ilpm {
namespace {

// A sum over the workgroup's 256 threads, given to all of them.
__device__ inline float sum256(float v, float *lds)
{
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();  // what an earlier sum left has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Any width, strides and alignment: a workgroup per row, which reads the row
// again for each sum it needs.  Each element is written by the thread that
// reads it, in the last pass, so r may be x and z may be y.
template <typename TX, typename TY, typename TP> __global__ __launch_bounds__(256) void norm_any(NormArgs a)
{
    __shared__ float lds[4];
    const int64_t row = blockIdx.x;
    const TX *x = (const TX *)a.x + row * a.x_row;
    const TY *y = a.y ? (const TY *)a.y + row * a.y_row : nullptr;
    const TP *gate = a.gate ? (const TP *)a.gate + row * a.gate_row : nullptr;
    const TP *pw = (const TP *)a.post_w, *pb = (const TP *)a.post_b;
    const TP *zw = (const TP *)a.pre_w, *zb = (const TP *)a.pre_b;
    const int n = a.width;
    const float inv_n = 1.f / (float)n;

    auto each = [&](auto &&f) {
        for (int i = threadIdx.x; i < n; i += 256) f(i);
    };
    float mean = 0.f, rstd = 1.f;
    if (y && a.post != ILPM_NORM_NONE) {
        float s = 0.f;
        if (a.post == ILPM_NORM_LAYER) {
            each([&](int i) { s += (float)y[i]; });
            mean = sum256(s, lds) * inv_n;
            s = 0.f;
        }
        each([&](int i) {
            const float d = (float)y[i] - mean;
            s += d * d;
        });
        rstd = 1.f / sqrtf(sum256(s, lds) * inv_n + a.eps);
    }
    auto residual = [&](int i) {
        const float xi = (float)x[i];
        if (!y) return xi;
        float v = (float)y[i];
        if (a.post != ILPM_NORM_NONE) {
            v = (v - mean) * rstd;
            if (pw) v *= (float)pw[i];
            if (pb) v += (float)pb[i];
        }
        if (gate) v *= (float)gate[i];
        return xi + a.scale * v;
    };
    float zmean = 0.f, zrstd = 1.f;
    if (a.pre != ILPM_NORM_NONE) {
        float s = 0.f;
        if (a.pre == ILPM_NORM_LAYER) {
            each([&](int i) { s += residual(i); });
            zmean = sum256(s, lds) * inv_n;
            s = 0.f;
        }
        each([&](int i) {
            const float d = residual(i) - zmean;
            s += d * d;
        });
        zrstd = 1.f / sqrtf(sum256(s, lds) * inv_n + a.eps);
    }
    TX *r = a.r ? (TX *)a.r + row * a.r_row : nullptr;
    TY *z = a.z ? (TY *)a.z + row * a.z_row : nullptr;
    each([&](int i) {
        const float v = residual(i);
        if (r) r[i] = (TX)v;
        if (z) {
            float u = (v - zmean) * zrstd;
            if (zw) u *= (float)zw[i];
            if (zb) u += (float)zb[i];
            z[i] = (TY)u;
        }
    });
}

template <typename TX, typename TY, typename TP> hipError_t launch(const NormArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_any<TX, TY, TP>), dim3(a.rows), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <typename TY> hipError_t launch_y(const NormArgs &a, bool x32, bool p32, hipStream_t stream)
{
    if (x32) return p32 ? launch<float, TY, float>(a, stream) : launch<float, TY, TY>(a, stream);
    return p32 ? launch<TY, TY, float>(a, stream) : launch<TY, TY, TY>(a, stream);
}

}  // namespace

hipError_t norm_launch(const NormArgs &a, int x_dtype, int y_dtype, int param_dtype, hipStream_t stream)
{
    const bool x32 = x_dtype == ILPM_F32, p32 = param_dtype == ILPM_F32;
    if (y_dtype == ILPM_F32) return launch<float, float, float>(a, stream);
    if (y_dtype == ILPM_F16) return launch_y<_Float16>(a, x32, p32, stream);
    return launch_y<__bf16>(a, x32, p32, stream);
}

}  // namespace ilpm
