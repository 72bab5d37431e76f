// residual_norm: r = x + scale * gate * post(y), z = pre(r), a row per token.
#include "decode.h"

#include <algorithm>

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
// again for each sum it needs (very wide rows, and those of less than a pack).
// Each element is written by the thread that reads it, in the last pass, so r may
// be x and z may be y.
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

// Lane permutations within rows of 16, in the vector unit.
template <int CTRL> __device__ inline float plus_permuted(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// The sum over groups of LANES (16 or 64) lanes.
template <int LANES> __device__ inline float lanes_sum(float v)
{
    v = plus_permuted<0xB1>(v);   // lanes 1 0 3 2 of each four
    v = plus_permuted<0x4E>(v);   // lanes 2 3 0 1 of each four
    v = plus_permuted<0x141>(v);  // the other four of eight
    v = plus_permuted<0x140>(v);  // the other eight of sixteen
    if constexpr (LANES == 64) {
        unsigned x = __builtin_bit_cast(unsigned, v);
        const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        const unsigned p0 = p[0], p1 = p[1];
        x = __builtin_bit_cast(unsigned, __builtin_bit_cast(float, p0) + __builtin_bit_cast(float, p1));
        const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const unsigned q0 = q[0], q1 = q[1];
        v = __builtin_bit_cast(float, q0) + __builtin_bit_cast(float, q1);
    }
    return v;
}

// Rows of up to T * E values: T threads hold a row in registers, E values each,
// in packs of VEC, so each input is read once and each output written once.  T
// is 16 or 64, part of a wave or a wave (no barrier), or 1024: of these a
// workgroup has as many waves as the row fills.  Weights and biases stay in
// registers over the rows that a workgroup takes, and a row is read while the one
// before it is worked on (7512 f32 rows of 2247 59 -> 47 us).
//
// LOOSE: rows of any alignment and of any width from VEC on.  The last pack then
// ends with the row, over some values of the pack before it: these count in no
// sum, and only the pack that they belong to stores them (the row may be
// overwritten in place).
//
// Mean and variance come from the values in registers, in two steps, so a mean
// far from zero costs the variance nothing.  What bounds it: the bytes of x, y,
// gate, r and z (16381 rows of 4096, f32 over bf16: 190 us, 5.7 TB/s).  Of 16-bit
// rows of several thousand values that are no whole packs it is the work on them and
// the sums that wait for each other, which one row a compute unit does not hide (6556
// bf16 rows of 6723, rms norms: 97 us, 3.6 TB/s; the vector unit issues in 43% of the
// cycles, and waves wait for 68% of theirs).
template <typename TX, typename TY, typename TP, int T, int E, int VEC, bool LOOSE>
__global__ __launch_bounds__(T <= 64 ? 256 : T) void norm_rows(NormArgs a)
{
    constexpr int NV = E / VEC, ROWS = T <= 64 ? 256 / T : 1, WAVES = T > 64 ? T / 64 : 1;
    const int threads = T <= 64 ? T : (int)blockDim.x;  // of a row
    // Beyond, neither weights nor a second row fit beside the row: read for each, when it comes.
    constexpr bool HOLD = T * E <= 8192;
    __shared__ float lds[WAVES > 1 ? 2 * WAVES : 1];
    const int tid = T <= 64 ? threadIdx.x % T : threadIdx.x;
    const float inv_n = 1.f / (float)a.width;
    int turn = 0;
    auto total = [&](float v) {
        v = lanes_sum<(T < 64 ? T : 64)>(v);
        if constexpr (WAVES > 1) {
            // Two sets of places in turn: what is written now was read before the last barrier.
            float *part = lds + turn * WAVES;
            turn ^= 1;
            if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
            __syncthreads();
            const int wave = threadIdx.x % WAVES;
            v = lanes_sum<WAVES>(wave * 64 < threads ? part[wave] : 0.f);
        }
        return v;
    };
    // Pack i of this thread begins at `at`; its first `skip` values are another's.
    auto at = [&](int i) { return (tid + i * threads) * VEC; };
    auto skip = [&](int i) { return LOOSE ? max(0, at(i) + VEC - a.width) : 0; };
    auto get = [&](const auto *row, int i) {
        using TD = std::remove_cv_t<std::remove_reference_t<decltype(*row)>>;
        Pack<TD, VEC> p = {};
        if (row && at(i) < a.width) {
            if constexpr (LOOSE) p = load_loose<TD, VEC>(row + at(i) - skip(i));
            else p = load_pack<TD, VEC>(row + at(i));
        }
        return p;
    };
    auto put = [&](auto *row, int i, const float (&v)[VEC]) {
        using TD = std::remove_reference_t<decltype(*row)>;
        if (at(i) >= a.width) return;
        Pack<TD, VEC> p;
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.v[j] = (TD)v[j];
        if constexpr (!LOOSE) {
            store_pack<TD, VEC>(row + at(i), p);
        } else if (skip(i) == 0) {
            store_loose<TD, VEC>(row + at(i), p);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (j >= skip(i)) row[at(i) - skip(i) + j] = p.v[j];
        }
    };
    auto live = [&](int i, int j) { return at(i) < a.width && (!LOOSE || j >= skip(i)); };

    // Of most waves all values count.
    const bool full = __all(at(NV - 1) + VEC <= a.width);
    Pack<TP, VEC> post_w[NV], post_b[NV], pre_w[NV], pre_b[NV];
#pragma unroll
    for (int i = 0; HOLD && i < NV; ++i) {
        post_w[i] = get((const TP *)a.post_w, i);
        post_b[i] = get((const TP *)a.post_b, i);
        pre_w[i] = get((const TP *)a.pre_w, i);
        pre_b[i] = get((const TP *)a.pre_b, i);
    }
    // (v - mean) / sqrt(variance + eps) * w + b of the values in v.
    auto normed = [&](float (&v)[NV][VEC], int kind, const void *w, const void *b, const auto &wh, const auto &bh) {
        // The sum of term(v) over the row.
        auto sum = [&](auto term) {
            float s = 0.f;
            if (full) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s += term(v[i][j]);
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float t = term(v[i][j]);
                        s += live(i, j) ? t : 0.f;
                    }
            }
            return total(s);
        };
        if (kind == ILPM_NORM_LAYER) {
            const float mean = sum([](float x) { return x; }) * inv_n;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] -= mean;
        }
        const float rstd = rsqrtf(sum([](float x) { return x * x; }) * inv_n + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Pack<TP, VEC> wp = HOLD ? wh[i] : get((const TP *)w, i), bp = HOLD ? bh[i] : get((const TP *)b, i);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] *= rstd;
                if (w) v[i][j] *= (float)wp.v[j];
                if (b) v[i][j] += (float)bp.v[j];
            }
        }
    };

    struct Row {
        Pack<TX, VEC> x[NV];
        Pack<TY, VEC> y[NV];
        Pack<TP, VEC> gate[NV];
    };
    const int64_t step = (int64_t)gridDim.x * ROWS;
    auto load = [&](Row &t, int64_t row) {
        const TP *grow = a.gate ? (const TP *)a.gate + row * a.gate_row : nullptr;
#pragma unroll
        for (int i = 0; i < NV; ++i) t.y[i] = get(a.y ? (const TY *)a.y + row * a.y_row : (const TY *)nullptr, i);
#pragma unroll
        for (int i = 0; i < NV; ++i) t.x[i] = get((const TX *)a.x + row * a.x_row, i);
#pragma unroll
        for (int i = 0; i < NV; ++i) t.gate[i] = get(grow, i);
    };
    Row next;
    int64_t row = (int64_t)blockIdx.x * ROWS + (T < 64 ? (int)threadIdx.x / T : T == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / T) : 0);
    if (HOLD && row < a.rows) load(next, row);
    for (; row < a.rows; row += step) {
        float v[NV][VEC], u[NV][VEC];
        if (!HOLD) load(next, row);
        const Row t = next;
        const auto &x = t.x;
        const auto &y = t.y;
        const auto &gate = t.gate;
        if (HOLD && row + step < a.rows) load(next, row + step);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = (float)x[i].v[j];
        if (a.y) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) u[i][j] = (float)y[i].v[j];
            if (a.post != ILPM_NORM_NONE) normed(u, a.post, a.post_w, a.post_b, post_w, post_b);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (a.gate) u[i][j] *= (float)gate[i].v[j];
                    v[i][j] += a.scale * u[i][j];
                }
        }
        if (a.r) {
#pragma unroll
            for (int i = 0; i < NV; ++i) put((TX *)a.r + row * a.r_row, i, v[i]);
        }
        if (a.z) {
            normed(v, a.pre, a.pre_w, a.pre_b, pre_w, pre_b);
#pragma unroll
            for (int i = 0; i < NV; ++i) put((TY *)a.z + row * a.z_row, i, v[i]);
        }
    }
}

// As many workgroups as the 256 compute units hold at once, with the same number
// of rows each, give or take one: more would read the weights again (9116 f32 rows
// of 1015 23.0 -> 22.2 us).  By their registers that is 16 waves a unit, of 16-bit
// rows in workgroups of up to four waves 20 (3822 bf16 rows of 1732 14.1 -> 13.2
// us).  Of f32 rows more of them at once than the next power of two would hold
// are slower (8000 f32 rows of 2052 over bf16: two workgroups of five waves a unit
// 57 us, three 65; bf16 rows 55 and 42).  Rows of 3584 to 4096 values, which are
// seven and eight waves, otherwise go two workgroups a unit; where more bytes than the
// 256 MB cache before the memory holds are moved, one is faster (us with two and one:
// 16000 f32 rows of 3584 over bf16 with f32 gates by rows 175 and 161, of 4096 203 and
// 190; 8000 of 3584 over bf16 alone, 344 MB, 63 and 61; 16000 bf16 rows of 3584 90 and
// 90, of 4096 100 and 93, but 8000 of 4096, 262 MB, 42 and 48; 14016 f16 ones of 3651,
// which are LOOSE, 92 and 97).  Narrower rows of two workgroups a unit are left as they
// are: there it goes by the types (16000 rows of 2568: f32 over bf16 125 and 116, bf16
// 69 and 86).
constexpr int64_t kBeyondCache = 320000000;

template <typename TX, typename TY, typename TP, int T, int E, int VEC, bool LOOSE>
void launch_rows(const NormArgs &a, hipStream_t stream)
{
    constexpr int per = T <= 64 ? 256 / T : 1;
    const int block = T <= 64 ? 256 : ceil_div(a.width, E * 64) * 64, waves = block / 64;
    const int64_t bytes = (int64_t)a.rows * a.width *
                          (sizeof(TX) * (1 + !!a.r) + sizeof(TY) * (!!a.y + !!a.z) + sizeof(TP) * (a.gate && a.gate_row > 0));
    const bool alone = !LOOSE && a.width >= 3584 && a.width <= 4096 && bytes > kBeyondCache;
    const int full = waves <= 1 ? 1 : waves <= 2 ? 2 : waves <= 4 ? 4 : waves <= 8 ? 8 : 16;
    const int per_cu = alone ? 1 : sizeof(TX) == 2 ? (waves <= 4 ? 20 : 16) / waves : 16 / full;
    const int rows = ceil_div(a.rows, per), turns = ceil_div(rows, 256 * per_cu);
    const int groups = ceil_div(rows, turns);
    hipLaunchKernelGGL((norm_rows<TX, TY, TP, T, E, VEC, LOOSE>), dim3(groups), dim3(block), 0, stream, a);
}

// By the width: 8 values a thread.  With 16 too few waves fit a compute unit to cover
// each other's waits (13447 bf16 rows of 675 28.8 -> 23.6 us with two waves for
// one, 14016 f16 rows of 3651 135 -> 92 with eight for four); rows beyond 8192 have
// no more threads to go to.
template <typename TX, typename TY, typename TP, int VEC, bool LOOSE> bool launch_width(const NormArgs &a, hipStream_t stream)
{
    if (a.width < VEC) return false;
    if (a.width <= 128) launch_rows<TX, TY, TP, 16, 8, VEC, LOOSE>(a, stream);
    else if (a.width <= 512) launch_rows<TX, TY, TP, 64, 8, VEC, LOOSE>(a, stream);
    else if (a.width <= 8192) launch_rows<TX, TY, TP, 1024, 8, VEC, LOOSE>(a, stream);
    else if (!LOOSE && a.width <= 16384) launch_rows<TX, TY, TP, 1024, 16, VEC, false>(a, stream);
    else return false;
    return true;
}

template <typename TX, typename TY, typename TP> hipError_t launch(const NormArgs &a, hipStream_t stream)
{
    constexpr int VEC = 16 / (int)sizeof(TY);
    auto fits = [&](const void *p, int64_t stride, int size) {
        return (uintptr_t)p % std::min(16, VEC * size) == 0 && stride % VEC == 0;
    };
    const int sx = sizeof(TX), sy = sizeof(TY), sp = sizeof(TP);
    const bool packs = a.width % VEC == 0 && fits(a.x, a.x_row, sx) && fits(a.r, a.r_row, sx) && fits(a.y, a.y_row, sy) &&
                       fits(a.z, a.z_row, sy) && fits(a.gate, a.gate_row, sp) && fits(a.post_w, 0, sp) &&
                       fits(a.post_b, 0, sp) && fits(a.pre_w, 0, sp) && fits(a.pre_b, 0, sp);
    if (!(packs ? launch_width<TX, TY, TP, VEC, false>(a, stream) : launch_width<TX, TY, TP, VEC, true>(a, stream)))
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
