// kv_append_norm: new tokens' keys and values into the paged cache at slots of
// their own, keys and queries normed for each head and rotated by their
// positions on the way.
//
// A head h becomes rotated((h - mean) / sqrt(var + eps) w): its sums need all of
// it, a rotation two values at a time, so a head lies in the registers of
// neighbouring lanes of one wave, in the packs that the rotation takes.  All of a
// head is read before any of it is written, by one wave, which lets queries be
// normed in place.
#include "draft.h"

namespace ilpm {
namespace {

// Where a token goes: its page and slot, -1 where it is not written.
struct Place {
    int page, slot;
};

__device__ inline Place place_of(const AppendNormArgs &n, int t, const Divisor &by_page)
{
    const AppendArgs &a = n.a;
    Place p = {-1, 0};
    const int seq = a.seq_ids[t], slot = n.slots[t];
    if (seq < 0 || seq >= a.n_seqs || slot < 0) return p;
    const int at = by_page.of(slot);
    if (at >= a.max_pages) return p;
    const int page = a.table[(int64_t)seq * a.table_stride + at];
    if (page < 0 || page >= a.n_pages) return p;
    p.page = page;
    p.slot = slot - at * a.page_size;
    return p;
}

template <typename TP> __device__ inline float weight(const void *w, int i) { return w ? (float)((const TP *)w)[i] : 1.f; }

__device__ inline float sum_lanes(float v, int lanes)
{
    for (int d = 1; d < lanes; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

constexpr int kMostDim = 1024;

// Any sizes: a wave per head of a token, which lies in LDS between its norm and
// its rotation.
template <typename TX, typename TC, typename TP> __global__ __launch_bounds__(256) void append_norm_any(AppendNormArgs n, Divisor by_heads, Divisor by_page, int total)
{
    __shared__ float rows[4][kMostDim];
    const AppendArgs &a = n.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int id = (int)blockIdx.x * 4 + wave;
    if (id >= total) return;
    float *row = rows[wave];
    const int heads = a.q_heads + 2 * a.kv_heads, t = by_heads.of(id), i = id - t * heads;
    const bool query = i < a.q_heads, value = i >= a.q_heads + a.kv_heads;
    const int h = query ? i : value ? i - a.q_heads - a.kv_heads : i - a.q_heads;
    const int pos = a.positions[t], half = a.rot_dim / 2;
    const bool turn = !value && a.rot_dim > 0 && pos >= 0 && pos < a.n_positions;
    Place at = {-1, 0};
    if (!query) {
        at = place_of(n, t, by_page);
        if (at.page < 0 || (a.rot_dim > 0 && !(pos >= 0 && pos < a.n_positions))) return;
    }
    const TX *src = query ? (const TX *)a.q + (int64_t)t * a.q_row + h * a.q_head
                  : value ? (const TX *)a.v + (int64_t)t * a.v_row + h * a.v_head : (const TX *)a.k + (int64_t)t * a.k_row + h * a.k_head;
    float sum = 0.f;
    for (int e = lane; e < a.dim; e += 64) {
        row[e] = (float)src[e];
        sum += row[e];
    }
    if (!value && n.norm != ILPM_NORM_NONE) {
        const float inv = 1.f / (float)a.dim, mean = n.norm == ILPM_NORM_LAYER ? sum_lanes(sum, 64) * inv : 0.f;
        float var = 0.f;
        for (int e = lane; e < a.dim; e += 64) var += (row[e] - mean) * (row[e] - mean);
        const float rstd = 1.f / sqrtf(sum_lanes(var, 64) * inv + n.eps);
        const void *w = query ? n.q_w : n.k_w;
        for (int e = lane; e < a.dim; e += 64) row[e] = (row[e] - mean) * rstd * weight<TP>(w, e);
    }
    // (Only this wave touches its row, and a wave's LDS accesses keep their order.)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    auto put = [&](auto *dst) {
        using TD = std::remove_reference_t<decltype(*dst)>;
        for (int e = lane; e < a.dim; e += 64) {
            float x = row[e];
            if (turn && e < a.rot_dim) {
                const int u = a.pairs ? e / 2 : e < half ? e : e - half;
                const bool second = a.pairs ? (e & 1) != 0 : e >= half;
                const float other = row[a.pairs ? e ^ 1 : second ? e - half : e + half];
                const float c = a.cos[(int64_t)pos * half + u], s = a.sin[(int64_t)pos * half + u];
                x = second ? x * c + other * s : x * c - other * s;
            }
            dst[e] = (TD)x;
        }
    };
    if (query) put((TX *)a.q_out + (int64_t)t * a.qo_row + h * a.qo_head);
    else if (value) put((TC *)a.vc + (int64_t)at.page * a.vc_page + (int64_t)at.slot * a.vc_slot + h * a.vc_head);
    else put((TC *)a.kc + (int64_t)at.page * a.kc_page + (int64_t)at.slot * a.kc_slot + h * a.kc_head);
}

template <typename TX, typename TC, typename TP> hipError_t launch(const AppendNormArgs &n, hipStream_t stream)
{
    const AppendArgs &a = n.a;
    const int heads = a.q_heads + 2 * a.kv_heads, total = heads * a.n_tokens;
    hipLaunchKernelGGL((append_norm_any<TX, TC, TP>), dim3(ceil_div(total, 4)), dim3(256), 0, stream, n, Divisor((unsigned)heads),
                       Divisor((unsigned)a.page_size), total);
    return hipGetLastError();
}

}  // namespace

hipError_t append_norm_launch(const AppendNormArgs &n, int x_dtype, int cache_dtype, int param_dtype, hipStream_t stream)
{
    if (x_dtype == ILPM_F32) {
        if (cache_dtype == ILPM_F32) return launch<float, float, float>(n, stream);
        if (cache_dtype == ILPM_F16) return launch<float, _Float16, float>(n, stream);
        return launch<float, __bf16, float>(n, stream);
    }
    if (x_dtype == ILPM_F16) {
        if (param_dtype == ILPM_F32) return launch<_Float16, _Float16, float>(n, stream);
        return launch<_Float16, _Float16, _Float16>(n, stream);
    }
    if (param_dtype == ILPM_F32) return launch<__bf16, __bf16, float>(n, stream);
    return launch<__bf16, __bf16, __bf16>(n, stream);
}

}  // namespace ilpm
