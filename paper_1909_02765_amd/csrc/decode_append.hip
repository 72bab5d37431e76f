// kv_append: new tokens' keys and values into the paged cache, keys and
// queries rotated by their positions on the way.
//
// A rotation turns the pair (a, b) of a head by the angle of its position,
//   a' = a c - b s,  b' = b c + a s,
// so whoever writes one of the two needs both: a thread takes whole pairs, and
// reads them before it writes, which is also what lets the queries be rotated
// in place.
#include "decode.h"

namespace ilpm {
namespace {

// Where a token goes: its page and slot, -1 where it is not written.
struct Place {
    int page, slot;
};

__device__ inline Place place_of(const AppendArgs &a, int t, int pos)
{
    Place p = {-1, 0};
    const int seq = a.seq_ids[t];
    if (seq < 0 || seq >= a.n_seqs || pos < 0) return p;
    const int at = pos / a.page_size;
    if (at >= a.max_pages) return p;
    const int page = a.table[(int64_t)seq * a.table_stride + at];
    if (page < 0 || page >= a.n_pages) return p;
    p.page = page;
    p.slot = pos - at * a.page_size;
    return p;
}

// Any sizes, strides and alignment: a workgroup per token, an element or a
// pair of them per thread and step.
template <typename TX, typename TC> __global__ __launch_bounds__(256) void append_any(AppendArgs a)
{
    const int t = blockIdx.x;
    const int pos = a.positions[t];
    const bool turn = a.rot_dim > 0 && pos >= 0 && pos < a.n_positions;
    Place at = place_of(a, t, pos);
    if (a.rot_dim > 0 && !turn) at.page = -1;
    const int half = a.rot_dim / 2, units = a.dim - half;  // of a rotated head: pairs, then single elements
    const float *cos = a.cos + (turn ? (int64_t)pos * half : 0), *sin = a.sin + (turn ? (int64_t)pos * half : 0);

    auto rotate = [&](const auto *src, auto *dst, int u) {
        using TD = std::remove_reference_t<decltype(*dst)>;
        if (u >= half) {
            dst[u + half] = (TD)(float)src[u + half];
            return;
        }
        const int i = a.pairs ? 2 * u : u, j = a.pairs ? 2 * u + 1 : u + half;
        const float x = (float)src[i], y = (float)src[j];
        const float c = turn ? cos[u] : 1.f, s = turn ? sin[u] : 0.f;
        dst[i] = (TD)(turn ? x * c - y * s : x);
        dst[j] = (TD)(turn ? y * c + x * s : y);
    };

    if (a.q) {
        const TX *q = (const TX *)a.q + (int64_t)t * a.q_row;
        TX *o = (TX *)a.q_out + (int64_t)t * a.qo_row;
        for (int i = threadIdx.x; i < a.q_heads * units; i += 256) {
            const int h = i / units;
            rotate(q + h * a.q_head, o + h * a.qo_head, i - h * units);
        }
    }
    if (at.page < 0) return;
    const TX *k = (const TX *)a.k + (int64_t)t * a.k_row, *v = (const TX *)a.v + (int64_t)t * a.v_row;
    TC *kc = (TC *)a.kc + (int64_t)at.page * a.kc_page + (int64_t)at.slot * a.kc_slot;
    TC *vc = (TC *)a.vc + (int64_t)at.page * a.vc_page + (int64_t)at.slot * a.vc_slot;
    for (int i = threadIdx.x; i < a.kv_heads * units; i += 256) {
        const int h = i / units;
        rotate(k + h * a.k_head, kc + h * a.kc_head, i - h * units);
    }
    for (int i = threadIdx.x; i < a.kv_heads * a.dim; i += 256) {
        const int h = i / a.dim, e = i - h * a.dim;
        vc[h * a.vc_head + e] = (TC)(float)v[h * a.v_head + e];
    }
}

template <typename TX, typename TC> hipError_t launch(const AppendArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((append_any<TX, TC>), dim3(a.n_tokens), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t append_launch(const AppendArgs &a, int x_dtype, int cache_dtype, hipStream_t stream)
{
    if (x_dtype == ILPM_F32) {
        if (cache_dtype == ILPM_F32) return launch<float, float>(a, stream);
        if (cache_dtype == ILPM_F16) return launch<float, _Float16>(a, stream);
        return launch<float, __bf16>(a, stream);
    }
    if (x_dtype == ILPM_F16) return launch<_Float16, _Float16>(a, stream);
    return launch<__bf16, __bf16>(a, stream);
}

}  // namespace ilpm
