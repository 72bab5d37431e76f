// kv_append: new tokens' keys and values into the paged cache, keys and
// queries rotated by their positions on the way.
//
// A rotation turns the pair (a, b) of a head by the angle of its position,
//   a' = a c - b s,  b' = b c + a s,
// so whoever writes one of the two needs both: a thread takes whole pairs, and
// reads them before it writes, which is also what lets the queries be rotated
// in place.
#include "decode.h"

#include <algorithm>

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

// Rows that divide into packs of VEC elements (of pairs: both halves do): a
// thread takes one pack of a token's head, or one of each half.  What bounds
// it: the bytes of queries, keys and values, read and written once.  (Threads
// that took several heads, to read the angles once for them, were slower: 16381
// tokens of 40 + 8 heads of 128 in bf16 90 us with one head a thread, 5.3 TB/s,
// 92 with two, 108 with four.)
template <typename TX, typename TC, int VEC> __global__ __launch_bounds__(256) void append_packs(AppendArgs a)
{
    const int half = a.rot_dim / 2;
    // Packs of a rotated head (the first `turned` of them with their partners, or
    // in pairs of neighbours), and of a value head.
    const int turned = (a.pairs ? a.rot_dim : half) / VEC, units = a.dim / VEC - (a.pairs ? 0 : half / VEC);
    const int vunits = a.dim / VEC, rotated_heads = a.q_heads + a.kv_heads;
    const unsigned per = rotated_heads * units + a.kv_heads * vunits;
    const unsigned id = blockIdx.x * 256u + threadIdx.x;  // (at most 2^24 workgroups)
    const int t = (int)(id / per);
    if (t >= a.n_tokens) return;
    const int i = (int)(id - t * per);
    const int pos = a.positions[t];
    const bool known = a.rot_dim > 0 && pos >= 0 && pos < a.n_positions;

    if (i >= rotated_heads * units) {  // of a value
        const int j = i - rotated_heads * units, h = j / vunits, e = (j - h * vunits) * VEC;
        const Pack<TX, VEC> p = load_pack<TX, VEC>((const TX *)a.v + (int64_t)t * a.v_row + h * a.v_head + e);
        const Place at = place_of(a, t, pos);
        if (at.page < 0 || (a.rot_dim > 0 && !known)) return;
        Pack<TC, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = (TC)(float)p.v[j];
        store_pack<TC, VEC>((TC *)a.vc + (int64_t)at.page * a.vc_page + (int64_t)at.slot * a.vc_slot + h * a.vc_head + e, o);
        return;
    }

    const int h = i / units, u = i - h * units;
    const bool rotated = u < turned, two = rotated && !a.pairs, turn = rotated && known, query = h < a.q_heads;
    // Elements e.. and, of halves, their partners from e2.
    const int e = a.pairs || rotated ? u * VEC : half + u * VEC, e2 = e + half;
    const TX *src = query ? (const TX *)a.q + (int64_t)t * a.q_row + h * a.q_head
                          : (const TX *)a.k + (int64_t)t * a.k_row + (h - a.q_heads) * a.k_head;
    const Pack<TX, VEC> p = load_pack<TX, VEC>(src + e);
    Pack<TX, VEC> p2 = {};
    if (two) p2 = load_pack<TX, VEC>(src + e2);
    // VEC angles for halves, VEC / 2 for pairs.
    constexpr int HV = VEC / 2;
    float c[VEC], s[VEC];
    if (turn) {
        const int64_t first = (int64_t)pos * half + (a.pairs ? e / 2 : e);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (n == 1 && !two) break;
            const Pack<float, HV> cp = load_pack<float, HV>(a.cos + first + n * HV);
            const Pack<float, HV> sp = load_pack<float, HV>(a.sin + first + n * HV);
#pragma unroll
            for (int j = 0; j < HV; ++j) c[n * HV + j] = cp.v[j], s[n * HV + j] = sp.v[j];
        }
    }
    // (The queries of a token are turned wherever its keys go.)
    Place at = {-1, 0};
    if (!query) {
        at = place_of(a, t, pos);
        if (at.page < 0 || (a.rot_dim > 0 && !known)) return;
    }
    float x[VEC], y[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = (float)p.v[j], y[j] = (float)p2.v[j];
    if (turn && two) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float v = x[j];
            x[j] = v * c[j] - y[j] * s[j];
            y[j] = y[j] * c[j] + v * s[j];
        }
    } else if (turn) {
#pragma unroll
        for (int j = 0; j < VEC; j += 2) {
            const float v = x[j], w = x[j + 1];
            x[j] = v * c[j / 2] - w * s[j / 2];
            x[j + 1] = w * c[j / 2] + v * s[j / 2];
        }
    }
    auto put = [&](auto *dst) {
        using TD = std::remove_reference_t<decltype(*dst)>;
        Pack<TD, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = (TD)x[j];
        store_pack<TD, VEC>(dst + e, o);
        if (!two) return;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = (TD)y[j];
        store_pack<TD, VEC>(dst + e2, o);
    };
    if (query) put((TX *)a.q_out + (int64_t)t * a.qo_row + h * a.qo_head);
    else put((TC *)a.kc + (int64_t)at.page * a.kc_page + (int64_t)at.slot * a.kc_slot + (h - a.q_heads) * a.kc_head);
}

// Whether everything divides into packs of `vec` elements, aligned to 16
// bytes or the pack's size.
bool packs_fit(const AppendArgs &a, int vec, int sx, int sc)
{
    auto at = [&](const void *p, int size) { return (uintptr_t)p % std::min(16, vec * size) == 0; };
    const int half = a.rot_dim / 2;
    if (a.dim % vec || (a.pairs ? a.rot_dim : half) % vec) return false;
    // (Half of a pack of angles is the unit in which they are read.)
    if (a.rot_dim > 0 && (half % (vec / 2) || !((uintptr_t)a.cos % std::min(16, vec / 2 * 4) == 0 && (uintptr_t)a.sin % std::min(16, vec / 2 * 4) == 0)))
        return false;
    for (int64_t s : {a.k_row, a.k_head, a.v_row, a.v_head, a.q_row, a.q_head, a.qo_row, a.qo_head, a.kc_page, a.kc_slot, a.kc_head,
                      a.vc_page, a.vc_slot, a.vc_head})
        if (s % vec) return false;
    return at(a.k, sx) && at(a.v, sx) && at(a.q, sx) && at(a.q_out, sx) && at(a.kc, sc) && at(a.vc, sc);
}

template <typename TX, typename TC, int VEC> bool launch_packs(const AppendArgs &a, hipStream_t stream)
{
    if (!packs_fit(a, VEC, sizeof(TX), sizeof(TC))) return false;
    const int units = a.dim / VEC - (a.pairs ? 0 : a.rot_dim / 2 / VEC);
    const int64_t per = (int64_t)(a.q_heads + a.kv_heads) * units + (int64_t)a.kv_heads * (a.dim / VEC);
    const int64_t groups = (per * a.n_tokens + 255) / 256;
    if (groups > (1 << 24) - 1) return false;
    hipLaunchKernelGGL((append_packs<TX, TC, VEC>), dim3((unsigned)groups), dim3(256), 0, stream, a);
    return true;
}

template <typename TX, typename TC> hipError_t launch(const AppendArgs &a, hipStream_t stream)
{
    if (!launch_packs<TX, TC, 8>(a, stream) && !launch_packs<TX, TC, 4>(a, stream) && !launch_packs<TX, TC, 2>(a, stream))
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
