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
// thread takes one pack, or one of each half, of up to HPT heads of a token, so
// it reads the angles once for all of them.  What bounds it: the bytes of
// queries, keys and values, read and written once.
template <typename TX, typename TC, int VEC, int HPT> __global__ __launch_bounds__(256) void append_packs(AppendArgs a)
{
    const int half = a.rot_dim / 2;
    // Packs of a rotated head (the first `turned` of them with their partners, or
    // in pairs of neighbours), and of a value head.
    const int turned = (a.pairs ? a.rot_dim : half) / VEC, units = a.dim / VEC - (a.pairs ? 0 : half / VEC);
    const int vunits = a.dim / VEC;
    const int heads = a.q_heads + a.kv_heads, slots = (heads + HPT - 1) / HPT, vslots = (a.kv_heads + HPT - 1) / HPT;
    const unsigned per = slots * units + vslots * vunits;
    const unsigned id = blockIdx.x * 256u + threadIdx.x;  // (at most 2^24 workgroups)
    const int t = (int)(id / per);
    if (t >= a.n_tokens) return;
    int i = (int)(id - t * per);
    const int pos = a.positions[t];

    if (i >= slots * units) {  // a value's packs
        i -= slots * units;
        const int slot = i / vunits, e = (i - slot * vunits) * VEC;
        const TX *v = (const TX *)a.v + (int64_t)t * a.v_row + e;
        Pack<TX, VEC> p[HPT];
#pragma unroll
        for (int n = 0; n < HPT; ++n) {
            const int h = slot + n * vslots;
            if (h < a.kv_heads) p[n] = *reinterpret_cast<const Pack<TX, VEC> *>(v + h * a.v_head);
        }
        Place at = place_of(a, t, pos);
        if (at.page < 0 || (a.rot_dim > 0 && pos >= a.n_positions)) return;
        TC *vc = (TC *)a.vc + (int64_t)at.page * a.vc_page + (int64_t)at.slot * a.vc_slot + e;
#pragma unroll
        for (int n = 0; n < HPT; ++n) {
            const int h = slot + n * vslots;
            Pack<TC, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) o.v[j] = (TC)(float)p[n].v[j];
            if (h < a.kv_heads) *reinterpret_cast<Pack<TC, VEC> *>(vc + h * a.vc_head) = o;
        }
        return;
    }

    const int slot = i / units, u = i - slot * units;
    const bool rotated = u < turned;
    // Elements e.. and, of halves, their partners from e2.
    const int e = a.pairs || rotated ? u * VEC : half + u * VEC, e2 = e + half;
    const bool two = rotated && !a.pairs;
    Pack<TX, VEC> p[HPT], p2[HPT];
    const TX *q = (const TX *)a.q + (int64_t)t * a.q_row, *k = (const TX *)a.k + (int64_t)t * a.k_row;
#pragma unroll
    for (int n = 0; n < HPT; ++n) {
        const int h = slot + n * slots;
        if (h >= heads) continue;
        const TX *src = h < a.q_heads ? q + h * a.q_head : k + (h - a.q_heads) * a.k_head;
        p[n] = *reinterpret_cast<const Pack<TX, VEC> *>(src + e);
        if (two) p2[n] = *reinterpret_cast<const Pack<TX, VEC> *>(src + e2);
    }
    const bool known = a.rot_dim > 0 && pos >= 0 && pos < a.n_positions, turn = rotated && known;
    // VEC angles for halves, VEC / 2 for pairs.
    float c[VEC], s[VEC];
    if (turn) {
        const int first = a.pairs ? e / 2 : e;
        const float *cos = a.cos + (int64_t)pos * half + first, *sin = a.sin + (int64_t)pos * half + first;
        constexpr int HV = VEC > 1 ? VEC / 2 : 1;
        const Pack<float, HV> c0 = *reinterpret_cast<const Pack<float, HV> *>(cos);
        const Pack<float, HV> s0 = *reinterpret_cast<const Pack<float, HV> *>(sin);
#pragma unroll
        for (int j = 0; j < HV; ++j) c[j] = c0.v[j], s[j] = s0.v[j];
        if (two) {
            const Pack<float, HV> c1 = *reinterpret_cast<const Pack<float, HV> *>(cos + HV);
            const Pack<float, HV> s1 = *reinterpret_cast<const Pack<float, HV> *>(sin + HV);
#pragma unroll
            for (int j = 0; j < HV; ++j) c[HV + j] = c1.v[j], s[HV + j] = s1.v[j];
        }
    }
    // (The queries of a token are turned wherever its keys go.)
    Place at = {-1, 0};
    if (slot + (HPT - 1) * slots >= a.q_heads) at = place_of(a, t, pos);
    if (a.rot_dim > 0 && !known) at.page = -1;
    TC *kc = (TC *)a.kc + (int64_t)max(at.page, 0) * a.kc_page + (int64_t)at.slot * a.kc_slot;
    TX *qo = (TX *)a.q_out + (int64_t)t * a.qo_row;
#pragma unroll
    for (int n = 0; n < HPT; ++n) {
        const int h = slot + n * slots;
        if (h >= heads) continue;
        float x[VEC], y[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = (float)p[n].v[j], y[j] = two ? (float)p2[n].v[j] : 0.f;
        if (turn && two) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float v = x[j];
                x[j] = v * c[j] - y[j] * s[j];
                y[j] = y[j] * c[j] + v * s[j];
            }
        } else if (turn) {
#pragma unroll
            for (int j = 0; j + 1 < VEC; j += 2) {
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
            *reinterpret_cast<Pack<TD, VEC> *>(dst + e) = o;
            if (!two) return;
#pragma unroll
            for (int j = 0; j < VEC; ++j) o.v[j] = (TD)y[j];
            *reinterpret_cast<Pack<TD, VEC> *>(dst + e2) = o;
        };
        if (h < a.q_heads) put(qo + h * a.qo_head);
        else if (at.page >= 0) put(kc + (h - a.q_heads) * a.kc_head);
    }
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
    const int half = a.rot_dim / 2, units = a.dim / VEC - (a.pairs ? 0 : half / VEC), vunits = a.dim / VEC;
    auto groups = [&](int hpt) {
        const int64_t per = (int64_t)ceil_div(a.q_heads + a.kv_heads, hpt) * units + (int64_t)ceil_div(a.kv_heads, hpt) * vunits;
        return (per * a.n_tokens + 255) / 256;
    };
    // One head a thread until the card is full of threads, then four.
    const bool four = groups(1) > 4096;
    if (groups(four ? 4 : 1) > (1 << 24) - 1) return false;
    if (four) hipLaunchKernelGGL((append_packs<TX, TC, VEC, 4>), dim3((unsigned)groups(4)), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((append_packs<TX, TC, VEC, 1>), dim3((unsigned)groups(1)), dim3(256), 0, stream, a);
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
