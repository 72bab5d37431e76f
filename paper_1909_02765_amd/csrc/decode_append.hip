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

// Division of 0 <= n < 2^31 by d >= 1 as a product: with 2^(s-1) < d <= 2^s and
// m = floor(2^32 (2^s - d) / d) + 1, n / d = (floor(n m / 2^32) + n) >> s.
struct Divisor {
    unsigned m, s;
    explicit Divisor(unsigned d) : s(0)
    {
        while ((1ull << s) < d) ++s;
        m = (unsigned)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ int of(int n) const { return (int)((__umulhi((unsigned)n, m) + (unsigned)n) >> s); }
};

// Where a token goes: its page and slot, -1 where it is not written.
struct Place {
    int page, slot;
};

template <typename F> __device__ inline Place place_of(const AppendArgs &a, int t, int pos, F page_of)
{
    Place p = {-1, 0};
    const int seq = a.seq_ids[t];
    if (seq < 0 || seq >= a.n_seqs || pos < 0) return p;
    const int at = page_of(pos);
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
    Place at = place_of(a, t, pos, [&](int n) { return n / a.page_size; });
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

// The packs of VEC that cover n elements: where they do not divide, the last one
// ends with them, over some of the one before it.  Both then write the same
// values there (which a rotation in place would not, see packs_fit).
template <int VEC> __host__ __device__ inline int packs(int n) { return (n + VEC - 1) / VEC; }
template <int VEC> __device__ inline int pack_at(int u, int n) { return min(u * VEC, n - VEC); }

// A thread takes one pack of VEC elements of a token's head or, where halves
// turn, one of each half; packs may have any alignment.  What bounds it: the
// bytes of queries, keys and values, read and written once.  (Threads that took
// several heads, to read the angles once for them, were slower: 16381 tokens of
// 40 + 8 heads of 128 in bf16 90 us with one head a thread, 5.3 TB/s, 92 with
// two, 108 with four.)
template <typename TX, typename TC, int VEC>
__global__ __launch_bounds__(256) void append_packs(AppendArgs a, Divisor by_per, Divisor by_units, Divisor by_vunits, Divisor by_page)
{
    const int half = a.rot_dim / 2, rest = a.dim - a.rot_dim, turns = a.pairs ? a.rot_dim : half;
    // Packs of a rotated head (the first `turned` of them with their partners, or
    // in pairs of neighbours), and of a value head.
    const int turned = packs<VEC>(turns), units = turned + packs<VEC>(rest);
    const int vunits = packs<VEC>(a.dim), rotated_heads = a.q_heads + a.kv_heads;
    const int per = rotated_heads * units + a.kv_heads * vunits;
    const int id = (int)(blockIdx.x * 256u + threadIdx.x);  // (fewer than 2^23 workgroups)
    const int t = by_per.of(id);
    if (t >= a.n_tokens) return;
    const int i = id - t * per;
    auto page_of = [&](int n) { return by_page.of(n); };
    const int pos = a.positions[t];
    const bool known = a.rot_dim > 0 && pos >= 0 && pos < a.n_positions;

    if (i >= rotated_heads * units) {  // of a value
        const int j = i - rotated_heads * units, h = by_vunits.of(j), e = pack_at<VEC>(j - h * vunits, a.dim);
        const Pack<TX, VEC> p = load_loose<TX, VEC>((const TX *)a.v + (int64_t)t * a.v_row + h * a.v_head + e);
        const Place at = place_of(a, t, pos, page_of);
        if (at.page < 0 || (a.rot_dim > 0 && !known)) return;
        Pack<TC, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = (TC)(float)p.v[j];
        store_loose<TC, VEC>((TC *)a.vc + (int64_t)at.page * a.vc_page + (int64_t)at.slot * a.vc_slot + h * a.vc_head + e, o);
        return;
    }

    const int h = by_units.of(i), u = i - h * units;
    const bool rotated = u < turned, two = rotated && !a.pairs, turn = rotated && known, query = h < a.q_heads;
    // Elements e.. and, of halves, their partners from e2.
    const int e = rotated ? pack_at<VEC>(u, turns) : a.rot_dim + pack_at<VEC>(u - turned, rest), e2 = e + half;
    const TX *src = query ? (const TX *)a.q + (int64_t)t * a.q_row + h * a.q_head
                          : (const TX *)a.k + (int64_t)t * a.k_row + (h - a.q_heads) * a.k_head;
    const Pack<TX, VEC> p = load_loose<TX, VEC>(src + e);
    Pack<TX, VEC> p2 = {};
    if (two) p2 = load_loose<TX, VEC>(src + e2);
    // VEC angles for halves, VEC / 2 for pairs.
    constexpr int HV = VEC / 2;
    float c[VEC], s[VEC];
    if (turn) {
        const int64_t first = (int64_t)pos * half + (a.pairs ? e / 2 : e);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (n == 1 && !two) break;
            const Pack<float, HV> cp = load_loose<float, HV>(a.cos + first + n * HV);
            const Pack<float, HV> sp = load_loose<float, HV>(a.sin + first + n * HV);
#pragma unroll
            for (int j = 0; j < HV; ++j) c[n * HV + j] = cp.v[j], s[n * HV + j] = sp.v[j];
        }
    }
    // (The queries of a token are turned wherever its keys go.)
    Place at = {-1, 0};
    if (!query) {
        at = place_of(a, t, pos, page_of);
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
        store_loose<TD, VEC>(dst + e, o);
        if (!two) return;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = (TD)y[j];
        store_loose<TD, VEC>(dst + e2, o);
    };
    if (query) put((TX *)a.q_out + (int64_t)t * a.qo_row + h * a.qo_head);
    else put((TC *)a.kc + (int64_t)at.page * a.kc_page + (int64_t)at.slot * a.kc_slot + (h - a.q_heads) * a.kc_head);
}

// Whether everything falls into packs of VEC: what turns, what does not, and
// values have one pack at least; packs of queries that are turned in place do not
// overlap, nor do those of 32 bytes (11864 tokens of 68 f32 heads of 72 turned by
// halves of 36: 104 us in overlapping packs of eight, 88 in packs of four).
template <int VEC> bool packs_fit(const AppendArgs &a, int element)
{
    const int turns = a.pairs ? a.rot_dim : a.rot_dim / 2, rest = a.dim - a.rot_dim;
    if ((turns > 0 && turns < VEC) || (rest > 0 && rest < VEC) || a.dim < VEC) return false;
    return (VEC * element <= 16 && (!a.q || a.q != a.q_out)) || (turns % VEC == 0 && rest % VEC == 0);
}

template <typename TX, typename TC, int VEC> bool launch_packs(const AppendArgs &a, hipStream_t stream)
{
    if (!packs_fit<VEC>(a, sizeof(TX))) return false;
    const int units = packs<VEC>(a.pairs ? a.rot_dim : a.rot_dim / 2) + packs<VEC>(a.dim - a.rot_dim), vunits = packs<VEC>(a.dim);
    const int64_t per = (int64_t)(a.q_heads + a.kv_heads) * units + (int64_t)a.kv_heads * vunits;
    const int64_t groups = (per * a.n_tokens + 255) / 256;
    if (groups >= 1 << 23) return false;
    hipLaunchKernelGGL((append_packs<TX, TC, VEC>), dim3((unsigned)groups), dim3(256), 0, stream, a, Divisor((unsigned)per),
                       Divisor((unsigned)units), Divisor((unsigned)vunits), Divisor((unsigned)a.page_size));
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
