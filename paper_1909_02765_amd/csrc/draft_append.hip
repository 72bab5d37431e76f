// kv_append_norm: new tokens' keys and values into the paged cache at slots of
// their own, keys and queries normed for each head and rotated by their
// positions on the way.
//
// A head h becomes rotated((h - mean) / sqrt(var + eps) w): its sums need all of
// it, a rotation two values at a time, so a head lies in the registers of
// neighbouring lanes of one wave, in the packs that the rotation takes.  All of a
// head is read before any of it is written, by one wave, which lets queries be
// normed in place.
#include <algorithm>

#include "draft.h"

namespace ilpm {
namespace {

// Where a token goes: its page and slot, -1 where it is not written.
struct Place {
    int page, slot;
};

__device__ inline Place place_of(const AppendArgs &a, int seq, int slot, const Divisor &by_page)
{
    Place p = {-1, 0};
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

// Sums over 2^log neighbouring lanes, in the vector unit.  (Once the lanes of a
// four or eight hold the same, a mirror is as good a partner as any.)
template <int CTRL> __device__ inline float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ inline float sum_lanes(float v, int log)
{
    if (log > 0) v += dpp<0xb1>(v);   // of pairs
    if (log > 1) v += dpp<0x4e>(v);   // of fours
    if (log > 2) v += dpp<0x141>(v);  // eight mirrored
    if (log > 3) v += dpp<0x140>(v);  // sixteen mirrored
    if (log > 4) {
        const unsigned x = __builtin_bit_cast(unsigned, v);
        const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        const unsigned a0 = a[0], a1 = a[1];
        v = __builtin_bit_cast(float, a0) + __builtin_bit_cast(float, a1);
    }
    if (log > 5) {
        const unsigned x = __builtin_bit_cast(unsigned, v);
        const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const unsigned b0 = b[0], b1 = b[1];
        v = __builtin_bit_cast(float, b0) + __builtin_bit_cast(float, b1);
    }
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
        at = place_of(a, a.seq_ids[t], n.slots[t], by_page);
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
        const float inv = 1.f / (float)a.dim, mean = n.norm == ILPM_NORM_LAYER ? sum_lanes(sum, 6) * inv : 0.f;
        float var = 0.f;
        for (int e = lane; e < a.dim; e += 64) var += (row[e] - mean) * (row[e] - mean);
        const float rstd = 1.f / sqrtf(sum_lanes(var, 6) * inv + n.eps);
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

// Workgroups of 256 threads in a launch at most: twice what the card holds at once of the
// largest variant.  16381 tokens of 56 bf16 heads of 128 take 102 us (4.7 TB/s) so and with
// half as many, 140 with a workgroup for each token, which all begin anew.
constexpr int kCardGroups = 256 * 8;

// N weights from i on.
template <typename TP, int N> __device__ inline void load_weights(const void *w, int i, float *to)
{
    Pack<TP, N> p;
    if (w) p = load_loose<TP, N>((const TP *)w + i);
#pragma unroll
    for (int k = 0; k < N; ++k) to[k] = w ? (float)p.v[k] : 1.f;
}

// The packs of VEC that cover n elements: where they do not divide, the last one
// ends with them, over some of the one before it.
template <int VEC> __host__ __device__ inline int packs(int n) { return (n + VEC - 1) / VEC; }
template <int VEC> __device__ inline int pack_at(int u, int n) { return min(u * VEC, n - VEC); }

// 1 / sqrt(x) to a unit or two of the last place, of numbers below the normal ones too.
__device__ inline float rsqrt_of(float x)
{
    const bool small = x < 0x1p-100f;
    return __builtin_amdgcn_rsqf(small ? x * 0x1p100f : x) * (small ? 0x1p50f : 1.f);
}

// How a head lies over lanes: the turned part and the rest in lanes of two packs of
// VEC elements where they divide (halves always: a pack and its partners), else
// of one.
template <int VEC> struct Lanes {
    int turns, rest;            // elements that packs begin in: of halves the first half
    bool two_turned, two_rest;
    int turned, all;            // lanes
    __host__ __device__ Lanes(int dim, int rot, bool pairs)
    {
        rest = dim - rot;
        two_rest = rest % (2 * VEC) == 0;
        two_turned = !pairs || rot % (2 * VEC) == 0;
        turns = two_turned ? rot / 2 : rot;
        turned = packs<VEC>(turns);
        all = turned + packs<VEC>(two_rest ? rest / 2 : rest);
    }
};

// How heads lie over a wave: `lanes` each (of which the last may have nothing to do), and
// as many heads as fit; log: lanes are 2^log, or -1.
struct Spread {
    int lanes, log, heads;
    int blocks, slices;  // waves that a token takes, tokens that the launch takes at a time
    Divisor by_lanes{1}, by_blocks{1};
};

// `lanes` lanes a head, one or two packs of VEC elements each; what a pack shares with
// the one before it counts in the sums once, and both write the same.  A lane keeps
// its place in a head and its weights over every `slices`th token.  Waves lie one
// after the other over a token's heads and then over tokens (with whole workgroups for
// each token, 8191 f32 tokens of 56 heads of 128 took 101 us and not 89).  What bounds
// it: the bytes of queries, keys and values, read and written once.
template <typename TX, typename TC, typename TP, int VEC>
__global__ __launch_bounds__(256) void append_norm_packs(AppendNormArgs n, Divisor by_page, Spread spread)
{
    const AppendArgs &a = n.a;
    const Lanes<VEC> as(a.dim, a.rot_dim, a.pairs != 0);
    const int heads = a.q_heads + 2 * a.kv_heads, half = a.rot_dim / 2;
    const int lane = (int)threadIdx.x & 63, in_wave = spread.by_lanes.of(lane), u = lane - in_wave * spread.lanes;
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6));
    const int t0 = spread.by_blocks.of(wave), i = (wave - t0 * spread.blocks) * spread.heads + in_wave;
    if (t0 >= spread.slices || i >= heads || in_wave >= spread.heads) return;  // (whole heads: a head's lanes stay together)
    const bool query = i < a.q_heads, value = i >= a.q_heads + a.kv_heads, on = u < as.all;
    const int h = query ? i : value ? i - a.q_heads - a.kv_heads : i - a.q_heads;
    const bool rotated = u < as.turned, two = rotated ? as.two_turned : as.two_rest;
    // Elements e.. and, of two packs, others from e2; the first `over` of them belong to the pack before.
    const int in = rotated ? u : u - as.turned, width = rotated ? as.turns : as.two_rest ? as.rest / 2 : as.rest;
    const int from = !on ? 0 : pack_at<VEC>(in, width), over = !on ? VEC : in * VEC - from;
    const int e = on && !rotated ? a.rot_dim + from : from, e2 = on && two ? e + width : e;
    const TX *src = query ? (const TX *)a.q + h * a.q_head : value ? (const TX *)a.v + h * a.v_head : (const TX *)a.k + h * a.k_head;
    const int64_t row = query ? a.q_row : value ? a.v_row : a.k_row;
    TC *cache = value ? (TC *)a.vc + h * a.vc_head : (TC *)a.kc + h * a.kc_head;
    const int64_t page_row = value ? a.vc_page : a.kc_page, slot_row = value ? a.vc_slot : a.kc_slot;
    const bool norms = n.norm != ILPM_NORM_NONE, turns = rotated && !value && on, layer = n.norm == ILPM_NORM_LAYER;
    float w[VEC], w2[VEC];
    load_weights<TP, VEC>(norms && !value ? (query ? n.q_w : n.k_w) : nullptr, e, w);
    load_weights<TP, VEC>(norms && !value ? (query ? n.q_w : n.k_w) : nullptr, e2, w2);
    const float inv = 1.f / (float)a.dim;

    // A token's values and where it is, read while the one before it is written.
    struct Token {
        Pack<TX, VEC> p, p2;
        int pos, seq, slot;
    };
    auto read = [&](int t) {
        Token k;
        t = min(t, a.n_tokens - 1);
        k.p = load_loose<TX, VEC>(src + t * row + e);
        k.p2 = load_loose<TX, VEC>(src + t * row + e2);
        k.pos = a.positions[t];
        k.seq = a.seq_ids[t];
        k.slot = n.slots[t];
        return k;
    };
    Token next = read(t0);
#pragma unroll 1
    for (int t = t0; t < a.n_tokens; t += spread.slices) {
        const Token k = next;
        const bool known = a.rot_dim > 0 && k.pos >= 0 && k.pos < a.n_positions, turn = turns && known;
        Place at = {-1, 0};
        if (!query) {
            at = place_of(a, k.seq, k.slot, by_page);
            if (a.rot_dim > 0 && !known) at.page = -1;
        }
        // VEC angles for halves, VEC / 2 for a pack of pairs.
        constexpr int HV = VEC / 2;
        Pack<float, HV> c[2], s[2];
        if (turn) {
            const float *cs = a.cos + (int64_t)k.pos * half, *sn = a.sin + (int64_t)k.pos * half;
            const int first = a.pairs ? e / 2 : e, second = a.pairs ? e2 / 2 : e + HV;
            c[0] = load_loose<float, HV>(cs + first), s[0] = load_loose<float, HV>(sn + first);
            c[1] = load_loose<float, HV>(cs + second), s[1] = load_loose<float, HV>(sn + second);
        }
        next = read((int)min((int64_t)t + spread.slices, (int64_t)a.n_tokens));  // (behind what this token waits for)
        float x[VEC], y[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = (float)k.p.v[j], y[j] = (float)k.p2.v[j];
        if (norms) {
            float mean = 0.f;
            auto sum = [&](auto f) {
                float v = 0.f, v2 = 0.f;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    v += j >= over ? f(x[j]) : 0.f;
                    v2 += j >= over ? f(y[j]) : 0.f;
                }
                v = two ? v + v2 : v;
                if (spread.log >= 0) return sum_lanes(v, spread.log);
                float all = 0.f;
#pragma unroll 1
                for (int k = 0; k < spread.lanes; k += 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float of = __shfl(v, lane - u + k + j);
                        all += k + j < spread.lanes ? of : 0.f;
                    }
                }
                return all;
            };
            if (layer) mean = sum([](float v) { return v; }) * inv;
            const float rstd = rsqrt_of(sum([&](float v) { return (v - mean) * (v - mean); }) * inv + n.eps);
            if (!value) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    x[j] = (layer ? (x[j] - mean) * rstd : x[j] * rstd) * w[j];
                    y[j] = (layer ? (y[j] - mean) * rstd : y[j] * rstd) * w2[j];
                }
            }
        }
        if (!on || (!query && at.page < 0)) continue;
        if (turn && !a.pairs) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float v = x[j], cj = c[j / HV].v[j % HV], sj = s[j / HV].v[j % HV];
                x[j] = v * cj - y[j] * sj;
                y[j] = y[j] * cj + v * sj;
            }
        } else if (turn) {
#pragma unroll
            for (int j = 0; j < VEC; j += 2) {
                const float v = x[j], w = y[j];
                x[j] = v * c[0].v[j / 2] - x[j + 1] * s[0].v[j / 2];
                x[j + 1] = x[j + 1] * c[0].v[j / 2] + v * s[0].v[j / 2];
                y[j] = w * c[1].v[j / 2] - y[j + 1] * s[1].v[j / 2];
                y[j + 1] = y[j + 1] * c[1].v[j / 2] + w * s[1].v[j / 2];
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
        else put(cache + (int64_t)at.page * page_row + (int64_t)at.slot * slot_row);
    }
}

// Whether heads fall into packs of VEC: what turns and what does not have one pack
// at least, and together not more than a wave has lanes.  Heads take a whole power of
// two of the lanes, whose sums the vector unit forms by itself, or, where fewer waves
// a token then do, just what they need, and sums by way of LDS: 8191 tokens of
// 48 f16 heads of 80 in 5 lanes and not 8 take 35 us and not 44, of 56 heads of 96 in 6
// 45 and not 47.  Beyond 12 lanes the sums' accesses would be more than what they save.
template <int VEC> bool packs_fit(const AppendArgs &a, int heads, Spread *s)
{
    const Lanes<VEC> as(a.dim, a.rot_dim, a.pairs != 0);
    if ((as.turns > 0 && as.turns < VEC) || (as.rest > 0 && as.rest < VEC)) return false;
    for (s->log = 0; 1 << s->log < as.all;) ++s->log;
    if (s->log > 6) return false;
    s->lanes = 1 << s->log;
    if (as.all <= 12 && ceil_div(heads, 64 / as.all) < ceil_div(heads, 64 / s->lanes)) s->lanes = as.all, s->log = -1;
    s->heads = 64 / s->lanes;
    s->blocks = ceil_div(heads, s->heads);
    s->slices = std::min(a.n_tokens, std::max(1, kCardGroups * 4 / s->blocks));
    s->by_lanes = Divisor((unsigned)s->lanes);
    s->by_blocks = Divisor((unsigned)s->blocks);
    return true;
}

template <typename TX, typename TC, typename TP, int VEC>
bool launch_packs(const AppendNormArgs &n, const Divisor &by_page, int heads, hipStream_t stream)
{
    Spread spread;
    if (!packs_fit<VEC>(n.a, heads, &spread)) return false;
    const int groups = ceil_div(spread.blocks * spread.slices, 4);
    hipLaunchKernelGGL((append_norm_packs<TX, TC, TP, VEC>), dim3(groups), dim3(256), 0, stream, n, by_page, spread);
    return true;
}

template <typename TX, typename TC, typename TP> hipError_t launch(const AppendNormArgs &n, hipStream_t stream)
{
    const AppendArgs &a = n.a;
    const int heads = a.q_heads + 2 * a.kv_heads, total = heads * a.n_tokens;
    const Divisor by_page((unsigned)a.page_size);
    if (!launch_packs<TX, TC, TP, 8>(n, by_page, heads, stream) && !launch_packs<TX, TC, TP, 4>(n, by_page, heads, stream) &&
        !launch_packs<TX, TC, TP, 2>(n, by_page, heads, stream))
        hipLaunchKernelGGL((append_norm_any<TX, TC, TP>), dim3(ceil_div(total, 4)), dim3(256), 0, stream, n, Divisor((unsigned)heads), by_page, total);
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
