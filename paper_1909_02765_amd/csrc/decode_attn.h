// attn_decode's kernel: attention of one new token a sequence over a paged
// cache,
//   x_j = scale <q, k_j>,  out = sum e^(x_j - m) v_j / sum e^(x_j - m),  m = max x_j,
// in one pass over the keys with the running maximum and sum of the softmax,
// split over the length and joined (decode_attn.hip).
//
// Both products run on the matrix cores, 16 keys x 16 query heads of one key
// head at a time.  The first gives the scores transposed, S[key][head] = sum_d
// K[key][d] Q[head][d], so that lane (n, g) = (lane % 16, lane / 16) holds keys
// 4g..4g+3 of head n.  That is the layout in which the second one
// (v_mfma_f32_16x16x4_f32) wants its operand, O[d][head] = sum_key V[key][d]
// P[key][head], with keys 4g + r as the contraction of instruction r: the
// probabilities stay in 32 bits and never leave their lane, the statistics of a
// head are one value per lane, and a lane's V operand is V[4g + r][d], an element
// of a row that it loads as it lies in memory (a 16-bit second product would
// want values of several keys in one register, and probabilities of 16 bits).
// The first product takes the 16-bit instruction (16x16x32) where queries and
// cache are of one 16-bit type, as both are exact there, else the 32-bit one.
//
// What bounds it: the cache's bytes.  A tile of 16 keys of 128 16-bit values is 8
// KiB and keeps a SIMD's matrix core busy for 1088 cycles, 30 bytes a cycle for
// a compute unit, where its share of the memory's rate is 8.
#pragma once

#include "decode.h"

namespace ilpm {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kHeads = 16;  // query heads of a workgroup
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// How rows lie in memory: whole (16-byte pieces, dim is the class's size), in
// 16-byte pieces, or in no such order (element by element).
enum Rows { kWhole, kPieces, kAny };

__device__ inline float load_f32(const void *p, int64_t i, int dtype)
{
    if (dtype == ILPM_F32) return ((const float *)p)[i];
    if (dtype == ILPM_F16) return (float)((const _Float16 *)p)[i];
    return (float)((const __bf16 *)p)[i];
}

__device__ inline void store_f32(void *p, int64_t i, int dtype, float v)
{
    if (dtype == ILPM_F32) ((float *)p)[i] = v;
    else if (dtype == ILPM_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// The keys of a sequence that the window leaves: [first, end).
__device__ inline void visible_range(const AttnArgs &a, int seq, int *first, int *end)
{
    const int length = a.lengths[seq], n = min(max(length, 0), a.capacity);
    *end = n;
    // (The window counts from the sequence's own length, also where the table ends before it.)
    *first = a.window > 0 ? min(n, max(length - a.window, 0)) : 0;
}

// Splits that a sequence's visible keys fill.
__device__ inline int splits_of(const AttnArgs &a, int keys)
{
    return min((int)(((int64_t)keys + a.chunk - 1) / a.chunk), a.splits);
}

// The maximum over the four lanes of a head (n, 0..3).  (The halves of a swap
// are taken out before they are cast: cast in place, both give the first.)
__device__ inline float max_of_head(float v)
{
    unsigned x = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const unsigned a0 = a[0], a1 = a[1];
    x = __builtin_bit_cast(unsigned, fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const unsigned b0 = b[0], b1 = b[1];
    return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// N elements of a row from element d on.  What lies beyond `dim` is 0 with
// ZERO, else any of the row's own values.
template <typename T, int N, Rows R, bool ZERO> __device__ inline Pack<T, N> load_row(const T *row, int d, int dim)
{
    Pack<T, N> p;
    if constexpr (R == kAny) {
#pragma unroll
        for (int i = 0; i < N; ++i) p.v[i] = d + i < dim ? row[d + i] : (T)0.f;
    } else {
        p = *reinterpret_cast<const Pack<T, N> *>(row + (R == kWhole || d < dim ? d : 0));
        if (R == kPieces && ZERO && d >= dim) p = Pack<T, N>{};
    }
    return p;
}

// TC: the cache's type.  Q16: the queries are of that same 16-bit type (else
// any, taken in 32 bits).  DC: the head size's class (64, 128 or 256).
template <typename TC, bool Q16, int DC, Rows R> struct AttnKernel {
    static constexpr int KV = 16 / (int)sizeof(TC);          // elements of a K load
    static constexpr int NK = DC / (4 * KV);                 // K loads of a lane
    static constexpr int VV = KV < DC / 16 ? KV : DC / 16;   // elements of a V load
    static constexpr int NV = DC / (16 * VV);                // V loads of a lane and key
    static constexpr int NO = NV * VV;                       // output tiles of 16 values
    // A tile of 16 keys: lane (n, g) holds pieces g, g + 4, ... of key n's K row,
    // and pieces n, n + 16, ... of the V rows of keys 4g..4g+3.
    struct Tile {
        Pack<TC, KV> k[NK];
        Pack<TC, VV> v[4][NV];
        bool seen[4];
    };
};

// Where the keys of a wave's group lie (64 keys: 4 of its tiles), -1 where
// not seen.
struct Places {
    int64_t k[64], v[64];
};

template <typename TC, bool Q16, int DC, Rows R> __global__ __launch_bounds__(256) void attn_split(AttnArgs a)
{
    using Cfg = AttnKernel<TC, Q16, DC, R>;
    using Tile = typename Cfg::Tile;
    constexpr int KV = Cfg::KV, NK = Cfg::NK, VV = Cfg::VV, NV = Cfg::NV, NO = Cfg::NO;
    __shared__ Places places[4][2];
    __shared__ float sm[4][kHeads], sl[4][kHeads];
    __shared__ float so[2][64][NO * 4 + 1];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int blocks = (a.group + kHeads - 1) / kHeads;      // of a key head's query heads
    int id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int hb = id % blocks;
    id /= blocks;
    const int kvh = id % a.kv_heads, seq = id / a.kv_heads;
    const int in_group = hb * kHeads + n16;                  // this lane's query head
    const bool has_head = in_group < a.group;
    const int head = kvh * a.group + in_group;

    int first, end;
    visible_range(a, seq, &first, &end);
    const int ns = splits_of(a, end - first);
    if (split >= max(ns, 1)) return;
    const int k0 = first + split * a.chunk;
    const int k1 = split == a.splits - 1 ? end : min(k0 + a.chunk, end);
    // Tile j of this wave is tile 4j + wave of the split.
    const int tiles = max(0, ((k1 - k0 + 15) / 16 - wave + 3) / 4);

    // Lane (n, t) looks up key n of tile 4*group + t.
    struct Entry {
        int page, slot;
    };
    auto look_up = [&](int group) {
        Entry e = {-1, 0};
        const int64_t key = k0 + ((int64_t)(group * 4 + g) * 4 + wave) * 16 + n16;
        if (key < k1) {
            const int at = (int)key / a.page_size;
            e.slot = (int)key - at * a.page_size;
            e.page = a.table[(int64_t)seq * a.table_stride + at];
            if (a.mask && (key >= a.mask_len || !a.mask[(int64_t)seq * a.mask_stride + key])) e.page = -1;
        }
        return e;
    };
    auto place = [&](int group, Entry e) {
        const bool ok = e.page >= 0 && e.page < a.n_pages;
        Places &p = places[wave][group & 1];
        p.k[lane] = ok ? (int64_t)e.page * a.k_page + (int64_t)e.slot * a.k_slot : -1;
        p.v[lane] = ok ? (int64_t)e.page * a.v_page + (int64_t)e.slot * a.v_slot : -1;
        // (Only this wave reads them, and a wave's LDS accesses keep their order.)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const TC *kh = (const TC *)a.k + (int64_t)kvh * a.k_head;
    const TC *vh = (const TC *)a.v + (int64_t)kvh * a.v_head;
    // A key that is not seen reads the pool's first row, and none of it is used.
    auto load = [&](int j, Tile &t) {
        const Places &p = places[wave][(j >> 2) & 1];
        const int at = (j & 3) * 16;
        const TC *krow = kh + max(p.k[at + n16], (int64_t)0);
#pragma unroll
        for (int c = 0; c < NK; ++c) t.k[c] = load_row<TC, KV, R, true>(krow, (g + 4 * c) * KV, a.dim);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t vo = p.v[at + 4 * g + r];
            t.seen[r] = vo >= 0;
            const TC *vrow = vh + max(vo, (int64_t)0);
#pragma unroll
            for (int c = 0; c < NV; ++c) t.v[r][c] = load_row<TC, VV, R, false>(vrow, (n16 + 16 * c) * VV, a.dim);
        }
    };

    Entry next = {};
    if (tiles > 0) {
        place(0, look_up(0));
        if (tiles > 4) next = look_up(1);
    }

    // The queries, in the layout of the K loads.
    Pack<TC, KV> q16[NK];
    float q32[NK][KV];
#pragma unroll
    for (int c = 0; c < NK; ++c)
#pragma unroll
        for (int i = 0; i < KV; ++i) {
            const int d = (g + 4 * c) * KV + i;
            const bool ok = has_head && d < a.dim;
            const int64_t at = (int64_t)seq * a.q_row + (int64_t)head * a.q_head + d;
            if constexpr (Q16) q16[c].v[i] = ok ? ((const TC *)a.q)[at] : (TC)0.f;
            else q32[c][i] = ok ? load_f32(a.q, at, a.q_dtype) : 0.f;
        }

    floatx4 o[NO];
#pragma unroll
    for (int i = 0; i < NO; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float scale2 = a.softcap > 0.f ? a.scale / a.softcap : a.scale * kLog2e;
    const float cap2 = a.softcap * kLog2e;

    auto compute = [&](const Tile &t) {
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            if constexpr (Q16 && sizeof(TC) == 2 && __is_same(TC, __bf16)) {
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[c]),
                                                            __builtin_bit_cast(bf16x8, q16[c]), s, 0, 0, 0);
            } else if constexpr (Q16) {
                s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, t.k[c]),
                                                           __builtin_bit_cast(f16x8, q16[c]), s, 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < KV; ++i)
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32((float)t.k[c].v[i], q32[c][i], s, 0, 0, 0);
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float x = s[r] * scale2;
            if (a.softcap > 0.f) x = cap2 * tanhf(x);
            s[r] = t.seen[r] ? x : -INFINITY;
            top = fmaxf(top, s[r]);
        }
        const float m_new = fmaxf(m, max_of_head(top));
        const float base = m_new == -INFINITY ? 0.f : m_new;
        if (__builtin_amdgcn_ballot_w64(m_new != m)) {  // (most tiles leave all maxima where they are)
            const float alpha = __builtin_amdgcn_exp2f(m - base);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < NO; ++i) o[i] *= alpha;
        }
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] - base);
        l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < VV; ++i)
                    o[c * VV + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.seen[r] ? (float)t.v[r][c].v[i] : 0.f, p[r],
                                                                        o[c * VV + i], 0, 0, 0);
    };

    // While a tile is computed the next one's rows are on their way, and the
    // next group's table entries.
    Tile buf[2];
    if (tiles > 0) load(0, buf[0]);
    for (int j = 0; j < tiles; j += 2) {
        if ((j & 3) == 2 && j + 2 < tiles) {
            place(j / 4 + 1, next);
            if (j + 6 < tiles) next = look_up(j / 4 + 2);
        }
        if (j + 1 < tiles) load(j + 1, buf[1]);
        compute(buf[0]);
        if (j + 2 < tiles) load(j + 2, buf[0]);
        if (j + 1 < tiles) compute(buf[1]);
    }

    // Join the four waves: l first over the lanes of a head, then all to their
    // common maximum.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        sm[wave][n16] = m;
        sl[wave][n16] = l;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(sm[0][n16], sm[1][n16]), fmaxf(sm[2][n16], sm[3][n16]));
    const float base = top == -INFINITY ? 0.f : top;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) l += sl[w][n16] * __builtin_amdgcn_exp2f(sm[w][n16] - base);
    const float f = __builtin_amdgcn_exp2f(m - base);
#pragma unroll
    for (int i = 0; i < NO; ++i) o[i] *= f;
    auto give = [&](int slot) {
#pragma unroll
        for (int i = 0; i < NO; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) so[slot][lane][i * 4 + r] = o[i][r];
    };
    auto take = [&](int slot) {
#pragma unroll
        for (int i = 0; i < NO; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[i][r] += so[slot][lane][i * 4 + r];
    };
    if (wave >= 2) give(wave - 2);
    __syncthreads();
    if (wave < 2) take(wave);
    if (wave == 1) give(1);
    __syncthreads();
    if (wave != 0 || !has_head) return;
    take(1);
    const bool whole = ns <= 1;
    const int64_t row = (int64_t)seq * a.q_heads + head;
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    float *part = whole ? nullptr : a.part_o + (row * a.splits + split) * a.dim;
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < VV; ++i) {
                const int d = (4 * g + r + 16 * c) * VV + i;
                if (d >= a.dim) continue;
                const float v = o[c * VV + i][r] * inv;
                if (whole) store_f32(a.out, (int64_t)seq * a.o_row + (int64_t)head * a.o_head + d, a.q_dtype, v);
                else part[d] = v;
            }
    if (g == 0) {
        if (whole) {
            if (a.lse) a.lse[row] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
        } else {
            float *ml = a.part_ml + (row * a.splits + split) * 2;
            ml[0] = top;
            ml[1] = l;
        }
    }
}

template <typename TC, bool Q16, int DC> hipError_t attn_split_launch(const AttnArgs &a, hipStream_t stream)
{
    const int64_t step = 16 / (int64_t)sizeof(TC);
    const bool pieces = a.dim % step == 0 && ((uintptr_t)a.k | (uintptr_t)a.v) % 16 == 0 &&
                        (a.k_page | a.k_slot | a.k_head | a.v_page | a.v_slot | a.v_head) % step == 0;
    const dim3 grid((unsigned)(a.n_seqs * a.kv_heads * ceil_div(a.group, kHeads) * a.splits));
    if (pieces && a.dim == DC) hipLaunchKernelGGL((attn_split<TC, Q16, DC, kWhole>), grid, dim3(256), 0, stream, a);
    else if (pieces) hipLaunchKernelGGL((attn_split<TC, Q16, DC, kPieces>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((attn_split<TC, Q16, DC, kAny>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <typename TC, bool Q16> hipError_t attn_split_by_dim(const AttnArgs &a, hipStream_t stream)
{
    if (a.dim <= 64) return attn_split_launch<TC, Q16, 64>(a, stream);
    if (a.dim <= 128) return attn_split_launch<TC, Q16, 128>(a, stream);
    return attn_split_launch<TC, Q16, 256>(a, stream);
}

}  // namespace
}  // namespace ilpm
