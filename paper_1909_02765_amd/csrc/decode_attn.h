// attn_decode's kernel: attention of one new token a sequence over a paged
// cache,
//   x_j = scale <q, k_j>,  out = sum e^(x_j - m) v_j / sum e^(x_j - m),  m = max x_j,
// in one pass over the keys with the running maximum and sum of the softmax.
//
// Both products run on the matrix cores, 16 keys x 16 query heads of one key
// head at a time.  The first gives the scores transposed, S[key][head] = sum_d
// K[key][d] Q[head][d], so that lane (n, g) = (lane % 16, lane / 16) holds keys
// 4g..4g+3 of head n.  That is the layout in which the second one wants its
// operand, O[d][head] = sum_key V[key][d] P[key][head], with keys 4g..4g+3 of
// the contraction in lane (n, g): the probabilities never leave their lane, and
// the statistics of a head are one value per lane.  A lane's V operand is values
// V[4g..4g+3][d], of rows that it loads as they lie in memory.
//
//   f32 cache: 16x16x4 instructions on 32-bit values, one key of each lane a time.
//   16-bit cache: 16x16x32 for the scores; for the second product 16x16x16, whose
//     operand of four keys comes together from four rows by byte permutations,
//     and in them keys that are not seen become 0.  Probabilities, and queries
//     of 32 bits, go in as 16-bit parts (one the value rounded, the next one what
//     is left, rounded).  Queries: three, which keep all their bits (over f16 those
//     above 2^-39 of the largest's).  Probabilities: two under 16-bit queries, which
//     hold bf16 ones to 2^-17 of them and f16 ones to 2^-23, for outputs of 8 and 11
//     bits; three under 32-bit queries over bf16, which keep all bits; two there over
//     f16, whose 2^-23 is a unit of the last place of 32 bits, as much as the
//     exponential itself may be off (a third costs up to 11%: 8 ragged sequences of up
//     to 30001 keys of 8 heads of 64 58.2 -> 64.8 us).  f16 parts are scaled by powers
//     of two so that they keep what is above 2^-40 of the largest.  The first part
//     has an accumulator of its own: an infinity in the cache makes infinities or
//     NaN of it as the definition does (of f16 probabilities below 2^-40, whose first
//     part is 0, NaN), while the products with the small parts may be NaN where
//     it has none (0 times infinity), and are left out if so.
//
// How the work is divided: the tiles of 16 keys of all (sequence, key head)
// units lie in one row, which the workgroups share out evenly, as many as the
// card holds at once (see Share).  A workgroup takes its share unit by unit; a
// unit that spans workgroups leaves partial results, which attn_join adds.
//
// What bounds it: the cache's bytes (131071 keys of 8 bf16 heads of 128 under 32
// query heads 106 us, 64 ragged sequences of up to 8191 of them 210 us, 5.0 TB/s
// with the join).  f32 queries over heads of 72 and 80 stay below that (117164 keys
// of 7 f16 heads of 72 under 84 79 us, 3.0 TB/s; their second product is done over the
// 128 values that sixteen lanes load), and so do single heads with window, mask and soft
// cap (24 sequences of 12 f16 heads of 80, window 1000: 27 us, 2.6 TB/s).  In both the
// vector unit issues in 32 to 40% of the cycles and the matrix cores are busy in 7 to
// 11%: neither is full, and two waves a SIMD do not cover each other's waits.  Of calls with a tile or two a wave it is the accesses that wait
// for each other (lengths, pages, rows, the join: f32 queries over 16 shared bf16
// heads of 256, 8 sequences of up to 2049, 15 us).
#pragma once

#include <climits>
#include <type_traits>

#include "decode.h"

namespace ilpm {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// How rows lie in memory: whole (16-byte pieces, dim is the class's size), in
// 16-byte pieces, or in no such order (element by element, for pools that are off
// that alignment and sizes that are no whole pieces: 131071 keys of 8 bf16 heads of 128
// under 32 take 573 us so in place of 107, 65000 of 8 heads of 64 under f32 queries 89
// in place of 33).
enum Rows { kWhole, kPieces, kAny };

// The keys of a sequence that the window leaves: [first, end).
__device__ inline void visible_range(const AttnArgs &a, int length, int *first, int *end)
{
    const int own = max(length, 0), n = min(own, a.capacity);
    *end = n;
    // (The window counts from the sequence's own length, also where the table ends before it.)
    *first = a.window > 0 ? min(n, max(own - a.window, 0)) : 0;
}

// Tiles of 16 keys of a unit of a sequence of this length; 1 for one without
// keys, so that somebody writes its output.  What a unit costs beside its tiles
// counts as kUnitCost of them (without it one workgroup got all the shortest
// sequences of a batch: 82 us where the others took 25).
__device__ inline int tiles_of(const AttnArgs &a, int length)
{
    int first, end;
    visible_range(a, length, &first, &end);
    return max(1, (int)(((unsigned)(end - first) + 15) / 16));
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

// tanh to a few units of the last place: its series near 0, where the form by
// the exponential would lose bits, else 1 - 2 / (e^2x + 1).
__device__ inline float tanh_of(float x)
{
    const float x2 = x * x;
    float near = 62.f / 2835.f;
    near = near * x2 - 17.f / 315.f;
    near = near * x2 + 2.f / 15.f;
    near = near * x2 - 1.f / 3.f;
    near = near * x2 * x + x;
    const float e = __builtin_amdgcn_exp2f(fminf(fabsf(x), 20.f) * (2.f * kLog2e));
    float far = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), x);
    asm("" : "+v"(near), "+v"(far));  // (both, without a branch)
    far = x != x ? x : far;
    return fabsf(x) < 0.25f ? near : far;
}

// Pieces of rows are held as machine words, whatever they mean: as arrays of
// 16-bit values the compiler takes them apart when they arrive, which waits
// for them at once, and puts them together again where they are used.
template <int BYTES> using Words = typename PackWord<BYTES>::type;
typedef Words<16> Words16;

__device__ const Words16 attn_zeros = {0, 0, 0, 0};

// N elements of a row from element d on.  What lies beyond `dim` is 0 with
// ZERO (a piece of zeros is read for it), else any of the row's own values.
template <typename T, int N, Rows R, bool ZERO> __device__ inline Words<sizeof(T) * N> load_row(const T *row, int d, int dim)
{
    using W = Words<sizeof(T) * N>;
    if constexpr (R == kAny) {
        Pack<T, N> p;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const T v = row[min(d + i, dim - 1)];
            p.v[i] = !ZERO || d + i < dim ? v : (T)0.f;
        }
        return __builtin_bit_cast(W, p);
    } else if constexpr (R == kPieces) {
        return *reinterpret_cast<const W *>(d < dim ? row + d : ZERO ? (const T *)&attn_zeros : row);
    } else {
        return *reinterpret_cast<const W *>(row + d);
    }
}

template <typename TC> __device__ inline floatx4 mfma_scores(Words16 k, Words16 q, floatx4 c)
{
    if constexpr (__is_same(TC, __bf16))
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, k), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
}
template <typename TC> __device__ inline floatx4 mfma_values(Words<8> v, Words<8> p, floatx4 c)
{
    if constexpr (__is_same(TC, __bf16))
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(shortx4, v), __builtin_bit_cast(shortx4, p), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, v), __builtin_bit_cast(f16x4, p), c, 0, 0, 0);
}

// TC: the cache's type.  Q16: queries and outputs are of that same 16-bit type
// (else f32).  DC: the head size's class (64, 96, 128, 192 or 256).  SHORT: for
// calls whose sequences are all short, a unit to a workgroup: one tile at a
// time, in half the registers and instructions (an instruction that runs once
// costs its fetching, and more workgroups fit a compute unit: 127 one-token
// sequences of 16 f32 heads of 192 39 -> 19 us).
template <typename TC, bool Q16, int DC, Rows R, bool SHORT> struct AttnKernel {
    static constexpr bool C16 = sizeof(TC) == 2;
    static constexpr int KV = 16 / (int)sizeof(TC);          // elements of a K load
    static constexpr int NK = DC / (4 * KV);                 // K loads of a lane
    // Elements of a V load: 16 bytes, or 8 where sixteen lanes then make up the row.
    static constexpr int VV = C16 && DC != 64 && DC != 192 ? 8 : 4;
    static constexpr int NV = (DC + 16 * VV - 1) / (16 * VV);  // V loads of a lane and key
    static constexpr int NO = NV * VV;                       // output tiles of 16 values
    static constexpr int DO = NO * 16;                       // values that they hold
    static constexpr int QP = C16 && !Q16 ? 3 : 1;           // parts of a query
    static constexpr int PP = __is_same(TC, __bf16) && !Q16 ? 3 : 2;  // parts of a probability (16-bit caches)
    // f16: probabilities go into the second product times this, and its sums come out so.
    // (Not by 2^(score + 15), which rounds the score at a magnitude of 15: probabilities
    // kept 21 bits that way.)
    static constexpr float UP = __is_same(TC, _Float16) ? 0x1p15f : 1.f;
    // Workgroups that a compute unit holds at once (waves of a SIMD): what the
    // registers of two tiles, the queries and the output leave.  (16-bit heads of up
    // to 96 keep up to nine of their registers in memory for the third: 4 key heads over
    // 48 x 14583 bf16 keys of 72 221 us with two, 175 with three.)  The bounds of SHORT
    // kernels are those of 16-bit queries.  Under 32-bit ones they are not reached at
    // 128 (two for three) and 256 (one for two), and at 64, where they are, up to 50
    // registers of f16 caches and 17 of bf16 ones lie in memory (1 sequence of 250 keys
    // of 2 bf16 heads under 8 of 32 bits: 7.4 us).  Rows taken element by element spill
    // as much as 181.
    static constexpr int PER_CU = SHORT ? (DC == 64 ? 5 : DC <= 128 ? 3 : 2) : DC == 64 ? (QP == 3 ? 3 : 4) : DC == 96 && C16 ? 3 : DC <= 128 ? 2 : 1;
    // Whether a tile is loaded where there is none (the pool's first row for it).
    // Loads behind a condition the compiler cannot count, and waits for all of them
    // before it goes on.  Where one wave has a vector unit for itself that shows (7
    // f32 heads of 192 over 2 x 57306 keys 131 us, without the condition 105);
    // where several have, a call of few tiles a wave is 1 us longer without it.
    static constexpr bool ALWAYS = !SHORT && !C16 && DC >= 192;
    // A tile of 16 keys: lane (n, g) holds pieces g, g + 4, ... of key n's K row,
    // and pieces n, n + 16, ... of the V rows of keys 4g..4g+3.
    struct Tile {
        Words16 k[NK];
        Words<sizeof(TC) * VV> v[4][NV];
        bool seen[4];
    };
};

// Where the keys of a wave's group lie (64 keys: 4 of its tiles), -1 where
// not seen.
struct Places {
    int64_t k[64], v[64];
};

// How the units are shared out: they lie in one row, each kUnitCost and then
// its tiles long, cut into shares of `size`; or (whole) a unit goes to a
// workgroup at a time, where the units are short and too few to fill the card.
// (All units together are shorter than 2^31: attn_plan.)
struct Share {
    int total;  // the row's length
    int size;
    bool whole;
};

// What is the same in all lanes, as the compiler cannot know of values from LDS.
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct FindShare {
    int sum[4], top[4];
    int seq, length, before;
};

// The sum over the workgroup of a value of each thread; *up_to: the sum up to
// and with this thread's.
__device__ inline int scan256(int v, int *up_to, FindShare &f)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 1
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    __syncthreads();
    if (lane == 63) f.sum[wave] = v;
    __syncthreads();
    const int s0 = f.sum[0], s1 = s0 + f.sum[1], s2 = s1 + f.sum[2];
    *up_to = v + (wave == 0 ? 0 : wave == 1 ? s0 : wave == 2 ? s1 : s2);
    return uniform(s2 + f.sum[3]);
}

// Units of a sequence (key heads x blocks of up to 16 of their query heads).
__device__ inline int units_of(const AttnArgs &a) { return a.kv_heads * a.blocks; }

// Where a share begins: in this sequence of this length, with units that take
// `before` of the row before it.
struct Begin {
    int seq, length, before;
};

__device__ inline Share share_of(const AttnArgs &a, int total, int top)
{
    Share s;
    s.total = total * units_of(a);
    const int even = (int)(((unsigned)s.total + gridDim.x - 1) / gridDim.x);
    s.size = max(kMinShare, even);
    s.whole = s.size == kMinShare && top <= kWholeTiles;
    return s;
}

// The shares of this call, and where share `wg` begins (if it lies in the row).
__device__ inline Share find_share(const AttnArgs &a, int wg, FindShare &f, Begin *begin)
{
    const int tid = threadIdx.x, units = units_of(a);
    *begin = Begin{0, 0, 0};
    if (a.n_seqs <= 64) {  // each wave for itself
        const int lane = tid & 63;
        const int length = lane < a.n_seqs ? a.lengths[lane] : 0;
        const int t = lane < a.n_seqs ? tiles_of(a, length) : 0, cost = t > 0 ? t + kUnitCost : 0;
        int top = t, up_to = cost;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = max(top, __shfl_xor(top, d));
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(up_to, d);
            up_to += lane >= d ? o : 0;
        }
        const Share s = share_of(a, __builtin_amdgcn_readlane(up_to, 63), uniform(top));
        const int64_t at = (int64_t)wg * s.size;
        if (s.whole || at >= s.total) return s;
        // The sequence that holds this place, counted in one unit of each.
        const int want = (int)at / units;
        const int seq = __builtin_ctzll(__builtin_amdgcn_ballot_w64(want < up_to));
        begin->seq = seq;
        begin->length = __builtin_amdgcn_readlane(length, seq);
        begin->before = __builtin_amdgcn_readlane(up_to - cost, seq) * units;
        return s;
    }
    int mine = 0, top = 0, up_to;
    for (int i = tid; i < a.n_seqs; i += 256) {
        const int t = tiles_of(a, a.lengths[i]);
        mine += t + kUnitCost;
        top = max(top, t);
    }
#pragma unroll 1
    for (int d = 32; d > 0; d >>= 1) top = max(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) f.top[tid >> 6] = top;
    const int total = scan256(mine, &up_to, f);
    const Share s = share_of(a, total, uniform(max(max(f.top[0], f.top[1]), max(f.top[2], f.top[3]))));
    const int64_t at = (int64_t)wg * s.size;
    if (s.whole || at >= s.total) return s;
    const int want = (int)at / units;
    int carry = 0;
    for (int i0 = 0; i0 < a.n_seqs && want >= carry; i0 += 256) {
        const int length = i0 + tid < a.n_seqs ? a.lengths[i0 + tid] : 0;
        const int t = i0 + tid < a.n_seqs ? tiles_of(a, length) + kUnitCost : 0;
        // (Up to 256 sequences the sums are there.)
        const int sum = a.n_seqs <= 256 ? total : scan256(t, &up_to, f);
        const int to = carry + up_to;
        if (want >= to - t && want < to) {
            f.seq = i0 + tid;
            f.length = length;
            f.before = (to - t) * units;
        }
        carry += sum;
    }
    __syncthreads();
    *begin = Begin{uniform(f.seq), uniform(f.length), uniform(f.before)};
    return s;
}

// Some of a unit's keys, as a workgroup takes them.
struct Segment {
    int seq, kvh, hb;
    int k0, k1;  // [k0, k1) of the sequence's tokens
};

template <typename Cfg, typename TC> struct AttnLds {
    Places places[4][2];
    // Each wave's maxima, sums and outputs of a segment (the rows 4 banks apart).
    float m[4][kAttnHeads], l[4][kAttnHeads];
    float o[4][kAttnHeads][Cfg::DO + 4];
    FindShare found;
    // The three parts of 32-bit queries, as the lanes of the first product take them.
    Words16 q[Cfg::QP == 3 ? 3 : 1][Cfg::QP == 3 ? Cfg::NK : 1][Cfg::QP == 3 ? 64 : 1];
    float unscale[kAttnHeads];
};

// The workgroup splits a unit's 32-bit queries into their parts (once for its
// four waves, and in a loop: instructions that run once cost their fetching).
template <typename TC, int DC, Rows R, typename Lds>
__device__ __forceinline__ void split_queries(const AttnArgs &a, const Segment &seg, Lds &lds)
{
    using Cfg = AttnKernel<TC, false, DC, R, false>;
    constexpr int KV = Cfg::KV, NK = Cfg::NK;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), n16 = lane & 15, g = lane >> 4;
    const int in_group = min(seg.hb * kAttnHeads + n16, a.group - 1);
    const float *row = (const float *)a.q + (int64_t)seg.seq * a.q_row + ((int64_t)seg.kvh * a.group + in_group) * a.q_head;
    struct Values {
        float v[KV];
    };
    auto get = [&](int c) {  // KV = 8 values: two pieces of four
        struct Halves {
            Words16 w[2];
        } h;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int d = (g + 4 * c) * KV + 4 * n;
            h.w[n] = a.q_pieces ? load_row<float, 4, kPieces, true>(row, d, a.dim) : load_row<float, 4, kAny, true>(row, d, a.dim);
        }
        return __builtin_bit_cast(Values, h);
    };
    float f = 1.f, back = 1.f;
    if constexpr (__is_same(TC, _Float16)) {
        // The largest becomes 2^14 to 2^15: parts keep what is above 2^-39 of it.
        float most = 0.f;
#pragma unroll 2
        for (int c = 0; c < NK; ++c) {
            const Values p = get(c);
#pragma unroll
            for (int i = 0; i < KV; ++i) most = fmaxf(most, fabsf(p.v[i]));
        }
        most = max_of_head(most);
        const int e = (int)(__builtin_bit_cast(unsigned, most) >> 23) - 127;  // 2^e <= most < 2^(e+1)
        const int by = most > 0.f && e < 128 ? min(14 - e, 126) : 0;
        f = __builtin_ldexpf(1.f, by);
        back = __builtin_ldexpf(1.f, -by);
    }
    if (wave == 0 && g == 0) lds.unscale[n16] = back;
    Values mine[(NK + 3) / 4];
#pragma unroll
    for (int j = 0; j < (NK + 3) / 4; ++j) mine[j] = get(min(wave + 4 * j, NK - 1));
#pragma unroll
    for (int j = 0; j < (NK + 3) / 4; ++j) {
        const int c = min(wave + 4 * j, NK - 1);  // (the last one several times over, with the same values)
        const Values p = mine[j];
        Pack<TC, KV> part[3];
#pragma unroll
        for (int i = 0; i < KV; ++i) {
            float v = p.v[i] * f;
            if constexpr (__is_same(TC, __bf16)) {
                // Cut off, not rounded, which beyond bf16's largest value gives infinity: the parts
                // after it hold the rest all the same.  (A NaN keeps a bit of its upper half.)
                v = __builtin_canonicalizef(v);
                part[0].v[i] = __builtin_bit_cast(__bf16, (unsigned short)(__builtin_bit_cast(unsigned, v) >> 16));
            } else {
                part[0].v[i] = (TC)v;
            }
            v -= (float)part[0].v[i];
            part[1].v[i] = (TC)v;
            part[2].v[i] = (TC)(v - (float)part[1].v[i]);
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) lds.q[n][c][lane] = __builtin_bit_cast(Words16, part[n]);
    }
    __syncthreads();
}

// A wave's part of a segment, every fourth tile of it, its results left in LDS.
template <typename TC, bool Q16, int DC, Rows R, bool SHORT>
__device__ __forceinline__ void attn_segment(const AttnArgs &a, const Segment &seg, AttnLds<AttnKernel<TC, Q16, DC, R, SHORT>, TC> &lds)
{
    using Cfg = AttnKernel<TC, Q16, DC, R, SHORT>;
    using Tile = typename Cfg::Tile;
    using TQ = std::conditional_t<Q16, TC, float>;
    constexpr int KV = Cfg::KV, NK = Cfg::NK, VV = Cfg::VV, NV = Cfg::NV, NO = Cfg::NO;
    constexpr int QP = Cfg::QP, PP = Cfg::PP;
    constexpr bool C16 = Cfg::C16;

    // (Formed anew for each segment: kept over them, what comes of the lane
    // would take the registers that the tiles need.)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int wave = uniform((int)(threadIdx.x >> 6));
    const int n16 = lane & 15, g = lane >> 4;
    const int in_group = seg.hb * kAttnHeads + n16;  // this lane's query head
    const bool has_head = in_group < a.group;
    const int seq = seg.seq, k0 = seg.k0, k1 = seg.k1;
    // Tile j of this wave is tile 4j + wave of the segment.  (None where there
    // are no keys: then there may be no pool either.)
    const int tiles = max(0, ((int)(((unsigned)(k1 - k0) + 15) / 16) - wave + 3) / 4);

    // Lane (n, t) looks up key n of tile 4*group + t.
    struct Entry {
        int page, slot;
    };
    auto look_up = [&](int group) {
        Entry e = {-1, 0};
        const int64_t key = k0 + ((int64_t)(group * 4 + g) * 4 + wave) * 16 + n16;
        if (key < k1) {
            const int p = (int)key / a.page_size;
            e.slot = (int)key - p * a.page_size;
            e.page = a.table[(int64_t)seq * a.table_stride + p];
            if (a.mask && (key >= a.mask_len || !a.mask[(int64_t)seq * a.mask_stride + key])) e.page = -1;
        }
        return e;
    };
    auto place = [&](int group, Entry e) {
        const bool ok = e.page >= 0 && e.page < a.n_pages;
        Places &p = lds.places[wave][group & 1];
        p.k[lane] = ok ? (int64_t)e.page * a.k_page + (int64_t)e.slot * a.k_slot : -1;
        p.v[lane] = ok ? (int64_t)e.page * a.v_page + (int64_t)e.slot * a.v_slot : -1;
        // (Only this wave reads them, and a wave's LDS accesses keep their order.)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const TC *kh = (const TC *)a.k + (int64_t)seg.kvh * a.k_head;
    const TC *vh = (const TC *)a.v + (int64_t)seg.kvh * a.v_head;
    // A key that is not seen reads the pool's first row, and none of it is used.
    auto load = [&](int j, Tile &t) {
        const Places &p = lds.places[wave][(j >> 2) & 1];
        const int i0 = (j & 3) * 16;
        const bool real = !Cfg::ALWAYS || j < tiles;
        const TC *krow = kh + (real ? max(p.k[i0 + n16], (int64_t)0) : 0);
#pragma unroll
        for (int c = 0; c < NK; ++c) t.k[c] = load_row<TC, KV, R, true>(krow, (g + 4 * c) * KV, a.dim);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t vo = p.v[i0 + 4 * g + r];
            t.seen[r] = vo >= 0;
            const TC *vrow = vh + (real ? max(vo, (int64_t)0) : 0);
#pragma unroll
            for (int c = 0; c < NV; ++c)  // (sixteen lanes may reach beyond a whole row)
                t.v[r][c] = load_row<TC, VV, R == kWhole && Cfg::DO != DC ? kPieces : R, false>(vrow, (n16 + 16 * c) * VV, a.dim);
        }
    };
    Entry e0 = {}, next = {};
    if (tiles > 0) e0 = look_up(0);
    if (!SHORT && tiles > 4) next = look_up(1);
    if constexpr (QP == 3) split_queries<TC, DC, R>(a, seg, lds);
    if (tiles > 0) place(0, e0);

    // The queries, in the layout of the K loads.  (Lanes without a head take
    // the last one's, and give nothing.)  Those in parts stay in LDS: beside the tiles
    // they would not fit the registers.
    Words16 q[QP == 3 ? 1 : NK];
    float unscale = 1.f;  // f16 parts of 32-bit queries are those of the queries over this
    if constexpr (QP == 3) {
        unscale = lds.unscale[n16];
    } else {
        const TQ *row = (const TQ *)a.q + (int64_t)seq * a.q_row + ((int64_t)seg.kvh * a.group + min(in_group, a.group - 1)) * a.q_head;
        if (a.q_pieces) {
#pragma unroll
            for (int c = 0; c < NK; ++c) q[c] = load_row<TQ, KV, R == kAny ? kPieces : R, true>(row, (g + 4 * c) * KV, a.dim);
        } else {
#pragma unroll
            for (int c = 0; c < NK; ++c) q[c] = load_row<TQ, KV, kAny, true>(row, (g + 4 * c) * KV, a.dim);
        }
    }

    floatx4 o[NO], ol[C16 ? NO : 1];  // (ol: of the probabilities' small parts)
    float m = -INFINITY, l = 0.f;
    const float scale2 = (a.softcap > 0.f ? a.scale / a.softcap : a.scale * kLog2e) * unscale;
    const float cap2 = a.softcap * kLog2e;

    auto compute = [&](const Tile &t) {
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
        if constexpr (!C16) {
#pragma unroll
            for (int c = 0; c < NK; ++c) {
#pragma unroll
                for (int i = 0; i < KV; ++i)
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(floatx4, t.k[c])[i], __builtin_bit_cast(floatx4, q[c])[i], s, 0, 0, 0);
            }
        } else {
            floatx4 low = s;
            int ql = lane;
            if constexpr (QP == 3) asm volatile("" : "+v"(ql));  // (read for each tile, not kept)
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                if constexpr (QP == 3) {
                    s = mfma_scores<TC>(t.k[c], lds.q[0][c][ql], s);
                    low = mfma_scores<TC>(t.k[c], lds.q[1][c][ql], low);
                    low = mfma_scores<TC>(t.k[c], lds.q[2][c][ql], low);
                } else {
                    s = mfma_scores<TC>(t.k[c], q[c], s);
                }
            }
            if constexpr (QP == 3) {
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] += low[r] - low[r] == 0.f ? low[r] : 0.f;
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float x = s[r] * scale2;
            if (a.softcap > 0.f) x = cap2 * tanh_of(x);
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
            for (int i = 0; i < NO; ++i) {
                o[i] *= alpha;
                if constexpr (C16) ol[i] *= alpha;
            }
        }
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] - base);
        l += (p[0] + p[1]) + (p[2] + p[3]);
        if constexpr (!C16) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int i = 0; i < VV; ++i)
                        o[c * VV + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.seen[r] ? __builtin_bit_cast(floatx4, t.v[r][c])[i] : 0.f, p[r],
                                                                            o[c * VV + i], 0, 0, 0);
        } else {
            Words<8> part[PP];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[r] *= Cfg::UP;
                if constexpr (Cfg::UP != 1.f) asm("" : "+v"(p[r]));  // (one product, not one for each of its uses)
            }
#pragma unroll
            for (int i = 0; i < PP; ++i) {
                Pack<TC, 4> h;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    h.v[r] = (TC)p[r];
                    p[r] -= (float)h.v[r];
                }
                part[i] = __builtin_bit_cast(Words<8>, h);
            }
            // Selectors of the lower and the upper halves of two rows' registers: a byte 0x0c gives 0.
            unsigned lower[2], upper[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned keep = (t.seen[2 * h] ? 0xffffu : 0u) | (t.seen[2 * h + 1] ? 0xffff0000u : 0u);
                lower[h] = (0x05040100u & keep) | (0x0c0c0c0cu & ~keep);
                upper[h] = (0x07060302u & keep) | (0x0c0c0c0cu & ~keep);
            }
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < VV; ++i) {
                    const Words<8> v = {__builtin_amdgcn_perm(t.v[1][c][i / 2], t.v[0][c][i / 2], i & 1 ? upper[0] : lower[0]),
                                        __builtin_amdgcn_perm(t.v[3][c][i / 2], t.v[2][c][i / 2], i & 1 ? upper[1] : lower[1])};
#pragma unroll
                    for (int k = 0; k < PP; ++k) {
                        floatx4 &sum = k == 0 ? o[c * VV + i] : ol[c * VV + i];
                        sum = mfma_values<TC>(v, part[k], sum);
                    }
                }
        }
    };

    // While a tile is computed the next one's rows are on their way, and the
    // next group's table entries.
#pragma unroll
    for (int i = 0; i < NO; ++i) {
        o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if constexpr (C16) ol[i] = o[i];
    }
    Tile buf[SHORT ? 1 : 2];
    if constexpr (SHORT) {
#pragma unroll 1
        for (int j = 0; j < tiles; ++j) {
            if (j > 0 && (j & 3) == 0) place(j / 4, look_up(j / 4));
            load(j, buf[0]);
            compute(buf[0]);
        }
    } else {
        if (tiles > 0) load(0, buf[0]);
        for (int j = 0; j < tiles; j += 2) {
            if ((j & 3) == 2 && j + 2 < tiles) {
                place(j / 4 + 1, next);
                if (j + 6 < tiles) next = look_up(j / 4 + 2);
            }
            if (Cfg::ALWAYS || j + 1 < tiles) load(j + 1, buf[1]);
            compute(buf[0]);
            if (Cfg::ALWAYS || j + 2 < tiles) load(j + 2, buf[0]);
            if (j + 1 < tiles) compute(buf[1]);
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if constexpr (C16) {
#pragma unroll
        for (int i = 0; i < NO; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[i][r] += ol[i][r] - ol[i][r] == 0.f ? ol[i][r] : 0.f;
    }
    // Lane (n, g) holds values (4g + r + 16c) * VV + i of head n.
    if (g == 0) {
        lds.m[wave][n16] = m;
        lds.l[wave][n16] = l;
    }
    if (has_head) {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                Pack<float, VV> p;
#pragma unroll
                for (int i = 0; i < VV; ++i) p.v[i] = o[c * VV + i][r];
                *reinterpret_cast<Pack<float, VV> *>(&lds.o[wave][n16][(4 * g + r + 16 * c) * VV]) = p;
            }
    }
}

template <typename TC, bool Q16, int DC, Rows R, bool SHORT>
__global__ __launch_bounds__(256, (AttnKernel<TC, Q16, DC, R, SHORT>::PER_CU)) void attn_split(AttnArgs a)
{
    using Cfg = AttnKernel<TC, Q16, DC, R, SHORT>;
    using TQ = std::conditional_t<Q16, TC, float>;
    __shared__ AttnLds<Cfg, TC> lds;

    // Workgroups go round the card's eight dies, each with a cache of its own.
    // Neighbouring shares, which often hold neighbouring heads of the same
    // tokens, stay on one die, so that a line of two heads' rows is fetched once
    // (131071 keys of 8 bf16 heads of 128 111 -> 108 us).
    const int die = blockIdx.x & 7, dies = gridDim.x >> 3;
    const int units = units_of(a), wg = die * dies + min(die, (int)(gridDim.x & 7)) + (int)(blockIdx.x >> 3);
    Share share = {0, 0, true};
    Begin begin;
    if constexpr (!SHORT)
        if (a.split) share = find_share(a, wg, lds.found, &begin);

    // This workgroup's place: a sequence, its length and its units' tiles, a unit
    // of it, and how far into the unit's length the share has come.
    int seq, length, unit, tiles_all, x0 = 0;
    int at = 0, last = 0;
    if (a.split && !a.part_of_unit && threadIdx.x == 0) a.parts[wg] = AttnPart{0, 0, 0, 0};  // (whatever follows, attn_join reads it)
    if (share.whole) {
        if (wg >= a.n_seqs * units) return;
        seq = wg / units;
        unit = wg - seq * units;
        length = uniform(a.lengths[seq]);
        tiles_all = tiles_of(a, length);
    } else {
        if ((int64_t)wg * share.size >= share.total) return;
        at = wg * share.size;
        last = (int)min((int64_t)at + share.size, (int64_t)share.total);
        seq = begin.seq;
        length = begin.length;
        tiles_all = tiles_of(a, length);
        const int in = at - begin.before;
        unit = in / (tiles_all + kUnitCost);
        x0 = in - unit * (tiles_all + kUnitCost);
    }

    for (;;) {
        const int x1 = share.whole ? tiles_all + kUnitCost : min(tiles_all + kUnitCost, x0 + (last - at));
        const int tile0 = max(0, x0 - kUnitCost), seg_tiles = max(0, x1 - kUnitCost) - tile0;
        if (seg_tiles == 0) return;  // the share ends before the unit's first tile
        Segment seg;
        seg.seq = seq;
        seg.kvh = unit / a.blocks;
        seg.hb = unit - seg.kvh * a.blocks;
        int first, end;
        visible_range(a, length, &first, &end);
        seg.k0 = first + tile0 * 16;
        seg.k1 = (int)min((int64_t)end, (int64_t)seg.k0 + (int64_t)seg_tiles * 16);
        const bool all = seg_tiles == tiles_all;  // of the unit's tiles
        attn_segment<TC, Q16, DC, R, SHORT>(a, seg, lds);
        __syncthreads();

        // Join the four waves, four values of a head at a time.
        const int heads = min(kAttnHeads, a.group - seg.hb * kAttnHeads), head0 = seg.kvh * a.group + seg.hb * kAttnHeads;
        // The part that begins a unit, or the one that goes on with it.
        const int64_t part = ((int64_t)wg * 2 + (tile0 == 0 ? 1 : 0)) * a.part_heads;
        constexpr int PER = DC / 4;
#pragma unroll 1
        for (int i = threadIdx.x; i < heads * PER; i += 256) {
            const int h = i / PER, d = (i - h * PER) * 4;
            if (d >= a.dim) continue;
            floatx4 o[4];
            float m[4], l[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                o[w] = *reinterpret_cast<const floatx4 *>(&lds.o[w][h][d]);
                m[w] = lds.m[w][h];
                l[w] = lds.l[w][h];
            }
            const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f(m[w] - base);
                o[w] *= f;
                l[w] *= f;
            }
            const float sum = (l[0] + l[1]) + (l[2] + l[3]);
            floatx4 v = (o[0] + o[1]) + (o[2] + o[3]);
            auto put = [&](auto *to) {
                using TO = std::remove_reference_t<decltype(*to)>;
                Pack<TO, 4> p;
#pragma unroll
                for (int k = 0; k < 4; ++k) p.v[k] = (TO)v[k];
                if (d + 4 <= a.dim) {
                    store_loose<TO, 4>(to + d, p);
                    return;
                }
                to[d] = p.v[0];
                if (d + 1 < a.dim) to[d + 1] = p.v[1];
                if (d + 2 < a.dim) to[d + 2] = p.v[2];
            };
            if (all) {
                v *= sum == 0.f ? 0.f : 1.f / (sum * Cfg::UP);
                put((TQ *)a.out + (int64_t)seq * a.o_row + (int64_t)(head0 + h) * a.o_head);
                if (d == 0 && a.lse)
                    a.lse[(int64_t)seq * a.q_heads + head0 + h] =
                        sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
            } else {
                v *= 1.f / Cfg::UP;
                put(a.part_o + (part + h) * a.dim);
                if (d == 0) {
                    a.part_ml[(part + h) * 2] = top;
                    a.part_ml[(part + h) * 2 + 1] = sum;
                }
            }
        }
        // Who begins a unit says whether others go on with it.
        if (a.split && threadIdx.x == 0 && tile0 == 0) {
            const int rest = tiles_all - seg_tiles;
            const int count = all ? 0 : 1 + (int)(((unsigned)rest + share.size - 1) / (unsigned)share.size);
            if (a.part_of_unit) a.parts[seq * units + unit] = AttnPart{seq, unit, wg, count};
            else if (!all) a.parts[wg] = AttnPart{seq, unit, wg, count};
        }
        if (share.whole) {
            // (Long before 2^31: units are at most 2^24, workgroups too.)
            const int u = seq * units + unit + (int)gridDim.x;
            if (!a.split || u >= a.n_seqs * units) return;
            seq = u / units;
            unit = u - seq * units;
            length = uniform(a.lengths[seq]);
            tiles_all = tiles_of(a, length);
            __syncthreads();  // the LDS that the next unit's waves write has been read
            continue;
        }
        at += x1 - x0;
        if (at >= last) return;
        __syncthreads();  // as above
        x0 = 0;
        if (++unit == units) {
            unit = 0;
            length = uniform(a.lengths[++seq]);
            tiles_all = tiles_of(a, length);
        }
    }
}

template <typename TC, bool Q16, int DC> hipError_t attn_split_launch(const AttnArgs &a, hipStream_t stream)
{
    const int64_t step = 16 / (int64_t)sizeof(TC);
    const bool pieces = a.dim % step == 0 && ((uintptr_t)a.k | (uintptr_t)a.v) % 16 == 0 &&
                        (a.k_page | a.k_slot | a.k_head | a.v_page | a.v_slot | a.v_head) % step == 0;
    AttnArgs args = a;
    const int64_t qs = Q16 ? sizeof(TC) : 4, qstep = 16 / qs;
    args.q_pieces = a.dim % step == 0 && (uintptr_t)a.q % 16 == 0 && (a.q_row | a.q_head) % qstep == 0;
    auto launch = [&](auto rows) {
        constexpr Rows R = decltype(rows)::value;
        if (a.split) hipLaunchKernelGGL((attn_split<TC, Q16, DC, R, false>), dim3(a.grid), dim3(256), 0, stream, args);
        else hipLaunchKernelGGL((attn_split<TC, Q16, DC, R, true>), dim3(a.grid), dim3(256), 0, stream, args);
    };
    if (pieces && a.dim == DC) launch(std::integral_constant<Rows, kWhole>{});
    else if (pieces) launch(std::integral_constant<Rows, kPieces>{});
    else launch(std::integral_constant<Rows, kAny>{});
    return hipGetLastError();
}

template <typename TC, bool Q16> hipError_t attn_split_by_dim(const AttnArgs &a, hipStream_t stream)
{
    if (a.dim <= 64) return attn_split_launch<TC, Q16, 64>(a, stream);
    if (a.dim <= 96) return attn_split_launch<TC, Q16, 96>(a, stream);
    if (a.dim <= 128) return attn_split_launch<TC, Q16, 128>(a, stream);
    if (a.dim <= 192) return attn_split_launch<TC, Q16, 192>(a, stream);
    return attn_split_launch<TC, Q16, 256>(a, stream);
}

// Workgroups of the class of a head size that the card holds at once.
template <typename TC, bool Q16> int attn_card_by_dim(int dim)
{
    return kAttnCus * (dim <= 64    ? AttnKernel<TC, Q16, 64, kWhole, false>::PER_CU
                       : dim <= 96  ? AttnKernel<TC, Q16, 96, kWhole, false>::PER_CU
                       : dim <= 128 ? AttnKernel<TC, Q16, 128, kWhole, false>::PER_CU
                       : dim <= 192 ? AttnKernel<TC, Q16, 192, kWhole, false>::PER_CU
                                    : AttnKernel<TC, Q16, 256, kWhole, false>::PER_CU);
}

}  // namespace
}  // namespace ilpm
