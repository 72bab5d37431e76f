// attn_tree's kernel: attention of the nodes of drafted trees over a paged
// cache, in one pass over the keys with the running maximum and sum of the
// softmax.  A key head's rows are its query heads of all nodes of a sequence.
//
// As attn_decode's (decode_attn.h) it runs both products on the matrix cores
// with keys along their rows, S[key][row] = K Q and O[d][row] = V P, so that
// probabilities stay in the lane that found them, and a wave takes keys of its
// own.  Here a wave holds several blocks of 16 rows: a tile of 16 keys is
// loaded once, and its V operands are put together once, for all of them.
//
// Which keys a row sees differs between the rows only where nodes lie, and
// where a window begins; tiles that hold neither go without a test for each
// row.  In the others a value that is not finite must not reach a row that does
// not see its key (0 times it is NaN): there such values are taken out of the
// product, and the rows that see them are marked and get NaN at the end.
//
// What bounds it.  Up to 64 rows of a key head the memory: 16 nodes of 32 / 8 bf16
// heads of 128 over 131071 keys take 120 us, 110 of them this kernel, 4.9 TB/s (a
// large copy: 4.9).  With more rows a tile's chain, score, softmax and product, of
// which two waves a SIMD cover a part: 512 rows of a key head over 65535 keys take 242 us,
// 570 TFLOP/s counting one part of each probability, two of which are multiplied.  f32
// queries over 16-bit keys are three parts for the first product.
#pragma once

#include "decode_attn.h"
#include "draft.h"

namespace ilpm {
namespace {

// The nodes that each node sees (itself and those above it), as bits; 0: no
// node.  Lane i holds node i.  Whoever is above whom is followed by doubling.
__device__ inline unsigned long long seen_nodes(int parent, int lane, int n)
{
    bool ok = lane < n && parent >= -1 && parent < lane;
    int up = ok ? parent : -1;
    unsigned lo = lane < 32 ? 1u << lane : 0, hi = lane >= 32 ? 1u << (lane - 32) : 0;
#pragma unroll 1
    for (int d = 1; d < n; d <<= 1) {
        const int from = up < 0 ? lane : up;
        const unsigned l = __shfl(lo, from), h = __shfl(hi, from);
        const int u = __shfl(up, from), k = __shfl((int)ok, from);
        lo |= l;
        hi |= h;
        ok = ok && k;
        up = up < 0 ? -1 : u;
    }
    return ok ? (unsigned long long)hi << 32 | lo : 0ull;
}

// The keys of a sequence that any of its nodes may see: the first `sinks` of
// them, and [first, end); the nodes begin at `length`.
struct TreeRange {
    int64_t length;
    int sinks, first, end;
};

__device__ inline TreeRange tree_range(const TreeArgs &t, int length)
{
    const AttnArgs &a = t.a;
    TreeRange r;
    r.length = max(length, 0);
    r.end = (int)min((int64_t)a.capacity, r.length + t.n_nodes);
    r.first = a.window > 0 ? (int)min((int64_t)r.end, max((int64_t)0, r.length + 1 - a.window)) : 0;
    r.sinks = min(t.sinks, r.first);
    if (r.sinks >= r.first - 15) r.sinks = r.first = 0;  // (they would share a tile)
    return r;
}

__device__ inline int tree_tiles(const TreeArgs &t, int length)
{
    const TreeRange r = tree_range(t, length);
    return max(1, (r.sinks + 15) / 16 + (int)(((unsigned)(r.end - r.first) + 15) / 16));
}

// N elements of a row from element d on, as load_row (decode_attn.h) takes them but
// in pieces of any alignment: kWhole and kPieces go by the head size alone.  (The
// address space is named: of a choice between a row and the zeros the compiler
// does not know it, and the loads that it takes then wait for LDS as well.)
template <typename T, int N, Rows R, bool ZERO> __device__ inline Words<sizeof(T) * N> load_piece(const T *row, int d, int dim)
{
    using W = Words<sizeof(T) * N>;
    if constexpr (R == kAny) return load_row<T, N, kAny, ZERO>(row, d, dim);
    typedef W At __attribute__((aligned(sizeof(T))));
    const T *at = R == kWhole || d < dim ? row + d : ZERO ? (const T *)&attn_zeros : row;
    return *(const __attribute__((address_space(1))) At *)(uintptr_t)at;
}

// The kernel's arguments, read anew from where they lie: kept in registers, the
// many that the loop over the tiles does not need take the place of those that it
// does (they were moved to and from lanes of vector registers in every tile).
typedef const __attribute__((address_space(4))) TreeArgs *TreeArgsAt;
__device__ inline const TreeArgs &args_of(TreeArgsAt at)
{
    asm volatile("" : "+s"(at));
    return *(const TreeArgs *)at;
}

// A head size's class, and what of AttnKernel's does not hold here.
// MA: blocks of 16 rows that a wave holds.  RS (for short sequences): the waves of a
// workgroup take a block each and all keys, in the place of all blocks and a quarter
// of the keys, and have nothing to join.
template <typename TC, bool Q16, int DC, Rows R, int MA, bool RS> struct TreeKernel : AttnKernel<TC, Q16, DC, R, false> {
    using Base = AttnKernel<TC, Q16, DC, R, false>;
    // Of the three that a wave gives to at the end, how many at once: what LDS has room for.
    static constexpr int GIVE = MA == 4 ? 2 : 3;
    // How far, in powers of two, scores may pass the reference of their row before it is
    // moved up to them, and what f16 probabilities are scaled by so that they still fit (up
    // to 2^15; a row's sum stays in 32 bits of a float's range for any length).  Outputs are
    // scaled anew in the first tiles only, not with each larger score.
    static constexpr float SLACK = __is_same(TC, _Float16) ? 4.f : 8.f;
    static constexpr float UP = __is_same(TC, _Float16) ? 0x1p11f : 1.f;
    static constexpr int WB = RS ? 4 : MA;  // blocks of rows of a workgroup
    // Whether a wave that takes rows keeps the first of their three query parts in registers: less to read, and of LDS
    // to hold (192 units of 189 rows of f32 over 130 bf16 keys, heads of 128 38.5 -> 32.5 us, of 192 62 -> 52; of 80 the
    // same, of 256 no room.  Queries in one part gain nothing by it, and lose up to a third where they take many registers).
    static constexpr bool KEEP = RS && Base::QP == 3 && DC >= 128 && DC <= 192;
    // Workgroups that a compute unit holds at once: what registers and LDS allow without spilling.
    static constexpr int PER_CU = R == kAny ? (DC >= 192 ? 1 : 2)
                                  : sizeof(TC) == 4 ? (DC >= 192 ? 1 : DC == 64 && MA == 1 ? 3 : 2)
                                  : KEEP && DC == 128 ? 3
                                  : MA == 1 ? (DC == 64 ? 4 : DC == 96 ? 3 : 2) : MA == 2 ? (DC == 64 ? 3 : DC <= 128 ? 2 : 1) : 2;
};

template <typename Cfg, int MA, bool RS> struct TreeLds {
    static constexpr int WB = Cfg::WB;
    Places places[4][2];
    FindShare found;
    // Of each row: the nodes that it sees, and the first place (a row of no node: 0 bits).
    unsigned long long bits[16 * WB];
    int low[16 * WB];
    float unscale[16 * WB];
    int top_low;  // the largest of low
    // Values of rows that are not finite for a key that not all rows see.
    int any_odd;
    unsigned odd[16 * WB][16];
    // Of each row each wave's maximum and sum.
    float m[RS ? 1 : 4][16 * MA], l[RS ? 1 : 4][16 * MA];
    union {
        // The queries, as the lanes of the first product take them, in parts those of 32 bits.
        Words16 q[Cfg::KEEP ? 2 : Cfg::QP][Cfg::NK][WB][64];
        // What each wave gives to another of its outputs, as they lie in registers.
        floatx4 give[RS ? 1 : Cfg::GIVE][RS ? 1 : 4][RS ? 1 : MA * Cfg::NO / 4][64];
    };
};

// A unit's tiles [tile0, tile1), as a workgroup takes them.
struct TreeSegment {
    int seq, kvh, block;
    int tile0, tile1;
    TreeRange range;
};

// Where row r of a segment's block lies in q, out and lse: its sequence's node and head.
__device__ inline int row_in_unit(const TreeSegment &seg, int rows_of_block, int r) { return seg.block * rows_of_block + r; }

// What a wave reads for a segment's rows: its lanes' parents, and queries as they
// lie in memory.  Wave w takes block w % WB, and of it every (4 / WB)-th piece.
template <typename TC, bool Q16, int DC, Rows R, int MA, bool RS> struct TreeRows {
    using Cfg = TreeKernel<TC, Q16, DC, R, MA, RS>;
    using TQ = std::conditional_t<Q16, TC, float>;
    static constexpr int KV = Cfg::KV, NK = Cfg::NK, QP = Cfg::QP, WB = Cfg::WB, STEP = 4 / WB, MINE = (NK + STEP - 1) / STEP;
    int parent;
    const TQ *row;
    Words16 q[QP == 1 ? MINE : 1];

    __device__ __forceinline__ void load(TreeArgsAt args, const TreeSegment &seg, int lane, int wave)
    {
        const TreeArgs &t = args_of(args);
        const AttnArgs &a = t.a;
        const int n16 = lane & 15, g = lane >> 4, ma = wave % WB, c0 = wave / WB;
        parent = lane < t.n_nodes ? t.parents[(int64_t)seg.seq * t.n_nodes + lane] : -2;
        const int in_unit = min(row_in_unit(seg, 16 * WB, ma * 16 + n16), t.rows - 1), node = t.by_group.of(in_unit);
        row = (const TQ *)a.q + ((int64_t)seg.seq * t.n_nodes + node) * a.q_row +
              ((int64_t)seg.kvh * a.group + (in_unit - node * a.group)) * a.q_head;
        if constexpr (QP == 1) {
#pragma unroll
            for (int i = 0; i < MINE; ++i) q[i] = load_piece<TQ, KV, R, true>(row, (g + 4 * min(c0 + i * STEP, NK - 1)) * KV, a.dim);
        }
    }

    // Rows' bits and lows, and the queries in their layout, into LDS or `kept`.
    template <typename Lds> __device__ __forceinline__ void store(TreeArgsAt args, const TreeSegment &seg, int lane, int wave, Lds &lds, Words16 *kept)
    {
        const TreeArgs &t = args_of(args);
        const AttnArgs &a = t.a;
        const int ma = wave % WB, c0 = RS ? 0 : wave / WB;
        for (int i = threadIdx.x; i < 16 * WB * 16; i += 256) lds.odd[i / 16][i % 16] = 0;
        if (threadIdx.x == 0) lds.any_odd = 0;
        if constexpr (QP == 1) {
#pragma unroll
            for (int i = 0; i < MINE; ++i) lds.q[0][min(c0 + i * STEP, NK - 1)][ma][lane] = q[i];
        } else {
            split(t, lane, ma, c0, lds, kept);
        }
        if (wave != 0) return;
        unsigned long long bits = seen_nodes(parent, lane, t.n_nodes);
        const int depth = __builtin_popcountll(bits) - 1;
        int low = 0;
        if (a.window > 0) {
            const unsigned long long above = bits;
#pragma unroll 1
            for (int n = 0; n < t.n_nodes; ++n) {
                const int dn = __builtin_amdgcn_readlane(depth, n);
                if (((above >> n) & 1) && depth - dn >= a.window && seg.range.length + dn >= t.sinks) bits &= ~(1ull << n);
            }
            low = (int)min((int64_t)INT_MAX, max((int64_t)0, seg.range.length + depth + 1 - a.window));
        }
        int top = low;
        if (a.window > 0)
#pragma unroll 1
            for (int d = 32; d > 0; d >>= 1) top = max(top, __shfl_xor(top, d));
        if (lane == 0) lds.top_low = top;
        static_assert(16 * WB <= 64, "a lane for each row");
        const int r = min(lane, 16 * WB - 1), in_block = row_in_unit(seg, 16 * WB, r), node = min(t.by_group.of(in_block), t.n_nodes - 1);
        const unsigned b0 = __shfl((unsigned)bits, node), b1 = __shfl((unsigned)(bits >> 32), node);
        const int l = __shfl(low, node);
        lds.bits[r] = in_block < t.rows ? (unsigned long long)b1 << 32 | b0 : 0ull;
        lds.low[r] = l;
    }

    // Queries of 32 bits in three parts (see decode_attn.h).
    template <typename Lds> __device__ __forceinline__ void split(const TreeArgs &t, int lane, int ma, int c0, Lds &lds, Words16 *kept)
    {
        const int n16 = lane & 15, g = lane >> 4, dim = t.a.dim;
        struct Values {
            float v[KV];
        };
        auto get = [&](int c) {  // KV = 8 values: two pieces of four
            struct Halves {
                Words16 w[2];
            } h;
#pragma unroll
            for (int n = 0; n < 2; ++n) h.w[n] = load_piece<float, 4, R, true>(row, (g + 4 * c) * KV + 4 * n, dim);
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
        if (c0 == 0 && g == 0) lds.unscale[ma * 16 + n16] = back;
        constexpr int ROLL = Cfg::KEEP ? NK : 2;
#pragma unroll ROLL
        for (int c = c0; c < NK; c += STEP) {
            const Values p = get(c);
            Pack<TC, KV> part[3];
#pragma unroll
            for (int i = 0; i < KV; ++i) {
                float v = p.v[i] * f;
                if constexpr (__is_same(TC, __bf16)) {
                    // (Cut off, not rounded: see decode_attn.h.)
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
            for (int n = 0; n < 3; ++n) {
                const Words16 w = __builtin_bit_cast(Words16, part[n]);
                if (Cfg::KEEP && n == 0) kept[Cfg::KEEP ? c : 0] = w;
                else lds.q[Cfg::KEEP ? n - 1 : n][c][ma][lane] = w;
            }
        }
    }
};

template <typename TC> __device__ inline floatx4 mfma_values32(Words16 v, Words16 p, floatx4 c) { return mfma_scores<TC>(v, p, c); }

// Of a word of two 16-bit values, ones in the places of those that are not finite.
template <typename TC> __device__ inline unsigned not_finite(unsigned w)
{
    constexpr unsigned E = __is_same(TC, __bf16) ? 0x7f80u : 0x7c00u;
    return ((w & E) == E ? 0xffffu : 0u) | ((w & (E << 16)) == (E << 16) ? 0xffff0000u : 0u);
}

// Joins the four waves' parts of all rows, and puts them out.
template <typename Cfg, int MA, typename Lds, typename Put>
__device__ __forceinline__ void tree_join(TreeArgsAt args, const TreeSegment &seg, Lds &lds, floatx4 (&o)[MA][Cfg::NO], float (&m)[MA],
                                          float (&l)[MA], int wave, int n16, int g, int lane, Put put)
{
    constexpr int NO = Cfg::NO, VV = Cfg::VV;
    // Join the waves.  Lane (n, g) holds values (4g + r + 16c) * VV + i of row n; what is no
    // node has seen keys of the sequence, and none counts.
#pragma unroll
    for (int ma = 0; ma < MA; ++ma) {
        l[ma] += __shfl_xor(l[ma], 16);
        l[ma] += __shfl_xor(l[ma], 32);
        if (g == 0) {
            const bool real = lds.bits[ma * 16 + n16] != 0;
            lds.m[wave][ma * 16 + n16] = real ? m[ma] : -INFINITY;
            lds.l[wave][ma * 16 + n16] = real ? l[ma] : 0.f;
        }
    }
    __syncthreads();  // the queries have been read; all odd values are marked
    // A quarter of the values of all rows to each wave, of one block of rows: the others give it theirs.
    constexpr int QUARTER = MA * NO / 4;
    const int my_block = wave * MA / 4;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int ma = 0; ma < MA; ++ma) {
        float mw[4], most = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mw[w] = lds.m[w][ma * 16 + n16];
            most = fmaxf(most, mw[w]);
        }
        const float base = most == -INFINITY ? 0.f : most;
        const bool real = lds.bits[ma * 16 + n16] != 0;
        const float f = real ? __builtin_amdgcn_exp2f(m[ma] - base) : 0.f;
        if (ma == my_block) {
            top = most;
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += lds.l[w][ma * 16 + n16] * __builtin_amdgcn_exp2f(mw[w] - base);
        }
#pragma unroll
        for (int i = 0; i < NO; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[ma][i][r] = real ? o[ma][i][r] * f : 0.f;
    }
    if (lds.any_odd) {
#pragma unroll
        for (int ma = 0; ma < MA; ++ma)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const unsigned odd = lds.odd[ma * 16 + n16][4 * g + r];
#pragma unroll
                for (int i = 0; i < NO; ++i) o[ma][i][r] = (odd >> i) & 1 ? __builtin_nanf("") : o[ma][i][r];
            }
    }
    floatx4 mine[QUARTER];
    // Each wave's quarter by numbers known at compile time.  (The barriers differ so that the four stay four: made one,
    // with a number found at run time, it would put all outputs into memory, from the loop over the tiles on.)
    auto quarter = [&](int w, auto f) {
        auto one = [&](auto number) {
            constexpr int k = decltype(number)::value;
            if (w != k) return;
#pragma unroll
            for (int i = 0; i < QUARTER; ++i) f(i, o[(k * QUARTER + i) / NO][(k * QUARTER + i) % NO]);
            __builtin_amdgcn_sched_barrier(k);
        };
        one(std::integral_constant<int, 0>{});
        one(std::integral_constant<int, 1>{});
        one(std::integral_constant<int, 2>{});
        one(std::integral_constant<int, 3>{});
    };
    quarter(wave, [&](int i, const floatx4 &v) { mine[i] = v; });
    if constexpr (Cfg::GIVE == 3) {
#pragma unroll
        for (int step = 1; step < 4; ++step)
            quarter((wave + step) & 3, [&](int i, const floatx4 &v) { lds.give[step - 1][wave][i][lane] = v; });
        __syncthreads();
#pragma unroll
        for (int step = 1; step < 4; ++step)
#pragma unroll
            for (int i = 0; i < QUARTER; ++i) mine[i] += lds.give[step - 1][(wave - step) & 3][i][lane];
    } else {
        // (What a step reads the one after the next writes, behind the next one's barrier.)
#pragma unroll 1
        for (int step = 1; step < 4; ++step) {
            quarter((wave + step) & 3, [&](int i, const floatx4 &v) { lds.give[step & 1][wave][i][lane] = v; });
            __syncthreads();
#pragma unroll
            for (int i = 0; i < QUARTER; ++i) mine[i] += lds.give[step & 1][(wave - step) & 3][i][lane];
        }
    }
    const int r_block = my_block * 16 + n16, first = wave * QUARTER % NO;
    if (row_in_unit(seg, 16 * MA, r_block) >= args_of(args).rows) return;
    constexpr int POW = QUARTER & -QUARTER, RUN = POW < VV ? POW : VV;  // values that lie together
    put(args_of(args), row_in_unit(seg, 16 * MA, r_block), r_block, top, sum, first == 0 && g == 0, [&](auto &&give) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < QUARTER; k += RUN) {
                Pack<float, RUN> p;
#pragma unroll
                for (int i = 0; i < RUN; ++i) p.v[i] = mine[k + i][r];
                const int c = (first + k) / VV, i = (first + k) % VV;
                give((4 * g + r + 16 * c) * VV + i, p);
            }
    });
}

// A wave's part of a segment, every fourth tile of it, and the join of the
// four waves' parts; or (RS) all tiles for a block of rows.
template <typename TC, bool Q16, int DC, Rows R, int MA, bool RS, typename Put>
__device__ __forceinline__ void tree_segment(TreeArgsAt args, const TreeSegment &seg, TreeLds<TreeKernel<TC, Q16, DC, R, MA, RS>, MA, RS> &lds, Put put)
{
    using Cfg = TreeKernel<TC, Q16, DC, R, MA, RS>;
    constexpr int KV = Cfg::KV, NK = Cfg::NK, VV = Cfg::VV, NV = Cfg::NV, NO = Cfg::NO;
    constexpr int QP = Cfg::QP, PP = Cfg::PP;
    constexpr bool C16 = Cfg::C16;
    constexpr int AHEAD = std::min(C16 ? 4 : 2, NK * QP * MA);  // query operands that are read before the one in use

    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int wave = uniform((int)(threadIdx.x >> 6));
    const int n16 = lane & 15, g = lane >> 4;
    const int seq = seg.seq;
    const TreeRange range = seg.range;
    const int sink_tiles = (range.sinks + 15) / 16;
    // Tile j of this wave is tile 4j + wave (RS: j) of the segment.
    constexpr int EVERY = RS ? 1 : 4, WB = Cfg::WB;
    const int tile_of = seg.tile0 + (RS ? 0 : wave);
    int tiles = max(0, (seg.tile1 - tile_of + EVERY - 1) / EVERY);
    auto block = [&](int ma) { return RS ? wave : ma; };  // of the workgroup's
    auto start_of = [&](int tile) { return tile < sink_tiles ? tile * 16 : range.first + (tile - sink_tiles) * 16; };

    // Lane (n, g) looks up key n of tile 4*group + g.
    struct Entry {
        int page, slot;
    };
    auto look_up = [&](int group) {
        const AttnArgs &a = args_of(args).a;
        Entry e = {-1, 0};
        const int tile = tile_of + (group * 4 + g) * EVERY;
        const int64_t key = (int64_t)start_of(tile) + n16;
        if (tile < seg.tile1 && key < (tile < sink_tiles ? range.sinks : range.end)) {
            const int p = (int)key / a.page_size;
            e.slot = (int)key - p * a.page_size;
            e.page = a.table[(int64_t)seq * a.table_stride + p];
            if (a.mask && (key >= a.mask_len || !a.mask[(int64_t)seq * a.mask_stride + key])) e.page = -1;
        }
        return e;
    };
    // Where a group's keys lie, in LDS (those that are not seen at the pool's first row: it is read, and none of it
    // used), and which are seen: bit 16t + n is key n of its tile t.
    unsigned long long seen_of[2] = {0, 0};
    auto place = [&](int group, Entry e) {
        const AttnArgs &a = args_of(args).a;
        const bool ok = e.page >= 0 && e.page < a.n_pages;
        Places &p = lds.places[wave][group & 1];
        p.k[lane] = ok ? (int64_t)e.page * a.k_page + (int64_t)e.slot * a.k_slot : 0;
        p.v[lane] = ok ? (int64_t)e.page * a.v_page + (int64_t)e.slot * a.v_slot : 0;
        const unsigned long long seen = __builtin_amdgcn_ballot_w64(ok);
        if (group & 1) seen_of[1] = seen;
        else seen_of[0] = seen;
        // (Only this wave reads them, and a wave's LDS accesses keep their order.)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const TreeArgs &t = args_of(args);
    const AttnArgs &a = t.a;
    const TC *kh = (const TC *)a.k + (int64_t)seg.kvh * a.k_head;
    const TC *vh = (const TC *)a.v + (int64_t)seg.kvh * a.v_head;
    const int dim = a.dim, all_sinks = t.sinks;
    const float softcap = a.softcap;
    Words16 kt[NK];
    Words<sizeof(TC) * VV> vt[4][NV];
    // (Behind the last tile that one again.)
    auto load_k = [&](int j) {
        j = min(j, tiles - 1);
        const TC *row = kh + lds.places[wave][(j >> 2) & 1].k[(j & 3) * 16 + n16];
#pragma unroll
        for (int c = 0; c < NK; ++c) kt[c] = load_piece<TC, KV, R, true>(row, (g + 4 * c) * KV, dim);
    };
    auto load_v = [&](int j) {
        j = min(j, tiles - 1);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const TC *row = vh + lds.places[wave][(j >> 2) & 1].v[(j & 3) * 16 + 4 * g + r];
#pragma unroll
            for (int c = 0; c < NV; ++c)  // (sixteen lanes may reach beyond a whole row)
                vt[r][c] = load_piece<TC, VV, R == kWhole && Cfg::DO != DC ? kPieces : R, false>(row, (n16 + 16 * c) * VV, dim);
        }
    };

    Entry e0 = {}, next = {};
    if (tiles > 0) e0 = look_up(0);
    if (tiles > 4) next = look_up(1);
    // The first tile, the rows' nodes and queries: none waits for another.
    TreeRows<TC, Q16, DC, R, MA, RS> rows;
    rows.load(args, seg, lane, wave);
    // (Behind the last node of a smaller tree there is nothing to do.)
    const unsigned long long nodes = __builtin_amdgcn_ballot_w64(rows.parent >= -1 && rows.parent < lane);
    if (row_in_unit(seg, 16 * WB, RS ? wave * 16 : 0) >= (64 - (nodes ? __builtin_clzll(nodes) : 64)) * a.group) tiles = 0;
    if (tiles > 0) {
        place(0, e0);
        load_k(0);
        load_v(0);
    }
    Words16 kept[Cfg::KEEP ? NK : 1];
    rows.store(args, seg, lane, wave, lds, kept);
    __syncthreads();

    floatx4 o[MA][NO];
    float m[MA], l[MA];
#pragma unroll
    for (int ma = 0; ma < MA; ++ma) {
        m[ma] = -INFINITY;
        l[ma] = 0.f;
#pragma unroll
        for (int i = 0; i < NO; ++i) o[ma][i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = softcap > 0.f ? a.scale / softcap : a.scale * kLog2e;
    const float cap2 = softcap * kLog2e;
    const int top_low = uniform(lds.top_low);
    constexpr bool UNSCALE = QP == 3 && __is_same(TC, _Float16);  // (parts of bf16 need none)
    // With a cap, or a scale that is not above 0, scores are scaled before their maximum is taken; and where a row's
    // scale is 0 or infinite only together with that of its parts (queries near either end of a float): such a product
    // of a score that is 0, or of -infinity for a key that is not seen, would be NaN.
    bool apart = softcap > 0.f || !(scale2 > 0.f);
    if constexpr (UNSCALE) {
#pragma unroll
        for (int ma = 0; ma < MA; ++ma) {
            const float by = scale2 * lds.unscale[block(ma) * 16 + n16];
            apart = apart || __builtin_amdgcn_ballot_w64(!(by > 0.f && by < INFINITY)) != 0;
        }
    }

    // Value i of piece c of a lane's four rows, put together from their 16-bit halves.
    auto values = [&](int c, int i) {
        const unsigned halves = i & 1 ? 0x07060302u : 0x05040100u;
        return Words<8>{__builtin_amdgcn_perm(vt[1][c][i / 2], vt[0][c][i / 2], halves), __builtin_amdgcn_perm(vt[3][c][i / 2], vt[2][c][i / 2], halves)};
    };
    // Which of the keys key0..key0 + 15 row r sees, where they are in the cache (what is no node none: no value that is
    // not finite may mark it).
    auto sees = [&](int r, int64_t key0) {
        auto upto = [](int64_t n) { return n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << (int)n) - 1u; };  // the first n keys
        const unsigned long long bits = lds.bits[r];
        const int64_t node0 = key0 - range.length;
        const unsigned nodes = (unsigned)(node0 >= 0 ? node0 < 64 ? bits >> (int)node0 : 0 : node0 > -16 ? bits << (int)-node0 : 0);
        const unsigned before = bits ? upto(-node0) : 0;  // the sequence's own
        return (nodes & ~before & 0xffffu) | (before & (~upto(lds.low[r] - key0) | upto(all_sinks - key0)));
    };
    // Takes values that are not finite out of a tile whose rows do not see the same keys, and marks the rows that see
    // them: bit c * VV + i of odd[row][n] stands for value (n + 16c) * VV + i.  (Hardly ever.)
    auto take_out = [&](int64_t key0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            unsigned odd = 0;
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                if constexpr (C16) {
#pragma unroll
                    for (int i = 0; i < VV / 2; ++i) {
                        const unsigned w = not_finite<TC>(vt[r][c][i]);
                        vt[r][c][i] &= ~w;
                        odd |= (w & 1u) << (c * VV + 2 * i) | (w >> 31) << (c * VV + 2 * i + 1);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < VV; ++i) {
                        const bool is = (vt[r][c][i] & 0x7f800000u) == 0x7f800000u;
                        vt[r][c][i] = is ? 0u : vt[r][c][i];
                        odd |= (is ? 1u : 0u) << (c * VV + i);
                    }
                }
            }
            if (odd == 0) continue;
            lds.any_odd = 1;
#pragma unroll 1
            for (int row = block(0) * 16; row < block(0) * 16 + 16 * MA; ++row)
                if ((sees(row, key0) >> (4 * g + r)) & 1) atomicOr(&lds.odd[row][n16], odd);
        }
    };

#pragma unroll 1
    for (int j = 0; j < tiles; ++j) {
        if ((j & 3) == 2 && j + 2 < tiles) {
            place(j / 4 + 1, next);
            if (j + 6 < tiles) next = look_up(j / 4 + 2);
        }
        const int tile = tile_of + j * EVERY;
        const int64_t key0 = start_of(tile);
        const bool special = key0 + 15 >= range.length || (tile >= sink_tiles && key0 < top_low);

        // The scores of the blocks of rows, then the next tile's keys are on their way.
        floatx4 s[MA];
        int ql = lane;
        asm volatile("" : "+v"(ql));  // (read for each tile, not kept)
        auto query = [&](int n, int c, int ma) {
            return Cfg::KEEP && n == 0 ? kept[Cfg::KEEP ? c : 0] : lds.q[Cfg::KEEP ? n - 1 : n][c][block(ma)][ql];
        };
#pragma unroll
        for (int ma = 0; ma < MA; ++ma) s[ma] = floatx4{0.f, 0.f, 0.f, 0.f};
        floatx4 low[MA];
#pragma unroll
        for (int ma = 0; ma < MA; ++ma) low[ma] = s[ma];
        // (Reads ahead, held in their places: the compiler, short of registers, waits for each.  8 trees of 1024 rows of f32
        // over up to 2049 bf16 keys of 256 73 -> 56 us, 64 such rows of 128 over 131071 keys 151 -> 136; as fast with 2,
        // 6 or, where registers last, 10 ahead of 4.)
        constexpr int ALL = NK * QP * MA;
        Words16 got[AHEAD + 1];
        auto read = [&](int i) { got[i % (AHEAD + 1)] = query(i / MA % QP, i / (MA * QP), i % MA); };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
        for (int i = 0; i < ALL; ++i) {
            if (i + AHEAD < ALL) read(i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
            floatx4 &x = i / MA % QP == 0 ? s[i % MA] : low[i % MA];
            const Words16 k = kt[i / (MA * QP)], q = got[i % (AHEAD + 1)];
            if constexpr (C16) {
                x = mfma_scores<TC>(k, q, x);
            } else {
#pragma unroll
                for (int e = 0; e < KV; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(floatx4, k)[e], __builtin_bit_cast(floatx4, q)[e], x, 0, 0, 0);
            }
        }
        if constexpr (QP == 3) {
#pragma unroll
            for (int ma = 0; ma < MA; ++ma)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[ma][r] += low[ma][r] - low[ma][r] == 0.f ? low[ma][r] : 0.f;
        }
        load_k(j + 1);

        // Scores times `by` are logarithms to the base 2; where that product would not do, they are first made so.
        float by[MA];
#pragma unroll
        for (int ma = 0; ma < MA; ++ma) by[ma] = UNSCALE ? scale2 * lds.unscale[block(ma) * 16 + n16] : scale2;
        if (apart) {
#pragma unroll
            for (int ma = 0; ma < MA; ++ma) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (UNSCALE) s[ma][r] *= lds.unscale[block(ma) * 16 + n16];
                    s[ma][r] *= scale2;
                    if (softcap > 0.f) s[ma][r] = cap2 * tanh_of(s[ma][r]);
                }
                by[ma] = 1.f;
            }
        }
        // Most tiles are seen whole by all rows.
        const unsigned tile_seen = (unsigned)((j & 4 ? seen_of[1] : seen_of[0]) >> ((j & 3) * 16)) & 0xffffu;
        if (special || tile_seen != 0xffffu) {
            bool seen[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) seen[r] = ((tile_seen >> (4 * g + r)) & 1) != 0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < NV; ++c) {
                    using V = std::remove_reference_t<decltype(vt[r][c])>;
                    vt[r][c] = seen[r] ? vt[r][c] : V{};
                }
            if (special) take_out(key0);
#pragma unroll
            for (int ma = 0; ma < MA; ++ma) {
                const unsigned see = (special ? sees(block(ma) * 16 + n16, key0) & tile_seen : tile_seen) >> (4 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[ma][r] = (see >> r) & 1 ? s[ma][r] : -INFINITY;
            }
        }
        constexpr int PW = !C16 ? 4 : PP == 3 ? 6 : 4;
        unsigned part[MA][PW];  // probabilities: hi and lo of four keys, a third part; or 32 bits
#pragma unroll
        for (int ma = 0; ma < MA; ++ma) {
            const float top = fmaxf(fmaxf(s[ma][0], s[ma][1]), fmaxf(s[ma][2], s[ma][3])) * by[ma];
            // (m may lie up to SLACK below the maximum: most tiles after the first leave it where it is.)
            if (__builtin_amdgcn_ballot_w64(top > m[ma] + Cfg::SLACK)) {
                const float m_new = fmaxf(m[ma], max_of_head(top));
                const float alpha = __builtin_amdgcn_exp2f(m[ma] - (m_new == -INFINITY ? 0.f : m_new));
                m[ma] = m_new;
                l[ma] *= alpha;
#pragma unroll
                for (int i = 0; i < NO; ++i) o[ma][i] *= alpha;
            }
            const float base = m[ma] == -INFINITY ? 0.f : m[ma];
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ma][r], by[ma], -base));
            l[ma] += (x[0] + x[1]) + (x[2] + x[3]);
            if constexpr (!C16) {
#pragma unroll
                for (int r = 0; r < 4; ++r) part[ma][r] = __builtin_bit_cast(unsigned, x[r]);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] *= Cfg::UP;
                    if constexpr (Cfg::UP != 1.f) asm("" : "+v"(x[r]));  // (one product, not one for each of its uses)
                }
#pragma unroll
                for (int i = 0; i < PP; ++i) {
                    Pack<TC, 4> h;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        h.v[r] = (TC)x[r];
                        x[r] -= (float)h.v[r];
                    }
                    const Words<8> w = __builtin_bit_cast(Words<8>, h);
                    part[ma][2 * i] = w[0];
                    part[ma][2 * i + 1] = w[1];
                }
            }
        }

        // The same four keys twice, against the first and second parts of their probabilities.
        auto weigh = [&](int ma, int i, Words16 vv) {
            floatx4 &sum = o[ma][i];
            sum = mfma_values32<TC>(vv, Words16{part[ma][0], part[ma][1], part[ma][2], part[ma][3]}, sum);
            // (By the same instruction: one of 16x16x16 right after it, on the same registers, found them as they were
            // before it.)
            if constexpr (PP == 3) sum = mfma_values32<TC>(vv, Words16{part[ma][4], part[ma][5], 0u, 0u}, sum);
        };
        if constexpr (!C16) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int i = 0; i < VV; ++i) {
                        const float v = __builtin_bit_cast(floatx4, vt[r][c])[i];
#pragma unroll
                        for (int ma = 0; ma < MA; ++ma) {
                            o[ma][c * VV + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, __builtin_bit_cast(float, part[ma][r]), o[ma][c * VV + i], 0, 0, 0);
                        }
                    }
        } else {
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < VV; ++i) {
                    const Words<8> v = values(c, i);
#pragma unroll
                    for (int ma = 0; ma < MA; ++ma) weigh(ma, c * VV + i, Words16{v[0], v[1], v[0], v[1]});
                }
        }
        load_v(j + 1);
    }

    if constexpr (RS) {
        l[0] += __shfl_xor(l[0], 16);
        l[0] += __shfl_xor(l[0], 32);
        const int r = wave * 16 + n16;
        if (row_in_unit(seg, 16 * WB, r) >= args_of(args).rows) return;
        const bool real = lds.bits[r] != 0;  // (what is no node has seen keys of the sequence, and none counts)
        // (Only this wave marked its rows, each lane for others.)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        unsigned odd[4] = {0, 0, 0, 0};
        if (lds.any_odd) {
#pragma unroll
            for (int i = 0; i < 4; ++i) odd[i] = lds.odd[r][4 * g + i];
        }
        put(args_of(args), row_in_unit(seg, 16 * WB, r), r, real ? m[0] : -INFINITY, real ? l[0] : 0.f, g == 0, [&](auto &&give) {
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    Pack<float, VV> p;
#pragma unroll
                    for (int i = 0; i < VV; ++i)
                        p.v[i] = !real ? 0.f : (odd[k] >> (c * VV + i)) & 1 ? __builtin_nanf("") : o[0][c * VV + i][k];
                    give((4 * g + k + 16 * c) * VV, p);
                }
        });
    } else {
        tree_join<Cfg, MA>(args, seg, lds, o, m, l, wave, n16, g, lane, put);
    }
}

template <typename TC, bool Q16, int DC, Rows R, int MA, bool RS>
__global__ __launch_bounds__(256, (TreeKernel<TC, Q16, DC, R, MA, RS>::PER_CU)) void tree_split(TreeArgs)
{
    using Cfg = TreeKernel<TC, Q16, DC, R, MA, RS>;
    const int unit_cost = tree_unit_cost(MA);
    using TQ = std::conditional_t<Q16, TC, float>;
    __shared__ TreeLds<Cfg, MA, RS> lds;
    const TreeArgsAt args = (TreeArgsAt)__builtin_amdgcn_kernarg_segment_ptr();
    const TreeArgs &t = args_of(args);
    const AttnArgs &a = t.a;

    // (Neighbours stay on one die: see decode_attn.h.)  The blocks of a share's rows are
    // neighbours and take its keys at the same time, so that their die's cache has them
    // for all but the first.
    const int die = blockIdx.x & 7, dies = gridDim.x >> 3;
    const int units = a.kv_heads, wg = die * dies + min(die, (int)(gridDim.x & 7)) + (int)(blockIdx.x >> 3);
    const int share_at = wg / a.blocks, block = wg - share_at * a.blocks, shares = (int)gridDim.x / a.blocks;
    Share share = {0, 0, true};
    Begin begin;
    if constexpr (!RS)
        if (a.split) share = find_share(a, share_at, shares, units, lds.found, &begin, [&](int n) { return tree_tiles(t, n); }, unit_cost);

    // This workgroup's place: a sequence, its length and its units' tiles, a unit
    // of it, and how far into the unit's length the share has come.
    int seq, length, unit, tiles_all, x0 = 0;
    int at = 0, last = 0;
    if (!RS && a.split && !a.part_of_unit && block == 0 && threadIdx.x == 0) a.parts[share_at] = AttnPart{0, 0, 0, 0};  // (whatever follows, the join reads it)
    if (share.whole) {
        if (share_at >= a.n_seqs * units) return;
        seq = share_at / units;
        unit = share_at - seq * units;
        length = uniform(a.lengths[seq]);
        tiles_all = tree_tiles(t, length);
    } else {
        if ((int64_t)share_at * share.size >= share.total) return;
        at = share_at * share.size;
        last = (int)min((int64_t)at + share.size, (int64_t)share.total);
        seq = begin.seq;
        length = begin.length;
        tiles_all = tree_tiles(t, length);
        const int in = at - begin.before;
        unit = in / (tiles_all + unit_cost);
        x0 = in - unit * (tiles_all + unit_cost);
    }

    const bool split = !RS && a.split, part_of_unit = a.part_of_unit;
    const int n_seqs = a.n_seqs;
    for (;;) {
        const int x1 = share.whole ? tiles_all + unit_cost : min(tiles_all + unit_cost, x0 + (last - at));
        const int tile0 = max(0, x0 - unit_cost), seg_tiles = max(0, x1 - unit_cost) - tile0;
        if (seg_tiles == 0) return;  // the share ends before the unit's first tile
        TreeSegment seg;
        seg.seq = seq;
        seg.kvh = unit;
        seg.block = block;
        seg.tile0 = tile0;
        seg.tile1 = tile0 + seg_tiles;
        seg.range = tree_range(args_of(args), length);
        if (seg.range.end == 0) seg.tile1 = tile0;  // (no keys, and perhaps no pool)
        const bool all = seg_tiles == tiles_all;  // of the unit's tiles
        // Row `row` of the unit, r of its block: its maximum and sum, and its values, in packs, from `each`.
        tree_segment<TC, Q16, DC, R, MA, RS>(args, seg, lds, [&](const TreeArgs &t, int row, int r, float top, float sum, bool lead, auto each) {
            const AttnArgs &a = t.a;
            auto put = [&](auto *to, float by) {
                each([&](int d, auto p) {
                    constexpr int N = sizeof(p.v) / sizeof(float);
                    using TO = std::remove_reference_t<decltype(*to)>;
                    Pack<TO, N> q;
#pragma unroll
                    for (int k = 0; k < N; ++k) q.v[k] = (TO)(p.v[k] * by);
                    if (d + N <= a.dim) {
                        store_loose<TO, N>(to + d, q);
                        return;
                    }
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (d + k < a.dim) to[d + k] = q.v[k];
                });
            };
            if (all) {
                const int node = t.by_group.of(row), head = seg.kvh * a.group + (row - node * a.group);
                const int64_t at_row = (int64_t)seg.seq * t.n_nodes + node;
                put((TQ *)a.out + at_row * a.o_row + (int64_t)head * a.o_head, sum == 0.f ? 0.f : 1.f / (sum * Cfg::UP));
                if (lead && a.lse) a.lse[at_row * a.q_heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
            } else {
                // The part that begins a unit, or the one that goes on with it.
                const int64_t part = ((int64_t)wg * 2 + (seg.tile0 == 0 ? 1 : 0)) * a.part_heads + r;
                put(a.part_o + part * a.dim, 1.f / Cfg::UP);
                if (lead) {
                    a.part_ml[part * 2] = top;
                    a.part_ml[part * 2 + 1] = sum;
                }
            }
        });
        if (RS) return;
        const AttnArgs &a = args_of(args).a;
        // Who begins a unit says whether others go on with it.
        if (split && block == 0 && threadIdx.x == 0 && tile0 == 0) {
            const int rest = tiles_all - seg_tiles;
            const int count = all ? 0 : 1 + (int)(((unsigned)rest + share.size - 1) / (unsigned)share.size);
            if (part_of_unit) a.parts[seq * units + unit] = AttnPart{seq, unit, share_at, count};
            else if (!all) a.parts[share_at] = AttnPart{seq, unit, share_at, count};
        }
        __syncthreads();  // the LDS that the next unit's waves write has been read
        if (share.whole) {
            const int u = seq * units + unit + shares;
            if (!split || u >= n_seqs * units) return;
            seq = u / units;
            unit = u - seq * units;
        } else {
            at += x1 - x0;
            if (at >= last) return;
            x0 = 0;
            if (++unit < units) continue;
            unit = 0;
            ++seq;
        }
        length = uniform(a.lengths[seq]);
        tiles_all = tree_tiles(args_of(args), length);
    }
}

// The largest number of row blocks of a workgroup for a class: what leaves two waves a
// SIMD, or from heads of 192 on one that takes two blocks, which is faster than two of one
// block (4 x 32000 bf16 keys of 4 heads of 256, 64 rows of each, 108 us and not 120).
template <typename TC, int DC> constexpr int kMostBlocks = sizeof(TC) == 4 ? (DC <= 128 ? 2 : 1) : DC <= 128 ? 4 : 2;

template <typename TC, bool Q16, int DC> hipError_t tree_split_launch(const TreeArgs &t, hipStream_t stream)
{
    constexpr int MOST = kMostBlocks<TC, DC>;
    auto launch = [&](auto rows, auto blocks) {
        hipLaunchKernelGGL((tree_split<TC, Q16, DC, decltype(rows)::value, decltype(blocks)::value, false>), dim3(t.a.grid), dim3(256), 0, stream, t);
        return hipGetLastError();
    };
    auto by_blocks = [&](auto rows) {
        if (t.by_rows) {
            hipLaunchKernelGGL((tree_split<TC, Q16, DC, decltype(rows)::value, 1, true>), dim3(t.a.grid), dim3(256), 0, stream, t);
            return hipGetLastError();
        }
        if constexpr (MOST >= 4)
            if (t.row_blocks == 4) return launch(rows, std::integral_constant<int, 4>{});
        if constexpr (MOST >= 2)
            if (t.row_blocks == 2) return launch(rows, std::integral_constant<int, 2>{});
        return launch(rows, std::integral_constant<int, 1>{});
    };
    if (t.a.dim == DC) return by_blocks(std::integral_constant<Rows, kWhole>{});
    if (t.pieces) return by_blocks(std::integral_constant<Rows, kPieces>{});
    return launch(std::integral_constant<Rows, kAny>{}, std::integral_constant<int, 1>{});
}

// Of a head size's class: the most row blocks of a workgroup, and the
// workgroups that the card holds at once.
template <typename TC, bool Q16, typename F> auto tree_by_class(int dim, F f)
{
    if (dim <= 64) return f(std::integral_constant<int, 64>{});
    if (dim <= 96) return f(std::integral_constant<int, 96>{});
    if (dim <= 128) return f(std::integral_constant<int, 128>{});
    if (dim <= 192) return f(std::integral_constant<int, 192>{});
    return f(std::integral_constant<int, 256>{});
}
template <typename TC, bool Q16> hipError_t tree_split_by_dim(const TreeArgs &t, hipStream_t stream)
{
    return tree_by_class<TC, Q16>(t.a.dim, [&](auto dc) { return tree_split_launch<TC, Q16, decltype(dc)::value>(t, stream); });
}
template <typename TC, bool Q16> int tree_most_by_dim(int dim)
{
    return tree_by_class<TC, Q16>(dim, [](auto dc) { return kMostBlocks<TC, decltype(dc)::value>; });
}
template <typename TC, bool Q16> int tree_card_by_dim(int dim, bool pieces, int blocks)
{
    return kAttnCus * tree_by_class<TC, Q16>(dim, [&](auto dc) {
        constexpr int DC = decltype(dc)::value;
        if (!pieces) return TreeKernel<TC, Q16, DC, kAny, 1, false>::PER_CU;
        return blocks == 4 ? TreeKernel<TC, Q16, DC, kPieces, 4, false>::PER_CU
               : blocks == 2 ? TreeKernel<TC, Q16, DC, kPieces, 2, false>::PER_CU : TreeKernel<TC, Q16, DC, kPieces, 1, false>::PER_CU;
    });
}

}  // namespace
}  // namespace ilpm
