// verify_drafts: which nodes of a tree of drafted tokens are kept, and the next
// token, from the target's probabilities and given random numbers.
//
// The walk from the root needs a few values of the rows only; a whole row is read
// where it ends, to draw from what is left of it.  With draft rows that is, after
// m refused children of a node, max(a p - b q, 0) with a and b numbers: from
// w' = max(w / Z - q, 0) follow a' = a / Z and b' = b / Z + 1.  So a row is never
// stored, and w of any token is known from a and b.
//
// Sums are 64 bits: a row of 2^17 values in 32 would move the places where one
// token ends and the next begins by more than many a token's share.
#include <algorithm>

#include "draft.h"

namespace ilpm {
namespace {

// A probability as it counts: nothing that is not above 0, nothing beyond fp32.
template <typename T> __device__ inline float prob(T v)
{
    return fminf(fmaxf((float)v, 0.f), 3.402823466e38f);  // (of a NaN and a number the number)
}

// (Rounded in the same places wherever it is formed: what a sum found above 0 the search in
// it must find above 0 again.)
__device__ inline double left_of(double a, double b, float p, float q)
{
    return fmax(__builtin_fma(a, (double)p, -(b * (double)q)), 0.);
}

// What is the same in all lanes, as the compiler cannot know of values from LDS.
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A value's two words, each moved as the vector unit can: sums over a wave lie in every
// chain here, and by way of LDS cost 2 of 12 us for a row of 32000 values, of 17.6 for 64 of
// 131072.
template <typename F> __device__ inline double by_words(double v, F f)
{
    const unsigned long long x = __builtin_bit_cast(unsigned long long, v);
    return __builtin_bit_cast(double, (unsigned long long)f((unsigned)(x >> 32)) << 32 | f((unsigned)x));
}
// (Where the other lane would lie in another sixteen, 0.)
template <int CTRL> __device__ inline double dpp(double v)
{
    return by_words(v, [](unsigned w) { return (unsigned)__builtin_amdgcn_mov_dpp((int)w, CTRL, 0xf, 0xf, true); });
}
__device__ inline double of_lane(double v, int lane)
{
    return by_words(v, [=](unsigned w) { return (unsigned)__builtin_amdgcn_readlane((int)w, lane); });
}

// (Once the lanes of a four or eight hold the same, a mirror is as good a partner as any.)
__device__ inline double sum_wave(double v)
{
    v += dpp<0xb1>(v);   // of pairs
    v += dpp<0x4e>(v);   // of fours
    v += dpp<0x141>(v);  // eight mirrored
    v += dpp<0x140>(v);  // sixteen mirrored
    return (of_lane(v, 0) + of_lane(v, 16)) + (of_lane(v, 32) + of_lane(v, 48));
}

// The sum of a lane's value and those of all lanes before it.
__device__ inline double sum_up_to(double v)
{
    v += dpp<0x111>(v);  // of the lane 1 before it in its sixteen, then 2, 4 and 8
    v += dpp<0x112>(v);
    v += dpp<0x114>(v);
    v += dpp<0x118>(v);
    const double a = of_lane(v, 15), b = a + of_lane(v, 31), c = b + of_lane(v, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return v + (row == 0 ? 0. : row == 1 ? a : row == 2 ? b : c);
}

// The sum over the workgroup, in all threads.
template <int THREADS> __device__ inline double sum_all(double v, double *lds)
{
    v = sum_wave(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
    return s;
}

template <typename T> __device__ inline const T *row_of(const void *base, int64_t seq_stride, int64_t node_stride, int seq, int node)
{
    return (const T *)base + (int64_t)seq * seq_stride + (int64_t)node * node_stride;
}

// N elements of a row from i on, as they are read: in pieces of 16 bytes, the last
// ones end with the row (over some elements before i), so that no load waits for a
// condition.
template <typename T, bool DRAFT, int N> struct Run {
    static constexpr int VEC = 16 / sizeof(T);
    Pack<T, VEC> p[N / VEC], q[DRAFT ? N / VEC : 1];
};

// What is left of a node's row.
template <typename T, bool DRAFT> struct Rest {
    static constexpr int VEC = 16 / sizeof(T);
    const T *p, *q;
    double a, b;
    int vocab;
    const unsigned *hole;  // a bit for each element from `first` on that is taken out (without draft rows), or NULL
    int first;

    __device__ __forceinline__ int place(int64_t i) const { return (int)min(i, (int64_t)(vocab - VEC)); }
    template <int N> __device__ __forceinline__ void load(int64_t i, Run<T, DRAFT, N> &r) const
    {
        if (vocab < VEC) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const bool in = i + k < vocab;
                r.p[k / VEC].v[k % VEC] = in ? p[i + k] : (T)0.f;
                if constexpr (DRAFT) r.q[k / VEC].v[k % VEC] = in ? q[i + k] : (T)0.f;
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < N / VEC; ++k) {
            r.p[k] = load_loose<T, VEC>(p + place(i + k * VEC));
            if constexpr (DRAFT) r.q[k] = load_loose<T, VEC>(q + place(i + k * VEC));
        }
    }
    // The sum of a run that lies in the row.
    template <int N> __device__ __forceinline__ double sum_inside(int i, const Run<T, DRAFT, N> &r) const
    {
        double s = 0.;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float pe = prob(r.p[k / VEC].v[k % VEC]);
            double w = pe;
            if constexpr (DRAFT) {
                w = left_of(a, b, pe, prob(r.q[k / VEC].v[k % VEC]));
            } else {
                if (hole && ((hole[(i + k - first) >> 5] >> ((i + k - first) & 31)) & 1)) w = 0.;
            }
            s += w;
        }
        return s;
    }
    // f(element, its weight) of those of the run that lie in the row, in order; of the
    // others f(.., 0).  whole: the row itself in the place of what is left of it.
    template <int N, typename F> __device__ __forceinline__ void each(int64_t i, const Run<T, DRAFT, N> &r, bool whole, F f) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t own = i + k - k % VEC;
            const int e = vocab < VEC ? (int)min(i + k, (int64_t)vocab) : place(own) + k % VEC;
            const float pe = prob(r.p[k / VEC].v[k % VEC]);
            double w = pe;
            if constexpr (DRAFT) {
                if (!whole) w = left_of(a, b, pe, prob(r.q[k / VEC].v[k % VEC]));
            } else {
                if (hole && !whole && e >= own && ((hole[(e - first) >> 5] >> ((e - first) & 31)) & 1)) w = 0.;
            }
            f(e, e >= own && e < vocab ? w : 0.);
        }
    }
    template <int N> __device__ __forceinline__ double sum(int64_t i, const Run<T, DRAFT, N> &r, bool whole) const
    {
        double s = 0.;
        each(i, r, whole, [&](int, double w) { s += w; });
        return s;
    }
};

// A sequence's walk: the node where it ended (-1: no tree), what is left of its row,
// and which children were refused; lane i holds node i's token.
struct Walk {
    int node, token;
    double a, b;
    unsigned long long gone;
};

// All threads of a workgroup walk alike; they are needed only where a node has
// several children and draft rows, for the sums after a refusal.
template <typename T, bool DRAFT, int THREADS> __device__ __forceinline__ Walk walk_tree(const ilpm_verify_args &v, int seq, double *lds, bool write)
{
    const int lane = threadIdx.x & 63, n = v.n_nodes;
    const int64_t at = (int64_t)seq * n;
    // Lane i holds node i, and its probabilities below its parent.
    int parent = -2, token = -1;
    float u = 0.f, p = 0.f, q = 0.f;
    if (lane < n) {
        parent = v.parents[at + lane];
        token = v.tokens[at + lane];
        u = v.uniforms[at + lane];
        if (token < 0 || token >= v.vocab) token = -1;
        if (token >= 0 && parent >= 0 && parent < lane) {
            p = prob(row_of<T>(v.target, v.target_seq_stride, v.target_node_stride, seq, parent)[token]);
            if constexpr (DRAFT) q = prob(row_of<T>(v.draft, v.draft_seq_stride, v.draft_node_stride, seq, parent)[token]);
        }
    }
    const bool real = __builtin_amdgcn_readlane(parent, 0) == -1;
    int cur = 0, count = 1;
    int mine = lane == 0 ? 0 : -1;  // path[lane]
    double wa = 1., wb = 0., z = 1.;
    unsigned long long gone = 0;  // refused children of the current node
    unsigned long long kids = __builtin_amdgcn_ballot_w64(parent == 0 && lane > 0 && token >= 0);
    auto of_lane = [](float x, int c) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), c)); };
    while (real && kids) {
        const int c = __builtin_ctzll(kids);
        kids &= kids - 1;
        const int x = __builtin_amdgcn_readlane(token, c);
        const double uc = of_lane(u, c);
        const float pc = of_lane(p, c), qc = of_lane(q, c);
        bool keep;
        double w;
        if constexpr (DRAFT) {
            w = left_of(wa, wb, pc, qc);
            keep = z > 0. && uc * (double)qc * z < w;
        } else {
            // (A token that was refused before has nothing left.)
            const bool again = __builtin_amdgcn_ballot_w64(((gone >> lane) & 1) && token == x) != 0;
            w = again ? 0. : (double)pc;
            keep = z > 0. && uc * z < w;
        }
        if (keep) {
            cur = c;
            if (lane == count) mine = c;
            ++count;
            wa = z = 1.;
            wb = 0.;
            gone = 0;
            kids = __builtin_amdgcn_ballot_w64(parent == c && lane > c && token >= 0);
            continue;
        }
        if (!(z > 0.)) continue;
        if constexpr (DRAFT) {
            wa /= z;
            wb = wb / z + 1.;
            if (!kids) continue;
            // Four pieces of a thread are on their way at once.
            const Rest<T, true> r = {row_of<T>(v.target, v.target_seq_stride, v.target_node_stride, seq, cur),
                                     row_of<T>(v.draft, v.draft_seq_stride, v.draft_node_stride, seq, cur), wa, wb, v.vocab, nullptr, 0};
            constexpr int VEC = 16 / sizeof(T), STEP = THREADS * VEC;
            const int mine = threadIdx.x * VEC;
            double s = 0.;
            int64_t i0 = 0;
            for (; i0 + 4 * STEP <= v.vocab; i0 += 4 * STEP) {
                Run<T, true, VEC> run[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) r.load(i0 + k * STEP + mine, run[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k) s += r.sum_inside((int)i0 + k * STEP + mine, run[k]);
            }
#pragma unroll 1
            for (; i0 < v.vocab; i0 += STEP) {
                Run<T, true, VEC> run;
                r.load(i0 + mine, run);
                s += r.sum(i0 + mine, run, false);
            }
            z = sum_all<THREADS>(s, lds);
        } else {
            z -= w;
            gone |= 1ull << c;
        }
    }
    if (write) {
        if (threadIdx.x < n) v.path[at + lane] = real ? mine : -1;
        if (threadIdx.x == 0) v.counts[seq] = real ? count : 0;
    }
    return Walk{real ? cur : -1, token, wa, wb, gone};
}

// Marks in `hole` the tokens of refused children among `elements` from `first` on.
__device__ __forceinline__ void mark(unsigned long long gone, int token, unsigned *hole, int first, int elements)
{
    for (int i = threadIdx.x; i < (elements + 31) / 32; i += blockDim.x) hole[i] = 0;
    __syncthreads();
    if (threadIdx.x < 64 && ((gone >> threadIdx.x) & 1)) {
        const int i = token - first;
        if (i >= 0 && i < elements) atomicOr(&hole[i >> 5], 1u << (i & 31));
    }
    __syncthreads();
}

template <typename T, bool DRAFT> __device__ __forceinline__ Rest<T, DRAFT> rest_of(const ilpm_verify_args &v, int seq, int node, double a, double b)
{
    return Rest<T, DRAFT>{row_of<T>(v.target, v.target_seq_stride, v.target_node_stride, seq, node),
                          DRAFT ? row_of<T>(v.draft, v.draft_seq_stride, v.draft_node_stride, seq, node) : nullptr, a, b, v.vocab, nullptr, 0};
}

// How much of `total` lies before the next token.  (A number below 0 counts as 0: the
// searches end where they have passed what is wanted, and must have found a place by then.)
__device__ inline double wanted(const ilpm_verify_args &v, int seq, double total)
{
    const float u = v.uniforms[(int64_t)seq * v.n_nodes];
    return (double)(u < 0.f ? 0.f : u) * total;
}

// Of 64 lanes' values in their order the first at which the sum with all before
// it passes `want`, else the last above 0 (-1: none); *before: the sum before it.
__device__ inline int pick_lane(double own, double want, double *before)
{
    const double up_to = sum_up_to(own);
    const unsigned long long passed = __builtin_amdgcn_ballot_w64(own > 0. && up_to > want);
    const unsigned long long some = __builtin_amdgcn_ballot_w64(own > 0.);
    const int at = passed ? __builtin_ctzll(passed) : some ? 63 - __builtin_clzll(some) : -1;
    *before = of_lane(up_to - own, max(at, 0));
    return at;
}

// The same of a thread's elements from i on.
template <int N, typename T, bool DRAFT> __device__ inline int pick_run(const Rest<T, DRAFT> &r, int64_t i, const Run<T, DRAFT, N> &run, bool whole, double want)
{
    double up_to = 0.;
    int found = -1, some = -1;
    r.each(i, run, whole, [&](int e, double w) {
        up_to += w;
        if (w > 0.) {
            some = e;
            if (found < 0 && up_to > want) found = e;
        }
    });
    return found >= 0 ? found : some;
}

// ---- short rows: a workgroup does all of a sequence ----
// A piece of 16 bytes a thread and round, so that neighbours read neighbouring
// pieces; the rounds, in them the waves and in them the lanes are in the row's order.
constexpr int kShortThreads = 1024, kRounds = 8;
template <typename T> constexpr int kShortVocab = kRounds * kShortThreads * 16 / (int)sizeof(T);

template <typename T, bool DRAFT> __global__ __launch_bounds__(kShortThreads) void verify_short(VerifyArgs a)
{
    constexpr int WAVES = kShortThreads / 64, VEC = 16 / sizeof(T);
    static_assert(kRounds * WAVES == 128, "two values a lane");
    __shared__ double lds[WAVES], sums[kRounds * WAVES];
    __shared__ unsigned hole[kShortVocab<T> / 32];
    const ilpm_verify_args &v = a.v;
    const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const Walk end = walk_tree<T, DRAFT, kShortThreads>(v, seq, lds, true);
    if (end.node < 0) {
        if (tid == 0) v.next_tokens[seq] = -1;
        return;
    }
    Rest<T, DRAFT> r = rest_of<T, DRAFT>(v, seq, end.node, end.a, end.b);
    if (end.gone) {
        mark(end.gone, end.token, hole, 0, v.vocab);
        r.hole = hole;
    }
    auto piece = [&](int k) { return (int64_t)(k * kShortThreads + tid) * VEC; };
    // What is left of the row, or, where that is nothing, the row itself.  (In loops: most of the instructions run
    // once or twice, and cost their fetching.  With the rounds unrolled this took 30 us for 32000 values, in loops 12, and now 10.)
    const int rounds = (v.vocab + kShortThreads * VEC - 1) / (kShortThreads * VEC);
    double own[2], total = 0.;
    bool whole = false;
#pragma unroll 1
    for (;;) {
        Run<T, DRAFT, VEC> next;
        r.load(piece(0), next);
#pragma unroll 1
        for (int k = 0; k < rounds; ++k) {
            const Run<T, DRAFT, VEC> run = next;
            r.load(piece(k + 1), next);
            const bool inside = (k + 1) * kShortThreads * VEC <= v.vocab && !whole;
            const double s = sum_wave(inside ? r.sum_inside((int)piece(k), run) : r.sum(piece(k), run, whole));
            if (lane == 0) sums[k * WAVES + wave] = s;
        }
        __syncthreads();
        own[0] = lane < rounds * WAVES ? sums[lane] : 0.;
        own[1] = 64 + lane < rounds * WAVES ? sums[64 + lane] : 0.;
        total = sum_wave(own[0] + own[1]);
        if (total > 0. || whole) break;
        whole = true;
        __syncthreads();
    }
    if (!(total > 0.)) {
        if (tid == 0) v.next_tokens[seq] = -1;
        return;
    }
    double want = wanted(v, seq, total), before;
    // The wave and round that hold it: among the first 64, or the others where there are any.
    int at = -1;
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
        const double mine = h == 0 ? own[0] : own[1];
        double b;
        const int in = uniform(pick_lane(mine, want, &b));
        if (in >= 0) {
            at = h * 64 + in;
            before = want - b;
        }
        want -= sum_wave(mine);
        if (want < 0.) break;
    }
    if (wave != at % WAVES) return;
    // (Its piece again, and then the lane and the element.)
    const int64_t i = piece(at / WAVES);
    Run<T, DRAFT, VEC> run;
    r.load(i, run);
    double before_lane;
    const int in = pick_lane(r.sum(i, run, whole), before, &before_lane);
    if (lane == in) v.next_tokens[seq] = pick_run(r, i, run, whole, before - before_lane);
}

// ---- long rows: a workgroup for each chunk ----
constexpr int kRun = 16, kThreads = kVerifyChunk / kRun;  // elements of a thread

template <typename T> __global__ __launch_bounds__(1024) void verify_walk(VerifyArgs a)
{
    __shared__ double lds[16];
    const int seq = blockIdx.x, lane = threadIdx.x & 63;
    const Walk end = walk_tree<T, true, 1024>(a.v, seq, lds, true);
    VerifyEnd &to = a.ends[seq];
    if (threadIdx.x == 0) {
        to.node = end.node;
        to.a = end.a;
        to.b = end.b;
        to.gone = end.gone;
    }
    if (threadIdx.x < 64 && lane < a.v.n_nodes) to.token[lane] = end.token;
}

// Without draft rows a walk costs its few accesses, and every workgroup does
// it for itself.
template <typename T, bool DRAFT> __global__ __launch_bounds__(kThreads) void verify_sums(VerifyArgs a)
{
    __shared__ double lds[kThreads / 64];
    __shared__ unsigned hole[kVerifyChunk / 32];
    const int seq = blockIdx.y, chunk = blockIdx.x, lane = threadIdx.x & 63;
    Walk end;
    if constexpr (!DRAFT) {
        end = walk_tree<T, false, kThreads>(a.v, seq, lds, chunk == 0);
        if (chunk == 0) {
            VerifyEnd &to = a.ends[seq];
            if (threadIdx.x == 0) {
                to.node = end.node;
                to.a = end.a;
                to.b = end.b;
                to.gone = end.gone;
            }
            if (threadIdx.x < 64 && lane < a.v.n_nodes) to.token[lane] = end.token;
        }
    } else {
        const VerifyEnd &from = a.ends[seq];
        end = Walk{from.node, lane < a.v.n_nodes ? from.token[lane] : -1, from.a, from.b, from.gone};
    }
    if (end.node < 0) return;
    Rest<T, DRAFT> r = rest_of<T, DRAFT>(a.v, seq, end.node, end.a, end.b);
    r.first = chunk * kVerifyChunk;
    // (Neighbouring threads read neighbouring pieces; the sums' order does not matter here.)
    constexpr int VEC = 16 / sizeof(T), PIECES = kRun / VEC;
    Run<T, DRAFT, VEC> run[PIECES];
    auto piece = [&](int k) { return (int64_t)r.first + (k * kThreads + (int)threadIdx.x) * VEC; };
#pragma unroll
    for (int k = 0; k < PIECES; ++k) r.load(piece(k), run[k]);
    if (end.gone) {
        mark(end.gone, end.token, hole, r.first, kVerifyChunk);
        r.hole = hole;
    }
    double sum = 0.;
    if ((int64_t)r.first + kVerifyChunk <= a.v.vocab) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) sum += r.sum_inside((int)piece(k), run[k]);
    } else {
#pragma unroll 1
        for (int k = 0; k < PIECES; ++k) {
            sum += r.sum(piece(k), run[0], false);
#pragma unroll
            for (int n = 0; n + 1 < PIECES; ++n) run[n] = run[n + 1];
        }
    }
    sum = sum_all<kThreads>(sum, lds);
    if (threadIdx.x == 0) a.sums[(int64_t)seq * a.chunks + chunk] = sum;
}

template <typename T, bool DRAFT> __global__ __launch_bounds__(kThreads) void verify_pick(VerifyArgs a)
{
    constexpr int WAVES = kThreads / 64;
    __shared__ double lds[64];
    __shared__ unsigned hole[kVerifyChunk / 32];
    const ilpm_verify_args &v = a.v;
    const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const VerifyEnd &end = a.ends[seq];
    const int node = uniform(end.node);
    if (node < 0) {
        if (tid == 0) v.next_tokens[seq] = -1;
        return;
    }
    // Every wave finds the chunk.
    double *sums = a.sums + (int64_t)seq * a.chunks;
    auto sum_of_all = [&] {
        double s = 0.;
        for (int c = lane; c < a.chunks; c += 64) s += sums[c];
        return sum_wave(s);
    };
    double total = sum_of_all();
    const bool whole = !(total > 0.);
    if (whole) {  // nothing is left: the row itself, summed here
        const Rest<T, DRAFT> r = rest_of<T, DRAFT>(v, seq, node, end.a, end.b);
        for (int c = 0; c < a.chunks; ++c) {
            double s = 0.;
#pragma unroll 1
            for (int k = 0; k < kRun / (16 / (int)sizeof(T)); ++k) {
                constexpr int VEC = 16 / sizeof(T);
                const int64_t i = (int64_t)c * kVerifyChunk + (k * kThreads + tid) * VEC;
                Run<T, DRAFT, VEC> run;
                r.load(i, run);
                s += r.sum(i, run, true);
            }
            s = sum_all<kThreads>(s, lds);
            if (tid == 0) sums[c] = s;
        }
        __threadfence_block();
        __syncthreads();
        total = sum_of_all();
    }
    if (!(total > 0.)) {
        if (tid == 0) v.next_tokens[seq] = -1;
        return;
    }
    double want = wanted(v, seq, total), before = 0., rest = 0.;
    int chunk = 0;
    for (int c0 = 0; c0 < a.chunks; c0 += 64) {
        const double own = c0 + lane < a.chunks ? sums[c0 + lane] : 0.;
        double up_to;
        const int at = uniform(pick_lane(own, want - before, &up_to));
        if (at >= 0) {
            chunk = c0 + at;
            rest = want - before - up_to;
        }
        before += sum_wave(own);
        if (before > want) break;
    }
    Rest<T, DRAFT> r = rest_of<T, DRAFT>(v, seq, node, end.a, end.b);
    r.first = chunk * kVerifyChunk;
    if (end.gone) {
        mark(end.gone, lane < v.n_nodes ? end.token[lane] : -1, hole, r.first, kVerifyChunk);
        r.hole = hole;
    }
    // Wave w takes the w-th quarter of the chunk, in rounds of a piece a lane.
    constexpr int VEC = 16 / sizeof(T), ROUNDS = kRun / VEC;
    auto piece = [&](int k) { return (int64_t)r.first + (((wave * ROUNDS) + k) * 64 + lane) * VEC; };
    Run<T, DRAFT, VEC> run[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) r.load(piece(k), run[k]);
#pragma unroll 1
    for (int k = 0; k < ROUNDS; ++k) {
        const double s = sum_wave(r.sum(piece(k), run[0], whole));
        if (lane == 0) lds[wave * ROUNDS + k] = s;
#pragma unroll
        for (int n = 0; n + 1 < ROUNDS; ++n) run[n] = run[n + 1];
    }
    __syncthreads();
    double before_run, before_lane;
    const int at = uniform(pick_lane(lane < WAVES * ROUNDS ? lds[lane] : 0., rest, &before_run));
    if (wave != at / ROUNDS) return;
    const int64_t i = piece(at % ROUNDS);
    r.load(i, run[0]);
    const int in = pick_lane(r.sum(i, run[0], whole), rest - before_run, &before_lane);
    if (lane == in) v.next_tokens[seq] = pick_run(r, i, run[0], whole, rest - before_run - before_lane);
}

template <typename T, bool DRAFT> hipError_t launch(const VerifyArgs &a, hipStream_t stream)
{
    if (a.chunks == 0) {
        hipLaunchKernelGGL((verify_short<T, DRAFT>), dim3(a.v.n_seqs), dim3(kShortThreads), 0, stream, a);
        return hipGetLastError();
    }
    if constexpr (DRAFT) hipLaunchKernelGGL((verify_walk<T>), dim3(a.v.n_seqs), dim3(1024), 0, stream, a);
    hipLaunchKernelGGL((verify_sums<T, DRAFT>), dim3(a.chunks, a.v.n_seqs), dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL((verify_pick<T, DRAFT>), dim3(a.v.n_seqs), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename T> hipError_t launch(const VerifyArgs &a, hipStream_t stream)
{
    return a.v.draft ? launch<T, true>(a, stream) : launch<T, false>(a, stream);
}

size_t ends_bytes(int n_seqs) { return ((size_t)n_seqs * sizeof(VerifyEnd) + 15) / 16 * 16; }

}  // namespace

// Rows of up to 128 KB are one kernel's work, a workgroup a sequence, bounded by a chain
// of accesses (10 us for one row of 32000 f32 values); longer ones are summed in chunks by
// many (64 rows of 131072 values, 34 MB, 16 us, 7 of it in the second kernel, which finds
// the chunk and the token).  1, 16, 64 and 256 rows of 16384 f32 values take 7.3, 8.1, 8.9 and
// 10.1 us in one kernel and 9.9, 11.3, 12.4 and 14.7 in chunks; of 32768 10.3, 11.7, 12.2 and
// 14.4, and 10.4, 12.0, 13.0 and 17.7.  For 16-bit rows the border by bytes is high: 1 and 64
// rows of 65536 bf16 values 13.9 and 16.2 in one kernel, 11.3 and 14.7 in chunks.
size_t verify_plan(VerifyArgs *a)
{
    const int most = a->v.dtype == ILPM_F32 ? kShortVocab<float> : kShortVocab<__bf16>;
    a->chunks = a->v.vocab <= most ? 0 : (a->v.vocab + kVerifyChunk - 1) / kVerifyChunk;
    return a->chunks == 0 ? 0 : ends_bytes(a->v.n_seqs) + (size_t)a->v.n_seqs * (size_t)a->chunks * sizeof(double);
}

void verify_workspace(VerifyArgs *a, void *ws)
{
    a->ends = (VerifyEnd *)ws;
    a->sums = (double *)((char *)ws + ends_bytes(a->v.n_seqs));
}

hipError_t verify_launch(const VerifyArgs &a, hipStream_t stream)
{
    if (a.v.dtype == ILPM_F32) return launch<float>(a, stream);
    if (a.v.dtype == ILPM_F16) return launch<_Float16>(a, stream);
    return launch<__bf16>(a, stream);
}

}  // namespace ilpm
