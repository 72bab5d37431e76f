// attn_tree: how a call is shared out over the card, and the join of units that
// span workgroups (the kernel over the keys is in draft_attn.h).
#include <algorithm>
#include <climits>

#include "draft.h"

namespace ilpm {

#define ILPM_TREE_KERNELS(name)                                          \
    hipError_t tree_split_##name(const TreeArgs &t, hipStream_t stream); \
    int tree_most_##name(int dim);                                       \
    int tree_card_##name(int dim, bool pieces, int blocks);
ILPM_TREE_KERNELS(f32)
ILPM_TREE_KERNELS(f16)
ILPM_TREE_KERNELS(f16_q32)
ILPM_TREE_KERNELS(bf16)
ILPM_TREE_KERNELS(bf16_q32)
#undef ILPM_TREE_KERNELS

namespace {

constexpr int kMaxParts = 4 * kAttnCus;  // of a unit: workgroups of a call
constexpr float kLn2 = 0.69314718055994530942f;
typedef float floatx4 __attribute__((ext_vector_type(4)));

__device__ inline void store_f32(void *p, int64_t i, int dtype, float v)
{
    if (dtype == ILPM_F32) ((float *)p)[i] = v;
    else if (dtype == ILPM_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// Part i of a unit, for a row of it: of the workgroup of the row's block that holds the
// unit's i-th share, its part that begins a unit or the one that goes on with it.
__device__ inline int64_t part_at(const TreeArgs &t, const AttnPart &u, int row, int i)
{
    const int block = row / (16 * t.row_blocks), in_block = row - block * 16 * t.row_blocks;
    return ((((int64_t)u.first + i) * t.a.blocks + block) * 2 + (i == 0)) * t.a.part_heads + in_block;
}

// Joins the parts of the unit at place blockIdx.y, for its row blockIdx.x and 64
// values of it, blockIdx.z, as attn_decode's parts are (attn_join).
template <int V> __global__ __launch_bounds__(256) void tree_join(TreeArgs t)
{
    constexpr int T = 64 / V, G = 256 / T, AHEAD = 4, OWN = kMaxParts / 256;
    __shared__ float red[2][4], w[kMaxParts];
    __shared__ Pack<float, V> sum[G][T];
    const AttnArgs &a = t.a;
    const AttnPart u = a.parts[blockIdx.y];
    if (u.count == 0) return;
    const int row = blockIdx.x, node = t.by_group.of(row), head = u.unit * a.group + (row - node * a.group), tid = threadIdx.x;
    const int64_t out_row = (int64_t)u.seq * t.n_nodes + node;
    auto slot = [&](int i) { return part_at(t, u, row, i); };
    const int group = tid / T, d = (int)blockIdx.z * 64 + tid % T * V;
    auto part = [&](int i) {
        Pack<float, V> p = {};
        if (i < u.count && d < a.dim) p = load_pack<float, V>(a.part_o + slot(i) * a.dim + d);
        return p;
    };
    float m[OWN], l[OWN], top = -INFINITY, total = 0.f;
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int i = tid + k * 256;
        m[k] = i < u.count ? a.part_ml[slot(i) * 2] : -INFINITY;
        l[k] = i < u.count ? a.part_ml[slot(i) * 2 + 1] : 0.f;
    }
    Pack<float, V> ahead[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ahead[k] = part(group + k * G);
#pragma unroll
    for (int k = 0; k < OWN; ++k) top = fmaxf(top, m[k]);
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) red[0][tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const float f = __builtin_amdgcn_exp2f(m[k] - base);
        total += l[k] * f;
        if (tid + k * 256 < u.count) w[tid + k * 256] = f;
    }
    for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
    if ((tid & 63) == 0) red[1][tid >> 6] = total;
    __syncthreads();
    Pack<float, V> v = {};
    auto add = [&](const Pack<float, V> &p, int i) {
        if (i >= u.count) return;
#pragma unroll
        for (int k = 0; k < V; ++k) v.v[k] += p.v[k] * w[i];
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) add(ahead[k], group + k * G);
#pragma unroll 4
    for (int i = group + AHEAD * G; i < u.count; i += G) add(part(i), i);
    sum[group][tid % T] = v;
    __syncthreads();
    total = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int e = (int)blockIdx.z * 64 + tid;
    if (tid < 64 && e < a.dim) {
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) x += sum[g][tid / V].v[tid % V];
        store_f32(a.out, out_row * a.o_row + (int64_t)head * a.o_head + e, a.q_dtype, x * inv);
    }
    if (e == 0 && a.lse) a.lse[out_row * a.q_heads + head] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// The same where there are many: a thread takes four values of a row, over all
// parts.
__global__ __launch_bounds__(256) void tree_join_rows(TreeArgs t, int lanes, Divisor by_lanes)
{
    const AttnArgs &a = t.a;
    const AttnPart u = a.parts[blockIdx.y];
    if (u.count == 0) return;
    const int r = by_lanes.of((int)threadIdx.x), lane = (int)threadIdx.x - r * lanes, per = by_lanes.of(256);
    const int row = (int)blockIdx.x * per + r, d = lane * 4;
    if (r >= per || row >= t.rows) return;
    const int node = t.by_group.of(row), head = u.unit * a.group + (row - node * a.group);
    const int64_t out_row = (int64_t)u.seq * t.n_nodes + node;
    auto slot = [&](int i) { return part_at(t, u, row, i); };
    float top = -INFINITY, total = 0.f;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    // (A part at a time with the maximum so far: in their order, two accesses each that do not wait for others.)
#pragma unroll 4
    for (int i = 0; i < u.count; ++i) {
        const int64_t at = slot(i);
        const float m = a.part_ml[at * 2], l = a.part_ml[at * 2 + 1];
        const floatx4 p = *reinterpret_cast<const floatx4 *>(a.part_o + at * a.dim + d);
        const float now = fmaxf(top, m), base = now == -INFINITY ? 0.f : now;
        const float old = __builtin_amdgcn_exp2f(top - base), own = __builtin_amdgcn_exp2f(m - base);
        top = now;
        total = total * old + l * own;
        v = v * old + p * own;
    }
    v *= total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int k = 0; k < 4; ++k) store_f32(a.out, out_row * a.o_row + (int64_t)head * a.o_head + d + k, a.q_dtype, v[k]);
    if (d == 0 && a.lse) a.lse[out_row * a.q_heads + head] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

}  // namespace

// As attn_plan: either a unit (a key head of a sequence) goes to a workgroup for each
// of its blocks of rows, or as many workgroups as the card holds share all tiles,
// each share a workgroup for each block, and a second kernel joins their parts.  Up to
// 16 tiles, and with W workgroups up to W / 2 tiles and 100, units are faster (tiles of
// more than 8 KB count as several: 140 units of 64 tiles of 32 KB 45 us shared and 63 by units): 40 x 600
// bf16 keys of 8 heads of 128 under 16 nodes of 32 heads 40 us shared and 31 by units
// (W 320, 39 tiles), 8 x 400 25 and 18 (64, 26), 20 x 1200 35 and 33 (160, 76), but 8 x
// 800 under 3 nodes, f32 over f16 heads of 80, 18 and 19 (64, 51), 8 x 1500 20 and 28.
//
// By units, up to 16 tiles and for more than 32 rows, the waves of a workgroup take rows
// and not keys: a unit of one tile then takes 7 us in the place of 12 (2048 units of 64
// rows, bf16 heads of 128, 48 -> 29 us; at 8 tiles 66 and 65).  With few workgroups, which
// leave compute units idle, that makes the tiles' chain longer from 5 tiles on (12 nodes
// of 80 / 8 f32 heads over 60 keys 13.6 -> 16.1 us), and keys are split there.
size_t tree_plan(TreeArgs *t, int cache_dtype, bool q32, int max_len)
{
    AttnArgs *a = &t->a;
    t->rows = t->n_nodes * a->group;
    t->by_group = Divisor((unsigned)a->group);
#define ILPM_TREE_OF(f, ...)                                                 \
    (cache_dtype == ILPM_F32   ? f##_f32(__VA_ARGS__)                        \
     : cache_dtype == ILPM_F16 ? (q32 ? f##_f16_q32(__VA_ARGS__) : f##_f16(__VA_ARGS__)) \
                               : (q32 ? f##_bf16_q32(__VA_ARGS__) : f##_bf16(__VA_ARGS__)))
    t->pieces = a->dim * element_bytes(cache_dtype) % 16 == 0;
    const int most = t->pieces ? ILPM_TREE_OF(tree_most, a->dim) : 1;
    t->row_blocks = std::min(most, t->rows > 32 ? 4 : t->rows > 16 ? 2 : 1);
    a->blocks = std::max(1, ceil_div(t->rows, 16 * t->row_blocks));
    const int64_t units = (int64_t)a->n_seqs * a->kv_heads;
    const int64_t sinks = a->window > 0 ? std::min<int64_t>(t->sinks, max_len) : 0;
    const int64_t keys = (a->window > 0 ? std::min<int64_t>(max_len, a->window) : max_len) + t->n_nodes;
    const int64_t tiles = std::max<int64_t>(1, (keys + 15) / 16 + (sinks + 15) / 16);
    // (Tiles are counted in 32 bits.  Where a table could name more, there are units enough without a split.)
    const int64_t span = (((int64_t)a->capacity + 15) / 16 + 2 + tree_unit_cost(t->row_blocks)) * units;
    const int64_t groups = units * a->blocks;
    const int64_t weight = std::max<int64_t>(8 << 10, (int64_t)a->dim * element_bytes(cache_dtype) * 32);
    a->split = tiles > kWholeTiles && tiles * weight > std::min<int64_t>(100, groups / 2) * (8 << 10) && units > 0 && (span < INT_MAX || units == 1);
    t->by_rows = !a->split && t->pieces && t->rows > 32 && tiles <= kWholeTiles && (tiles <= 4 || units * ceil_div(t->rows, 64) >= 32);
    if (!a->split) {
        if (t->by_rows) t->row_blocks = 4, a->blocks = ceil_div(t->rows, 64);
        a->grid = (int)units * a->blocks;
        return 0;
    }
    const int card = ILPM_TREE_OF(tree_card, a->dim, t->pieces, t->row_blocks);
#undef ILPM_TREE_OF
    const int shares = (int)std::min<int64_t>({std::max(1, std::min(card, kMaxParts) / a->blocks), units * ((tiles + tree_unit_cost(t->row_blocks) + kMinShare - 1) / kMinShare)});
    a->grid = shares * a->blocks;
    a->part_heads = std::min(t->rows, 16 * t->row_blocks);
    a->part_of_unit = units <= shares;
    return (size_t)a->grid * (sizeof(AttnPart) + 2 * a->part_heads * (size_t)(a->dim + 2) * sizeof(float));
}

void tree_workspace(TreeArgs *t, void *ws) { attn_workspace(&t->a, ws); }

hipError_t tree_launch(const TreeArgs &t, int cache_dtype, hipStream_t stream)
{
    const AttnArgs &a = t.a;
    const bool q32 = a.q_dtype == ILPM_F32;
    const hipError_t e = cache_dtype == ILPM_F32   ? tree_split_f32(t, stream)
                         : cache_dtype == ILPM_F16 ? (q32 ? tree_split_f16_q32(t, stream) : tree_split_f16(t, stream))
                                                   : (q32 ? tree_split_bf16_q32(t, stream) : tree_split_bf16(t, stream));
    if (e != hipSuccess || !a.split) return e;
    // A workgroup for each row and 64 values, or for many rows: 4 sequences of 8000 bf16 keys of 8
    // heads of 64 under 64 rows (2048 workgroups) 28.8 us and 29.2, 2 of 30000 of 128 (2048) 65.6 and
    // 67.6, 4 of 8000 of 128 (4096) 47.5 and 45.4, 16 of 4000 (16384) 91.9 and 75.3.
    const int joins = a.part_of_unit ? a.n_seqs * a.kv_heads : a.grid / a.blocks;
    if (a.dim % 4 == 0 && (int64_t)joins * t.rows * ceil_div(a.dim, 64) > 8 * kAttnCus) {
        const int lanes = a.dim / 4;
        hipLaunchKernelGGL(tree_join_rows, dim3(ceil_div(t.rows, 256 / lanes), joins), dim3(256), 0, stream, t, lanes, Divisor((unsigned)lanes));
        return hipGetLastError();
    }
    const dim3 grid(t.rows, joins, ceil_div(a.dim, 64));
    if (a.dim % 4) hipLaunchKernelGGL((tree_join<1>), grid, dim3(256), 0, stream, t);
    else hipLaunchKernelGGL((tree_join<4>), grid, dim3(256), 0, stream, t);
    return hipGetLastError();
}

}  // namespace ilpm
