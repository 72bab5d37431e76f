// What the decoder-step operators share: element types, their arguments as the
// kernels take them, and their launchers (the entry points check the
// arguments, decode_api.hip).
#pragma once

#include "internal.h"

namespace ilpm {

// ---- element types (ILPM_F32, ILPM_F16, ILPM_BF16) ----
template <int DT> struct ElementOf;
template <> struct ElementOf<ILPM_F32> { using type = float; };
template <> struct ElementOf<ILPM_F16> { using type = _Float16; };
template <> struct ElementOf<ILPM_BF16> { using type = __bf16; };

inline int element_bytes(int dtype) { return dtype == ILPM_F32 ? 4 : 2; }

// N elements that lie together, aligned to 16 bytes or their size: one memory
// access up to 16 bytes, several of 16 beyond.
template <typename T, int N> struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack { T v[N]; };

// A pack in memory, moved as whole words of the machine (taken by its elements
// the compiler may break a store into pieces: 16-bit values that only pass
// through were stored in four).
template <int BYTES> struct PackWord { typedef unsigned type __attribute__((ext_vector_type(4))); };
template <> struct PackWord<8> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <> struct PackWord<4> { typedef unsigned type; };
template <> struct PackWord<2> { typedef unsigned short type; };

// (ALIGN: of the address, in bytes.  The memory system takes words on any
// element's boundary whole as well.)
template <int ALIGN, typename T, int N> __device__ inline Pack<T, N> load_words(const T *p)
{
    using W = typename PackWord<(int)sizeof(Pack<T, N>)>::type;
    typedef W At __attribute__((aligned(ALIGN)));
    struct Words { W w[sizeof(Pack<T, N>) / sizeof(W)]; } words;
#pragma unroll
    for (unsigned i = 0; i < sizeof(words) / sizeof(W); ++i) words.w[i] = reinterpret_cast<const At *>(p)[i];
    return __builtin_bit_cast(Pack<T, N>, words);
}
template <int ALIGN, typename T, int N> __device__ inline void store_words(T *p, const Pack<T, N> &v)
{
    using W = typename PackWord<(int)sizeof(Pack<T, N>)>::type;
    typedef W At __attribute__((aligned(ALIGN)));
    struct Words { W w[sizeof(Pack<T, N>) / sizeof(W)]; };
    const Words words = __builtin_bit_cast(Words, v);
#pragma unroll
    for (unsigned i = 0; i < sizeof(words) / sizeof(W); ++i) reinterpret_cast<At *>(p)[i] = words.w[i];
}
// Of a pack that is aligned as one, and of one that is aligned to an element only.
template <typename T, int N> __device__ inline Pack<T, N> load_pack(const T *p) { return load_words<alignof(Pack<T, N>), T, N>(p); }
template <typename T, int N> __device__ inline Pack<T, N> load_loose(const T *p) { return load_words<sizeof(T), T, N>(p); }
template <typename T, int N> __device__ inline void store_pack(T *p, const Pack<T, N> &v) { store_words<alignof(Pack<T, N>), T, N>(p, v); }
template <typename T, int N> __device__ inline void store_loose(T *p, const Pack<T, N> &v) { store_words<sizeof(T), T, N>(p, v); }

// ---- kv_append ----
struct AppendArgs {
    // rows of heads: [token][head][dim], strides in elements
    const void *k, *v, *q;
    void *q_out;
    int64_t k_row, k_head, v_row, v_head, q_row, q_head, qo_row, qo_head;
    int n_tokens, q_heads, kv_heads, dim;
    // the cache's page pools, strides in elements
    void *kc, *vc;
    int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;
    const int32_t *table;
    int64_t table_stride;
    int n_seqs, max_pages, n_pages, page_size;
    const int32_t *seq_ids, *positions;
    const float *cos, *sin;  // [n_positions][rot_dim / 2]
    int n_positions, rot_dim, pairs;
};
hipError_t append_launch(const AppendArgs &a, int x_dtype, int cache_dtype, hipStream_t stream);

// ---- attn_decode ----
constexpr int kAttnHeads = 16;  // query heads of a workgroup
constexpr int kAttnCus = 256;   // compute units of the card
// Tiles of 16 keys, a workgroup's smallest share: a tile a wave (f32 queries over 16
// shared bf16 heads of 256, 8 sequences of up to 2049: 26 us with 10, 21 with 4).
constexpr int kMinShare = 4;
constexpr int kWholeTiles = 16; // units of so many are never split (see attn_plan)
constexpr int kUnitCost = 6;    // what a unit costs beside its tiles, in tiles

// A unit (key head x block of its query heads) that `count` workgroups share,
// from `first` on; count 0: none.
struct AttnPart {
    int seq, unit, first, count;
};

struct AttnArgs {
    const void *q;
    int64_t q_row, q_head;
    void *out;
    int64_t o_row, o_head;
    float *lse;  // [n_seqs][q_heads] or NULL
    int q_dtype;
    bool q_pieces;  // rows of q lie in 16-byte pieces
    const void *k, *v;
    int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;
    const int32_t *table;
    int64_t table_stride;
    int n_pages, page_size;
    int capacity;  // keys a row of the table can name
    const int32_t *lengths;
    const uint8_t *mask;  // [n_seqs][mask_len] or NULL
    int64_t mask_stride;
    int mask_len;
    int window;
    float scale, softcap;
    int n_seqs, q_heads, kv_heads, group, dim;
    int blocks;  // of up to kAttnHeads query heads of a key head
    int grid;
    bool split;  // the workgroups share all tiles out (else each takes a unit)
    int part_heads;  // heads of a part
    // The workspace of a split call: the shared units, each at its own place
    // (part_of_unit) or, where they are more than the workgroups, at the place of the
    // workgroup that began it; for each workgroup its two parts (the one that goes on
    // with a unit, the one that begins one), each its sums [part_heads][dim] and
    // its maximum and sum [part_heads][2].
    bool part_of_unit;
    AttnPart *parts;
    float *part_o, *part_ml;
};
// Fills blocks, grid, split and part_heads for sequences of up to max_len keys; the
// workspace bytes that they need, and their places in it.
size_t attn_plan(AttnArgs *a, int cache_dtype, bool q32, int max_len);
void attn_workspace(AttnArgs *a, void *ws);
hipError_t attn_launch(const AttnArgs &a, int cache_dtype, hipStream_t stream);

// ---- residual_norm ----
struct NormArgs {
    const void *x, *y;
    void *r, *z;
    int64_t x_row, y_row, r_row, z_row;
    const void *post_w, *post_b, *pre_w, *pre_b, *gate;
    int64_t gate_row;  // 0: one gate for all rows
    int rows, width, post, pre;
    float scale, eps;
};
hipError_t norm_launch(const NormArgs &a, int x_dtype, int y_dtype, int param_dtype, hipStream_t stream);

// ---- the C-ABI layer's helpers (ilpm_api.hip) ----
int api_hip_fail(hipError_t e);
int api_device_check(int *dev);
int api_workspace(int dev, size_t need, hipStream_t stream, void **ws);

}  // namespace ilpm
