// What the operators of a drafted decoder step share: their arguments as the
// kernels take them, and their launchers (the entry points check the
// arguments, draft_api.hip).
#pragma once

#include "decode.h"

namespace ilpm {

// ---- kv_append_norm ----
struct AppendNormArgs {
    AppendArgs a;  // (positions turn, slots place)
    const int32_t *slots;
    const void *q_w, *k_w;
    int norm;
    float eps;
};
hipError_t append_norm_launch(const AppendNormArgs &n, int x_dtype, int cache_dtype, int param_dtype, hipStream_t stream);

// ---- verify_drafts ----
// Probabilities that a workgroup sums: with 2048, 4096 and 8192 one row of 50000 f32 values takes
// 10.3, 10.7 and 10.9 us, 64 rows of 131072 17.4, 17.3 and 17.6, of draft rows as well 24.7,
// 24.1 and 26.6.
constexpr int kVerifyChunk = 4096;

// Where a sequence's walk ended, and what is left of that node's row: a p - b q, or p
// without the tokens of the children that are bits of `gone`.
struct VerifyEnd {
    int node;  // -1: no tree
    double a, b;
    unsigned long long gone;
    int token[ILPM_MAX_NODES];
};
struct VerifyArgs {
    ilpm_verify_args v;
    int chunks;  // of a row; 0: short rows, without a workspace
    VerifyEnd *ends;
    double *sums;  // [n_seqs][chunks]: of what is left of the row
};
size_t verify_plan(VerifyArgs *a);
void verify_workspace(VerifyArgs *a, void *ws);
hipError_t verify_launch(const VerifyArgs &a, hipStream_t stream);

// ---- kv_copy ----
struct CopyArgs {
    void *k, *v;
    int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;  // in bytes
    int row_bytes, kv_heads, n_pages, page_size;
    const int32_t *src_table, *dst_table;
    int64_t src_table_stride, dst_table_stride;
    int src_max_pages, dst_max_pages, n_seqs;
    const int32_t *src_start, *dst_start, *counts, *path;
    int64_t path_stride;
    int max_count;
};
hipError_t copy_launch(const CopyArgs &a, hipStream_t stream);

// ---- attn_tree ----
// (Of AttnArgs: lengths without the nodes; group, blocks and part_heads count the rows
// of a key head, its nodes' heads: row r is head r % group of node r / group.)
struct TreeArgs {
    AttnArgs a;
    const int32_t *parents;
    int n_nodes, sinks;
    int rows;        // of a key head: n_nodes * group
    Divisor by_group{1};
    int row_blocks;  // of 16 rows that a workgroup takes
    bool pieces;     // heads are whole pieces of 16 bytes
    bool by_rows;    // the waves take rows, not keys (short sequences)
};
// What a unit costs beside its tiles, in tiles, by its row blocks: its start, a chain of
// dependent accesses, and the join of its waves.  (Without it, shares of many short units
// are longer than those of few long ones: 24 windowed units of 13 nodes, 12 heads of 80, took 35 us,
// with 12 to 24 tiles 28 to 30; where all units are long any number does.)
__host__ __device__ inline int tree_unit_cost(int row_blocks) { return 12 + 4 * row_blocks; }
size_t tree_plan(TreeArgs *t, int cache_dtype, bool q32, int max_len);
void tree_workspace(TreeArgs *t, void *ws);
hipError_t tree_launch(const TreeArgs &t, int cache_dtype, hipStream_t stream);

}  // namespace ilpm
