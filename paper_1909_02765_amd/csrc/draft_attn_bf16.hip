// attn_tree's kernels for bf16 caches (see draft_attn.h).
#include "draft_attn.h"

namespace ilpm {

hipError_t tree_split_bf16(const TreeArgs &t, hipStream_t stream) { return tree_split_by_dim<__bf16, true>(t, stream); }
int tree_most_bf16(int dim) { return tree_most_by_dim<__bf16, true>(dim); }
int tree_card_bf16(int dim, bool pieces, int blocks) { return tree_card_by_dim<__bf16, true>(dim, pieces, blocks); }

}  // namespace ilpm
