// attn_tree's kernels for f32 caches (see draft_attn.h).
#include "draft_attn.h"

namespace ilpm {

hipError_t tree_split_f32(const TreeArgs &t, hipStream_t stream) { return tree_split_by_dim<float, true>(t, stream); }
int tree_most_f32(int dim) { return tree_most_by_dim<float, true>(dim); }
int tree_card_f32(int dim, bool pieces, int blocks) { return tree_card_by_dim<float, true>(dim, pieces, blocks); }

}  // namespace ilpm
