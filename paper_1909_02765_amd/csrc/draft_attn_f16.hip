// attn_tree's kernels for f16 caches (see draft_attn.h).
#include "draft_attn.h"

namespace ilpm {

hipError_t tree_split_f16(const TreeArgs &t, hipStream_t stream) { return tree_split_by_dim<_Float16, true>(t, stream); }
int tree_most_f16(int dim) { return tree_most_by_dim<_Float16, true>(dim); }
int tree_card_f16(int dim, bool pieces, int blocks) { return tree_card_by_dim<_Float16, true>(dim, pieces, blocks); }

}  // namespace ilpm
