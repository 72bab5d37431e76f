// attn_tree's kernels for f16 caches under 32-bit queries (see draft_attn.h).
#include "draft_attn.h"

namespace ilpm {

hipError_t tree_split_f16_q32(const TreeArgs &t, hipStream_t stream) { return tree_split_by_dim<_Float16, false>(t, stream); }
int tree_most_f16_q32(int dim) { return tree_most_by_dim<_Float16, false>(dim); }
int tree_card_f16_q32(int dim, bool pieces, int blocks) { return tree_card_by_dim<_Float16, false>(dim, pieces, blocks); }

}  // namespace ilpm
