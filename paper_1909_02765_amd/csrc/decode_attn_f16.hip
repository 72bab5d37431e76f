// attn_decode's kernels for f16 caches (see decode_attn.h).
#include "decode_attn.h"

namespace ilpm {

hipError_t attn_split_f16(const AttnArgs &a, hipStream_t stream) { return attn_split_by_dim<_Float16, true>(a, stream); }
int attn_card_f16(int dim) { return attn_card_by_dim<_Float16, true>(dim); }

}  // namespace ilpm
