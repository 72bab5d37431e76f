// attn_decode's kernels for f16 caches and f32 queries (see decode_attn.h).
#include "decode_attn.h"

namespace ilpm {

hipError_t attn_split_f16_q32(const AttnArgs &a, hipStream_t stream) { return attn_split_by_dim<_Float16, false>(a, stream); }
int attn_card_f16_q32(int dim) { return attn_card_by_dim<_Float16, false>(dim); }

}  // namespace ilpm
