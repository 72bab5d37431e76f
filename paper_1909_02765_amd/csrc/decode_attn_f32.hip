// attn_decode's kernels for f32 caches (see decode_attn.h).
#include "decode_attn.h"

namespace ilpm {

hipError_t attn_split_f32(const AttnArgs &a, hipStream_t stream) { return attn_split_by_dim<float, false>(a, stream); }
int attn_card_f32(int dim) { return attn_card_by_dim<float, false>(dim); }

}  // namespace ilpm
