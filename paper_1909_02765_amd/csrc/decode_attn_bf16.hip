// attn_decode's kernels for bf16 caches (see decode_attn.h).
#include "decode_attn.h"

namespace ilpm {

hipError_t attn_split_bf16(const AttnArgs &a, hipStream_t stream) { return attn_split_by_dim<__bf16, true>(a, stream); }
int attn_card_bf16(int dim) { return attn_card_by_dim<__bf16, true>(dim); }

}  // namespace ilpm
