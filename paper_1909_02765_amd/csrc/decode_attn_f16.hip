// attn_decode's kernels for f16 caches (see decode_attn.h).
#include "decode_attn.h"

namespace ilpm {

hipError_t attn_split_f16(const AttnArgs &a, hipStream_t stream) { return attn_split_by_dim<_Float16, true>(a, stream); }

}  // namespace ilpm
