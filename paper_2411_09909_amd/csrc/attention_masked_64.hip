// The masked attention for heads of 64 (attention_masked.h).
#include "attention_masked.h"

namespace amx {

hipError_t launch_attention_masked_64(int scale_kind, const MaskedOperands& m, const MaskedWork& w, int64_t q_heads, int chunks, bool small, bool pairs,
                                      hipStream_t s) {
  return launch_masked<64>(scale_kind, m, w, q_heads, chunks, small, pairs, s);
}

}  // namespace amx
