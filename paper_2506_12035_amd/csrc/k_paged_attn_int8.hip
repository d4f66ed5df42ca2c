// Attention over a paged cache of int8 (kernel in paged_attn.h).
#include "paged_attn.h"

namespace marche {

hipError_t launch_paged_attention_int8(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s) {
  return launch_paged_fmt<I8>(dt, head_dim, a, s);
}

}  // namespace marche
