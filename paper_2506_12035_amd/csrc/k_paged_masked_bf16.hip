// Attention over windows and drafted trees in a paged cache of bf16 (kernel in paged_attn.h).
#include "paged_attn.h"

namespace marche {

hipError_t launch_paged_masked_bf16(DType dt, int32_t head_dim, const PagedAttnArgs &a, hipStream_t s) {
  return launch_paged_fmt<BF, true>(dt, head_dim, a, s);
}

}  // namespace marche
