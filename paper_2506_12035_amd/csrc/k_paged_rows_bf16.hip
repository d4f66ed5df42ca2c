// Attention of many rows over a paged cache of bf16 (kernel in paged_rows.h).
#include "paged_rows.h"

namespace marche {

hipError_t launch_paged_rows_bf16(int32_t head_dim, const PagedAttnArgs &a, hipStream_t s) {
  return launch_paged_rows<BF>(head_dim, a, s);
}

}  // namespace marche
