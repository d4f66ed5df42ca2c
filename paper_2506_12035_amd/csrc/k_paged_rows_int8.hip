// Attention of many rows over a paged cache of int8 (kernel in paged_rows.h).
#include "paged_rows.h"

namespace marche {

hipError_t launch_paged_rows_int8(int32_t head_dim, const PagedAttnArgs &a, hipStream_t s) {
  return launch_paged_rows<I8>(head_dim, a, s);
}

}  // namespace marche
