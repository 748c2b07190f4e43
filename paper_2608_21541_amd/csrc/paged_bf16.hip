// Attention over a paged cache of bf16 rows (the kernel is in paged.h).
#include "paged.h"

namespace certkv {

certkv_status run_paged_bf16(const PagedArgs& a, int shape, hipStream_t s) {
  return launch_paged<CERTKV_CACHE_BF16>(a, shape, s);
}

}  // namespace certkv
