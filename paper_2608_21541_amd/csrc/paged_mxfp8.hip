// Attention over a paged cache of mxfp8 rows (the kernel is in paged.h).
#include "paged.h"

namespace certkv {

certkv_status run_paged_mxfp8(const PagedArgs& a, int shape, hipStream_t s) {
  return launch_paged<CERTKV_CACHE_MXFP8>(a, shape, s);
}

}  // namespace certkv
