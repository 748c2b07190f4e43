// Attention over a paged cache of mxfp4 rows (the kernel is in paged.h).
#include "paged.h"

namespace certkv {

certkv_status run_paged_mxfp4(const PagedArgs& a, int shape, hipStream_t s) {
  return launch_paged<CERTKV_CACHE_MXFP4>(a, shape, s);
}

}  // namespace certkv
