// Attention over a packed cache of mxfp8 rows (the kernel is in attend.h).
#include "attend.h"

namespace certkv {

certkv_status run_attend_mxfp8(const AttendArgs& a, hipStream_t s) {
  return a.g.D == 128 ? launch_attend_d<CERTKV_CACHE_MXFP8, 128>(a, s)
                      : launch_attend_d<CERTKV_CACHE_MXFP8, 64>(a, s);
}

}  // namespace certkv
