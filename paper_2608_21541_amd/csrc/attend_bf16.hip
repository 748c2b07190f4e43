// Attention over a packed cache of bf16 rows (the kernel is in attend.h).
#include "attend.h"

namespace certkv {

certkv_status run_attend_bf16(const AttendArgs& a, hipStream_t s) {
  return a.g.D == 128 ? launch_attend_d<CERTKV_CACHE_BF16, 128>(a, s)
                      : launch_attend_d<CERTKV_CACHE_BF16, 64>(a, s);
}

}  // namespace certkv
