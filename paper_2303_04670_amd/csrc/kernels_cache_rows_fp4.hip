// Attention over a cache in 4 bits for few rows; see cache_attend_rows.h.
#include <algorithm>

#include "cache_attend_rows.h"

namespace evk {

void launch_attend_rows_fp4(const AttendParams& p, hipStream_t s) {
  if (p.a.dtype == EVCONV_BF16) start_rows<true, true>(p, s);
  else start_rows<true, false>(p, s);
}

}  // namespace evk
