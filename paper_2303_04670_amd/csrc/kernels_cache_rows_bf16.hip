// Attention over a cache in bf16 for few rows; see cache_attend_rows.h.
#include <algorithm>

#include "cache_attend_rows.h"

namespace evk {

void launch_attend_rows_bf16(const AttendParams& p, hipStream_t s) {
  if (p.a.dtype == EVCONV_BF16) start_rows<false, true>(p, s);
  else start_rows<false, false>(p, s);
}

}  // namespace evk
