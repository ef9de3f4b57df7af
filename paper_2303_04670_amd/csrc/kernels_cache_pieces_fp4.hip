// Attention over a cache in 4 bits for pieces of sequences; see cache_attend_pieces.h.
#include <algorithm>

#include "cache_attend_pieces.h"

namespace evk {

void launch_attend_pieces_fp4(const AttendParams& p, hipStream_t s) {
  if (p.a.dtype == EVCONV_BF16) start_pieces<true, true>(p, s);
  else start_pieces<true, false>(p, s);
}

}  // namespace evk
