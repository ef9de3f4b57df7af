// Attention over a cache in bf16 for pieces of sequences; see cache_attend_pieces.h.
#include <algorithm>

#include "cache_attend_pieces.h"

namespace evk {

void launch_attend_pieces_bf16(const AttendParams& p, hipStream_t s) {
  if (p.a.dtype == EVCONV_BF16) start_pieces<false, true>(p, s);
  else start_pieces<false, false>(p, s);
}

}  // namespace evk
