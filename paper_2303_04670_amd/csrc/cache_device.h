// Device helpers of the cache operators: whose a workgroup's tokens are, where they lie.
#pragma once

#include "ops_device.h"
#include "ops_kernels.h"

namespace evk {

// What a wave wrote to its own part of LDS it reads after this: the memory keeps the order, the compiler has to.
__device__ __forceinline__ void lds_turn() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// A piece of a sequence: its tokens are rows [first, first + count) of the call's, and `at` is the piece's number in it.
struct Piece {
  int seq, first, count, at;
};

__device__ __forceinline__ int offset_of(const evconv_tokens& t, int s) {
  return min(max(t.seq_offsets[s], 0), (int)t.n_tokens);
}

// Piece number `index` where sequences are cut into pieces of `div` of their tokens * num.  Equal lengths: `per` pieces each.  Lengths of
// their own (per < 0): sequence s has the numbers from (offset * num) / div + extra * s on, which leaves it as many as it can need and
// grows with s; the wave looks for the last s whose numbers start at or before `index`, 64 at a time.
__device__ __forceinline__ Piece find_piece(const evconv_tokens& t, int64_t index, int per, int64_t num, int div, int extra) {
  Piece p;
  if (per >= 0) {
    const int len = (int)(t.n_tokens / t.n_seq);
    p.seq = (int)(index / per);
    p.at = (int)(index - (int64_t)p.seq * per);
    p.first = p.seq * len;
    p.count = len;
    return p;
  }
  auto start = [&](int s) __attribute__((always_inline)) { return (int64_t)offset_of(t, s) * num / div + (int64_t)extra * s; };
  int lo = 0, n = t.n_seq;
  const int lane = threadIdx.x & 63;
  while (n > 1) {
    const int step = (n + 63) / 64, s = lo + lane * step;
    const bool before = lane * step < n && start(s) <= index;
    const int last = max((int)__popcll(__ballot(before)) - 1, 0);
    const int end = lo + n;
    lo += last * step;
    n = min(step, end - lo);
  }
  p.seq = __builtin_amdgcn_readfirstlane(lo);
  p.first = offset_of(t, p.seq);
  p.count = max(offset_of(t, p.seq + 1) - p.first, 0);
  p.at = (int)min(index - start(p.seq), (int64_t)INT32_MAX);
  return p;
}

// Page of table entry `entry` of sequence `seq`, or -1.
__device__ __forceinline__ int page_of(const evconv_cache& c, const evconv_tokens& t, int seq, int64_t entry) {
  if (entry < 0 || entry >= t.width) return -1;
  const int p = t.table[seq * t.table_stride + entry];
  return p >= 0 && p < c.n_pages ? p : -1;
}

}  // namespace evk
