// Arithmetic of the choice among a row of pages: the range of keys that the last chosen one is in, cut into equal parts until a
// part is one key or has few.  Plain C++ (constexpr functions are device functions, too), so that it can be checked on the host.
#pragma once

namespace evk {

constexpr unsigned kForced = 0xffffffffu, kNotANumber = 0xfffffffeu;  // keys above those of all numbers
constexpr int kKeyParts = 2048;

struct KeyRange {
  unsigned lo, hi;  // both inside, lo <= hi
};

// log2 of the keys to a part, such that kKeyParts parts hold the range, and how many parts there are.
constexpr int part_shift(KeyRange r) {
  const unsigned span = r.hi - r.lo;
  const int bits = 32 - __builtin_clz(span > 1 ? span : 1);
  return bits > 11 ? bits - 11 : 0;
}
constexpr int part_count(KeyRange r, int shift) { return (int)((r.hi - r.lo) >> shift) + 1; }

// The keys of one of them.  (The topmost part may reach behind 2^32, so that distances are compared and not ends.)
constexpr KeyRange part_range(KeyRange r, int shift, int part) {
  const unsigned lo = r.lo + ((unsigned)part << shift), most = (1u << shift) - 1;
  return KeyRange{lo, r.hi - lo > most ? lo + most : r.hi};
}

}  // namespace evk
