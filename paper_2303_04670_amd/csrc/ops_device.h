// Device helpers that the sequence operators share: loads of fp32 or bf16 rows, values as bf16 parts.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace evk {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// fp32 -> bf16, round to nearest even, two values packed low / high
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  f32x2 v;
  v.x = lo;
  v.y = hi;
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, b16x2));
}
__device__ __forceinline__ float bf16_low(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_high(unsigned u) { return __uint_as_float(u & 0xffff0000u); }

template <bool BF16>
__device__ __forceinline__ float load_one(const void* q, int64_t i) {
  return BF16 ? __uint_as_float((unsigned)((const uint16_t*)q)[i] << 16) : ((const float*)q)[i];
}
__device__ __forceinline__ float load_any(const void* q, int64_t i, bool bf16) {
  return bf16 ? load_one<true>(q, i) : load_one<false>(q, i);
}
template <bool BF16>
__device__ __forceinline__ void store_one(void* q, int64_t i, float v) {
  if (BF16)
    ((uint16_t*)q)[i] = (uint16_t)pack_bf16(v, 0.0f);
  else
    ((float*)q)[i] = v;
}

// N (4 or a multiple of 8) values from element i on, zeros from `left` on.  VEC: the address is one of a
// wide load and `left` is a multiple of N or of 8, or not positive.
template <bool BF16, int N, bool VEC>
__device__ __forceinline__ void load_run(const void* q, int64_t i, int left, float (&v)[N]) {
  if constexpr (VEC && BF16) {
    constexpr int M = N < 8 ? N : 8;
#pragma unroll
    for (int c = 0; c < N; c += M) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (c < left) {
        if constexpr (M == 8) {
          u = *(const uint4*)((const uint16_t*)q + i + c);
        } else {
          const uint2 w = *(const uint2*)((const uint16_t*)q + i + c);
          u.x = w.x;
          u.y = w.y;
        }
      }
      const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < M; j += 2) {
        v[c + j] = bf16_low(w[j / 2]);
        v[c + j + 1] = bf16_high(w[j / 2]);
      }
    }
  } else if constexpr (VEC) {
#pragma unroll
    for (int c = 0; c < N; c += 4) {
      f32x4 u = {0, 0, 0, 0};
      if (c < left) u = *(const f32x4*)((const float*)q + i + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[c + j] = u[j];
    }
  } else {
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = c < left ? load_one<BF16>(q, i + c) : 0.0f;
  }
}

// Eight values as the sum of PARTS bf16 each: a part is the rounding of what the ones before it leave,
// so two hold 16 bits and three all 24 (of values of 2^-110 and more; smaller ones lose bits below 2^-133).
template <int PARTS>
__device__ __forceinline__ void split8(const float (&x)[8], b16x8 (&out)[PARTS]) {
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    uint4 u;
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = pack_bf16(r[2 * j], r[2 * j + 1]);
      if (q + 1 < PARTS) {
        r[2 * j] -= bf16_low(w[j]);
        r[2 * j + 1] -= bf16_high(w[j]);
      }
    }
    u.x = w[0]; u.y = w[1]; u.z = w[2]; u.w = w[3];
    out[q] = __builtin_bit_cast(b16x8, u);
  }
}

// acc[i] += a[i] b over operands of PA and PB parts, the smallest terms first; of the products of parts those
// whose places add up to at most ORDER (0: high * high) are taken: what ORDER 2 leaves out is less than 2^-24
// of a product, ORDER 1 less than 2^-15.  Neighbouring instructions are of different sums: one that continues the last one's
// would wait for it.
template <int ORDER, int N, int PA, int PB>
__device__ __forceinline__ void mfma_parts(f32x4* acc, const b16x8 (*a)[PA], const b16x8 (&b)[PB]) {
#pragma unroll
  for (int o = ORDER; o >= 0; --o)
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int j = o - i;
      if (j >= 0 && j < PB)
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n][i], b[j], acc[n], 0, 0, 0);
    }
}
template <int ORDER, int PA, int PB>
__device__ __forceinline__ void mfma_parts(f32x4& acc, const b16x8 (&a)[PA], const b16x8 (&b)[PB]) {
  mfma_parts<ORDER, 1>(&acc, &a, b);
}

}  // namespace evk
