// Appending to a paged cache (evconv_cache_append) and reading it back (evconv_cache_read) on gfx950.
//
// A workgroup takes the call's tokens of one page, in pieces of 32 slots, and a group of the heads; of a piece it computes the
// rotation's cosines and sines once, in LDS, for all its heads (in 64 bits: some 150 instructions an angle, which 40 heads that
// did it for themselves would spend twice the copy's time on).  A wave then takes a head at a time, 16 channels to a lane: two vectors
// of eight that the rotation mixes, so that no lane needs another's.  Whole pages belong to one workgroup, so that bounds and half-filled bytes are read, changed and
// written by one wave.  8 x 4096 tokens of 32 query and 8 key heads of 128 in bf16 take 232 us, 3.5 TB/s (a copy as large: 4.8), vector
// instructions in 59 % of the cycles; 16 single tokens of 4 and 4 heads of 64 in fp32 5.6 us, the chain of a launch, two reads, a sum, the angles and a write.
//   Two vectors of a rotated pair in one lane instead of each in its own: 815 -> 286 us; bounds as 16-bit integers: 286 -> 235.  (More rows
// under way would be 220, but do not fit the 168 registers that leave room for three waves of a SIMD: nothing here may spill to memory; 95 scalar registers lie in vector lanes.)
#include <algorithm>

#include "cache_device.h"

namespace evk {
namespace {

constexpr int kPiece = 32;  // slots that are dealt with at once

struct AppendParams {
  evconv_append_args a;
  int dp, log;      // padded channels, log2 of the page
  double per_channel;  // 1 / d
  int per;          // pages that a sequence of equal lengths can reach, or -1
  int roles;        // heads of queries and of keys with their values together
  int per_group;    // of them, those of a workgroup
  int groups;       // workgroups that share the roles of a page
  int64_t block0;   // first workgroup of this launch
  bool single;      // one token of every sequence
};

// How the rows of a call are read and turned: anything, a value at a time; vectors, partners of the rotation in whole vectors (or no
// rotation); vectors, partners next to each other.
enum { kAnyRows, kHalves, kNeighbours };

template <int LANES>
__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
  return v;
}
template <int LANES>
__device__ __forceinline__ unsigned lanes_max(unsigned v) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) v = max(v, (unsigned)__shfl_xor((int)v, d));
  return v;
}

// 1 / sqrt(m) rounded to fp32, of m in 64 bits: the hardware's estimate (2^-26 and better) and two terms of the series of its error e,
// y (1 + e / 2 + 3 e^2 / 8), which leaves less than 2^-60.
__device__ __forceinline__ float inverse_root(double m) {
  const double y = __builtin_amdgcn_rsq(m);
  const double e = fma(-m * y, y, 1.0);
  return (float)fma(y * e, fma(e, 0.375, 0.5), y);
}

// Sine and cosine of an angle in 64 bits, rounded to fp32: the angle less the nearest multiple of pi / 2 (in two parts of 53 bits; their
// product with the multiple is exact in the fused operation as far as it counts), then the Taylor series, whose first terms left out are
// 2^-54 and 2^-49 at pi / 4.  Angles from 2^45 on, of which 64 bits hold less than 2^-8, are none.
__device__ __forceinline__ void sine_cosine(double angle, float& sine, float& cosine) {
  if (!(fabs(angle) < 0x1p45)) angle = 0.0;
  const double turns = rint(angle * 0.63661977236758134308);
  double r = fma(-turns, 1.57079632679489661923, angle);
  r = fma(-turns, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = fma(z, -1.0 / 1307674368000.0, 1.0 / 6227020800.0), c = fma(z, -1.0 / 87178291200.0, 1.0 / 479001600.0);
  s = fma(s, z, -1.0 / 39916800.0);
  c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, 1.0 / 362880.0);
  c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, -1.0 / 5040.0);
  c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, 1.0 / 120.0);
  c = fma(c, z, 1.0 / 24.0);
  s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, -0.5);
  s = fma(s * z, r, r);
  c = fma(c, z, 1.0);
  const int quarter = (int)((long long)turns & 3);
  const double u = quarter & 1 ? c : s, v = quarter & 1 ? s : c;
  sine = (float)(quarter & 2 ? -u : u);
  cosine = (float)(quarter == 1 || quarter == 2 ? -v : v);
}

// The channels of a lane: two vectors of eight, ch[0] and ch[1] on, with left[] of them inside (not positive: none).
struct Channels {
  int ch[2], left[2];
  int at[2];  // ch, inside the padded row
};
template <int MODE>
__device__ __forceinline__ Channels channels_of(const AppendParams& p, int l) {
  Channels c;
  c.ch[0] = 16 * l;
  c.ch[1] = c.ch[0] + 8;
  if (MODE == kHalves) {
    const int pairs = p.a.rot / 16;
    if (l < pairs) {
      c.ch[0] = 8 * l;
      c.ch[1] = p.a.rot / 2 + 8 * l;
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    c.left[i] = p.a.cache.d - c.ch[i];
    c.at[i] = min(c.ch[i], p.dp - 8);
  }
  return c;
}

// A row's two vectors.  (Vectors: what is outside is read inside, where it costs no branch, and set to zero.)
template <bool BF16, int MODE>
__device__ __forceinline__ void load_row(const void* src, int64_t at, const Channels& c, int d, float (&x)[2][8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (MODE == kAnyRows) {
      load_run<BF16, 8, false>(src, at + c.ch[i], c.left[i], x[i]);
    } else {
      load_run<BF16, 8, true>(src, at + min(c.ch[i], d - 8), 8, x[i]);
    }
  }
}
template <int MODE>
__device__ __forceinline__ void zero_outside(const Channels& c, float (&x)[2][8]) {
  if constexpr (MODE != kAnyRows)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c.left[i] <= 0) x[i][j] = 0.0f;
}

// Cosines and sines of a token's angles: a row of LDS, or computed where they are wanted.
struct SharedAngles {
  const float *cosines, *sines;
  __device__ __forceinline__ void one(int f, float& co, float& si) const { co = cosines[f], si = sines[f]; }
  __device__ __forceinline__ void eight(int f, float (&co)[8], float (&si)[8]) const {  // (f a multiple of eight, and the row's length)
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const f32x4 c = *(const f32x4*)(cosines + f + j), s = *(const f32x4*)(sines + f + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) co[j + k] = c[k], si[j + k] = s[k];
    }
  }
};
struct OwnAngles {
  double position;
  const float* freqs;
  __device__ __forceinline__ void one(int f, float& co, float& si) const { sine_cosine(position * (double)freqs[f], si, co); }
  __device__ __forceinline__ void eight(int f, float (&co)[8], float (&si)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) one(f + j, co[j], si[j]);
  }
};

// Norm and rotation of a row; `weight` has whole padded rows.  No contraction: each product and sum is rounded by itself, so
// that the codes of a 4-bit row do not depend on how the compiler joins them.
template <bool BF16, int MODE, int LANES, typename Angles>
__device__ __forceinline__ void turn_row(const AppendParams& p, const void* src, int64_t at, const Channels& c, bool norm, const float* weight,
                                         const Angles& angles, float (&x)[2][8]) {
#pragma clang fp contract(off)
  const int rot = p.a.rot, half = rot / 2;
  float scale = 1.0f;
  if (norm) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fma((double)x[i][j], (double)x[i][j], sum);
    scale = inverse_root(fma(lanes_sum<LANES>(sum), p.per_channel, (double)p.a.eps));
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        const f32x4 w = *(const f32x4*)(weight + c.at[i] + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[i][j + k] = x[i][j + k] * scale * w[k];
      }
  }
  if (!rot) return;
  if constexpr (MODE == kHalves) {
    if (c.ch[0] >= half) return;
    float co[8], si[8];
    angles.eight(c.ch[0], co, si);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = x[0][j], v = x[1][j];
      x[0][j] = u * co[j] - v * si[j];
      x[1][j] = v * co[j] + u * si[j];
    }
  } else if (MODE == kNeighbours || p.a.pairs == EVCONV_PAIRS_NEIGHBOURS) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; j += 2)
        if (c.ch[i] + j < rot) {
          float co, si;
          angles.one((c.ch[i] + j) / 2, co, si);
          const float u = x[i][j], v = x[i][j + 1];
          x[i][j] = u * co - v * si;
          x[i][j + 1] = v * co + u * si;
        }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int ch = c.ch[i] + j;
        if (ch >= rot) break;
        const bool low = ch < half;
        const int other = low ? ch + half : ch - half, f = low ? ch : other;
        float v = load_one<BF16>(src, at + other);
        if (norm) v = v * scale * weight[other];
        float co, si;
        angles.one(f, co, si);
        const float xc = x[i][j] * co, ys = v * si;
        x[i][j] = low ? xc - ys : xc + ys;
      }
  }
}

// Largest magnitude's bits of a row, over its lanes
template <int LANES>
__device__ __forceinline__ unsigned row_largest(const float (&x)[2][8]) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(x[i][j]) & 0x7fffffffu);
  return lanes_max<LANES>(m);
}
constexpr unsigned kNoBf16 = 0x7f7f8000u;  // magnitudes from these bits on are no finite bf16 numbers

// Eight 4-bit codes of a row whose largest magnitude has these bits, the first in the lowest bits.  The quotient is the
// correctly rounded one: values of bf16 rows often lie right between two codes.  (Near fp32's largest, 6 x would be infinite.)
__device__ __forceinline__ unsigned codes_of(const float (&x)[8], unsigned largest) {
#pragma clang fp contract(off)
  if (largest == 0 || largest >= kNoBf16) return 0;
  const float shift = largest > 0x7e000000u ? 0x1p-10f : 1.0f, m = __uint_as_float(largest) * shift;
  unsigned w = 0;
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = 6.0f * (x[j] * shift) / m;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
  return w;
}
__device__ __forceinline__ float scale_of(unsigned largest) { return largest >= kNoBf16 ? NAN : __uint_as_float(largest) / 6.0f; }

template <bool VEC>
__device__ __forceinline__ void store_row(void* q, int64_t at, int ch, int left, const float (&x)[8], bool bf16) {
  if (left <= 0) return;
  if (VEC) {
    if (bf16) {
      *(uint4*)((uint16_t*)q + at + ch) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
      *(f32x4*)((float*)q + at + ch) = f32x4{x[0], x[1], x[2], x[3]};
      *(f32x4*)((float*)q + at + ch + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) {
        if (bf16) store_one<true>(q, at + ch + j, x[j]);
        else store_one<false>(q, at + ch + j, x[j]);
      }
  }
}

// Bytes of a channel's row of a piece of values in LDS: 32 bf16 or 32 codes, and four more, so that the eight channels of a lane
// and those of its neighbours do not meet in a bank.
__host__ __device__ constexpr int value_row(bool fp4) { return (fp4 ? 1 : 2) * kPiece + 4; }

// Least and largest of keys, two to a word: bf16 numbers as 16-bit integers of the same order.  What is no number counts as beyond both
// ends, and becomes one again.
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ i16x2 ordered(unsigned two) {
  const i16x2 v = __builtin_bit_cast(i16x2, two);
  return v ^ ((v >> 15) & (short)0x7fff);
}
__device__ __forceinline__ unsigned as_bf16(i16x2 v) { return __builtin_bit_cast(unsigned, v ^ ((v >> 15) & (short)0x7fff)); }
struct Bounds {
  i16x2 lo[2][4], hi[2][4];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) lo[h][j] = 32767, hi[h][j] = -32768;
  }
  __device__ __forceinline__ void add(int h, int j, i16x2 l, i16x2 u) {
    lo[h][j] = __builtin_elementwise_min(lo[h][j], l);
    hi[h][j] = __builtin_elementwise_max(hi[h][j], u);
  }
  // A key's eight values, as the cache in bf16 has them; of a row that is marked the numbers are none.
  __device__ __forceinline__ void add_key(int h, const unsigned (&w)[4], bool bad) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const i16x2 v = ordered(w[j]);
      const bool low = bad && (w[j] & 0x7fffu) > 0x7f80u, high = bad && (w[j] >> 16 & 0x7fffu) > 0x7f80u;
      i16x2 l = v, u = v;
      if (low) l.x = -32768, u.x = 32767;
      if (high) l.y = -32768, u.y = 32767;
      add(h, j, l, u);
    }
  }
  // Those that a page had: numbers, or none in both.
  __device__ __forceinline__ void add_old(int h, const uint4& low, const uint4& high) {
    const unsigned l[4] = {low.x, low.y, low.z, low.w}, u[4] = {high.x, high.y, high.z, high.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      i16x2 a = ordered(l[j]), b = ordered(u[j]);
      if ((l[j] & 0x7fffu) > 0x7f80u) a.x = -32768, b.x = 32767;
      if ((l[j] >> 16 & 0x7fffu) > 0x7f80u) a.y = -32768, b.y = 32767;
      add(h, j, a, b);
    }
  }
  __device__ __forceinline__ uint4 low(int h) const { return make_uint4(as_bf16(lo[h][0]), as_bf16(lo[h][1]), as_bf16(lo[h][2]), as_bf16(lo[h][3])); }
  __device__ __forceinline__ uint4 high(int h) const { return make_uint4(as_bf16(hi[h][0]), as_bf16(hi[h][1]), as_bf16(hi[h][2]), as_bf16(hi[h][3])); }
};

template <bool BF16, bool FP4, int MODE, int LANES>
__global__ __launch_bounds__(256, MODE == kAnyRows ? 1 : 3) void cache_append(AppendParams p) {
  constexpr bool VEC = MODE != kAnyRows;
  constexpr int ROWS = 64 / LANES;                    // tokens that a wave deals with at once
  constexpr int AT_ONCE = !VEC || LANES < 4 ? 1 : 2;  // ... has under way, of a query head, times that
  extern __shared__ __align__(16) char s_mem[];
  const evconv_append_args& a = p.a;
  const evconv_cache& c = a.cache;
  const evconv_tokens& tk = a.tokens;
  const int64_t block = p.block0 + blockIdx.x;
  const int group = (int)(block % p.groups);
  const Piece piece = find_piece(tk, block / p.groups, p.per, 1, c.page, 2);
  const int past = tk.past[piece.seq], d = c.d, half = a.rot / 2;
  const int64_t page = ((int64_t)past >> p.log) + piece.at;  // (rounds down for negative ones too)
  const int64_t begin = max((int64_t)past, page << p.log), end = min((int64_t)past + piece.count, (page + 1) << p.log);
  if (begin >= end) return;
  const int to = page_of(c, tk, piece.seq, page);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int row = lane / LANES;
  const Channels own = channels_of<MODE>(p, lane % LANES);
  float* const s_cos = (float*)s_mem;
  float* const s_sin = s_cos + kPiece * half;
  char* const s_v = s_mem + 2 * sizeof(float) * (kPiece * half + p.dp) + wave * p.dp * value_row(FP4);
  const int role_end = min((group + 1) * p.per_group, p.roles);
  float* const s_wq = (float*)(s_mem + 2 * sizeof(float) * kPiece * half);  // weights of the norms, zeros behind them
  float* const s_wk = s_wq + p.dp;
  for (int i = threadIdx.x; i < p.dp; i += blockDim.x) {
    s_wq[i] = a.q_norm && i < d ? a.q_norm[i] : 0.0f;
    s_wk[i] = a.k_norm && i < d ? a.k_norm[i] : 0.0f;
  }
  for (int64_t sub = begin & ~(int64_t)(kPiece - 1); sub < end; sub += kPiece) {
    const int64_t from = max(sub, begin);
    const int count = (int)(min(sub + kPiece, end) - from), token = piece.first + (int)(from - past);
    const int slot = (int)(from & (c.page - 1));
    __syncthreads();  // (the last piece's angles have been read)
    for (int i = threadIdx.x; i < count * half; i += blockDim.x) {
      const int r = i / half, f = i - r * half;
      sine_cosine((double)(a.positions ? a.positions[token + r] : from + r) * (double)a.freqs[f], s_sin[i], s_cos[i]);
    }
    __syncthreads();
    int role = group * p.per_group + wave;
    for (; role < min(role_end, a.heads_q); role += waves) {  // ---- a head of the queries
      const int64_t head_in = role * a.q.head_stride, head_out = role * a.q_out_head_stride;
      for (int r0 = 0; r0 < count; r0 += AT_ONCE * ROWS) {
        float x[AT_ONCE][2][8];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          const int r = min(r0 + i * ROWS + row, count - 1);
          load_row<BF16, MODE>(a.q.data, (token + r) * a.q.token_stride + head_in, own, d, x[i]);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          if (r0 + i * ROWS >= count) break;
          const int r = r0 + i * ROWS + row, r_in = min(r, count - 1);
          zero_outside<MODE>(own, x[i]);
          turn_row<BF16, MODE, LANES>(p, a.q.data, (token + r_in) * a.q.token_stride + head_in, own, a.q_norm, s_wq, SharedAngles{s_cos + r_in * half, s_sin + r_in * half}, x[i]);
          const int64_t at = (token + r_in) * a.q_out_token_stride + head_out;
#pragma unroll
          for (int h = 0; h < 2; ++h) store_row<VEC>(a.q_out, at, own.ch[h], r < count ? own.left[h] : 0, x[i][h], BF16);
        }
      }
    }
    for (; role < role_end && to >= 0; role += waves) {  // ---- a head of the keys and the values
      const int head = role - a.heads_q;
      const int64_t at = ((int64_t)to * c.heads + head) * c.page;  // tokens before this head's of the page
      const int64_t k_head = head * a.k.head_stride, v_head = head * a.v.head_stride;
      Bounds bounds;
      bounds.clear();
      for (int r0 = 0; r0 < count; r0 += ROWS) {
        const int r = r0 + row, r_in = min(r, count - 1);
        const bool live = r < count;
        const int64_t k_row = (token + r_in) * a.k.token_stride + k_head;
        float x[2][8], v[2][8];
        load_row<BF16, MODE>(a.k.data, k_row, own, d, x);
        load_row<BF16, MODE>(a.v.data, (token + r_in) * a.v.token_stride + v_head, own, d, v);
        zero_outside<MODE>(own, x);
        zero_outside<MODE>(own, v);
        turn_row<BF16, MODE, LANES>(p, a.k.data, k_row, own, a.k_norm, s_wk, SharedAngles{s_cos + r_in * half, s_sin + r_in * half}, x);
        const unsigned big_k = row_largest<LANES>(x), big_v = row_largest<LANES>(v);
        const bool bad = big_k >= kNoBf16 || (!FP4 && big_v >= kNoBf16);
        if (bad)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (j < own.left[h]) x[h][j] = NAN;
        if (!live) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int ch = own.ch[h];
          if (ch >= p.dp) continue;
          const unsigned kw[4] = {pack_bf16(x[h][0], x[h][1]), pack_bf16(x[h][2], x[h][3]), pack_bf16(x[h][4], x[h][5]), pack_bf16(x[h][6], x[h][7])};
          bounds.add_key(h, kw, bad);
          if constexpr (FP4) {
            const unsigned v4 = codes_of(v[h], big_v);
            *(unsigned*)((char*)c.k + (at + slot + r) * (p.dp / 2) + ch / 2) = codes_of(x[h], big_k);
#pragma unroll
            for (int j = 0; j < 8; ++j) s_v[(ch + j) * value_row(true) + slot % kPiece + r] = (char)(v4 >> (4 * j) & 15);
            if (ch == 0) {
              c.k_scale[at + slot + r] = scale_of(big_k);
              c.v_scale[at + slot + r] = scale_of(big_v);
            }
          } else {
            *(uint4*)((uint16_t*)c.k + (at + slot + r) * p.dp + ch) = make_uint4(kw[0], kw[1], kw[2], kw[3]);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              unsigned w = pack_bf16(v[h][j], v[h][j + 1]);
              if (big_v >= kNoBf16) {  // (no value of v that is not finite)
                if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
                if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
              }
              *(uint16_t*)(s_v + (ch + j) * value_row(false) + 2 * (slot % kPiece + r)) = (uint16_t)w;
              *(uint16_t*)(s_v + (ch + j + 1) * value_row(false) + 2 * (slot % kPiece + r)) = (uint16_t)(w >> 16);
            }
          }
        }
      }
      lds_turn();
      // ---- the values' rows of channels
      char* const v_rows = (char*)c.v + ((int64_t)to * c.heads + head) * p.dp * c.page * 2 / (FP4 ? 4 : 1);
      if constexpr (FP4) {
        // a lane to a channel: 16 bytes of 32 tokens; of those that are not this call's the bits stay
        const int first = slot % kPiece;
        for (int k = lane; k < p.dp; k += 64) {
          uint4* const q = (uint4*)(v_rows + ((int64_t)k * c.page + slot - first) / 2);
          const unsigned* const row32 = (const unsigned*)(s_v + k * value_row(true));
          uint4 old = make_uint4(0, 0, 0, 0);
          if (count < kPiece) old = *q;
          unsigned w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned u0 = row32[2 * i], u1 = row32[2 * i + 1];  // four codes each, a byte a code
            unsigned n = (u0 & 15) | (u0 >> 4 & 0xf0) | (u0 >> 8 & 0xf00) | (u0 >> 12 & 0xf000);
            n |= ((u1 & 15) | (u1 >> 4 & 0xf0) | (u1 >> 8 & 0xf00) | (u1 >> 12 & 0xf000)) << 16;
            const int b = min(max(first - 8 * i, 0), 8), e = min(max(first + count - 8 * i, 0), 8);
            const unsigned mask = e > b ? (unsigned)((1ull << (4 * e)) - (1ull << (4 * b))) : 0u;
            w[i] = (w[i] & ~mask) | (n & mask);
          }
          *q = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else if (count == kPiece) {
        for (int i = lane; i < p.dp * 4; i += 64) {
          const int k = i / 4, part = i % 4;
          const unsigned* const row32 = (const unsigned*)(s_v + k * value_row(false)) + 4 * part;
          *(uint4*)(v_rows + ((int64_t)k * c.page + slot + 8 * part) * 2) = make_uint4(row32[0], row32[1], row32[2], row32[3]);
        }
      } else {  // the call's tokens alone
        const int first = slot % kPiece, t = lane % kPiece;
        if (t >= first && t < first + count)
          for (int k = lane / kPiece; k < p.dp; k += 64 / kPiece)
            *(uint16_t*)(v_rows + ((int64_t)k * c.page + slot - first + t) * 2) = *(const uint16_t*)(s_v + k * value_row(false) + 2 * t);
      }
      lds_turn();
      // ---- bounds: over the piece's tokens, then with what the page had unless it begins here
      if (!c.bounds) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int s = LANES; s < 64; s *= 2)
            bounds.add(h, j, __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, bounds.lo[h][j]), s)),
                       __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, bounds.hi[h][j]), s)));
        if (row == 0 && own.ch[h] < p.dp) {
          uint4* const q = (uint4*)((uint16_t*)c.bounds + (((int64_t)to * c.heads + head) * 2) * p.dp + own.ch[h]);
          uint4* const q_hi = (uint4*)((uint16_t*)q + p.dp);
          if (slot > 0) bounds.add_old(h, *q, *q_hi);
          *q = bounds.low(h);
          *q_hi = bounds.high(h);
        }
      }
    }
  }
}

// One new token of every sequence: a wave to a head of 64 / LANES of them, each lane with its own angles, nothing shared: no barrier and no
// second round of anything, since all that such a call takes is the chain from the launch to the last write.
template <bool BF16, bool FP4, int MODE, int LANES>
__global__ __launch_bounds__(64) void append_single(AppendParams p) {
  constexpr bool VEC = MODE != kAnyRows;
  constexpr int ROWS = 64 / LANES;
  __shared__ float s_weight[256];
  const evconv_append_args& a = p.a;
  const evconv_cache& c = a.cache;
  const evconv_tokens& tk = a.tokens;
  const int64_t block = p.block0 + blockIdx.x;
  const int lane = threadIdx.x, d = c.d, role = (int)(block % p.roles);
  const int64_t t0 = block / p.roles * ROWS + lane / LANES;
  const bool live = t0 < tk.n_tokens;
  const int64_t token = min(t0, tk.n_tokens - 1);
  const Channels own = channels_of<MODE>(p, lane % LANES);
  const bool query = role < a.heads_q;
  const evconv_heads& src = query ? a.q : a.k;
  const int head = query ? role : role - a.heads_q;
  const int64_t row = token * src.token_stride + head * src.head_stride;
  const float* const norm = query ? a.q_norm : a.k_norm;
  float x[2][8], v[2][8];
  load_row<BF16, MODE>(src.data, row, own, d, x);
  if (!query) load_row<BF16, MODE>(a.v.data, token * a.v.token_stride + head * a.v.head_stride, own, d, v);
  const int past = tk.past[token];
  if (norm)
    for (int i = lane; i < p.dp; i += 64) s_weight[i] = i < d ? norm[i] : 0.0f;
  lds_turn();
  const double position = (double)(a.positions ? a.positions[token] : (int64_t)past);
  const int to = past < 0 ? -1 : page_of(c, tk, (int)token, past >> p.log);
  zero_outside<MODE>(own, x);
  turn_row<BF16, MODE, LANES>(p, src.data, row, own, norm, s_weight, OwnAngles{position, a.freqs}, x);
  if (query) {
    const int64_t at = token * a.q_out_token_stride + head * a.q_out_head_stride;
#pragma unroll
    for (int h = 0; h < 2; ++h) store_row<VEC>(a.q_out, at, own.ch[h], live ? own.left[h] : 0, x[h], BF16);
    return;
  }
  zero_outside<MODE>(own, v);
  const unsigned big_k = row_largest<LANES>(x), big_v = row_largest<LANES>(v);
  const bool bad = big_k >= kNoBf16 || (!FP4 && big_v >= kNoBf16);
  if (bad)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < own.left[h]) x[h][j] = NAN;
  if (!live || to < 0) return;
  const int slot = past & (c.page - 1);
  const int64_t at = ((int64_t)to * c.heads + head) * c.page + slot, column = ((int64_t)to * c.heads + head) * p.dp;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int ch = own.ch[h];
    if (ch >= p.dp) continue;
    const unsigned kw[4] = {pack_bf16(x[h][0], x[h][1]), pack_bf16(x[h][2], x[h][3]), pack_bf16(x[h][4], x[h][5]), pack_bf16(x[h][6], x[h][7])};
    if constexpr (FP4) {
      uint8_t* const q = (uint8_t*)c.v + (column + ch) * (c.page / 2) + slot / 2;
      unsigned old[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) old[j] = q[j * (c.page / 2)];
      const unsigned v4 = codes_of(v[h], big_v);
      const int shift = slot % 2 * 4;
      *(unsigned*)((char*)c.k + at * (p.dp / 2) + ch / 2) = codes_of(x[h], big_k);
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j * (c.page / 2)] = (uint8_t)((old[j] & (0xf0u >> shift)) | (v4 >> (4 * j) & 15) << shift);
      if (ch == 0) {
        c.k_scale[at] = scale_of(big_k);
        c.v_scale[at] = scale_of(big_v);
      }
    } else {
      *(uint4*)((uint16_t*)c.k + at * p.dp + ch) = make_uint4(kw[0], kw[1], kw[2], kw[3]);
      uint16_t* const q = (uint16_t*)c.v + (column + ch) * c.page + slot;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned w = pack_bf16(v[h][j], 0.0f) & 0xffffu;
        q[j * c.page] = (uint16_t)((w & 0x7f80u) == 0x7f80u ? 0 : w);
      }
    }
    if (c.bounds) {
      uint4* const q = (uint4*)((uint16_t*)c.bounds + 2 * column + ch);
      uint4* const q_hi = (uint4*)((uint16_t*)q + p.dp);
      Bounds bounds;
      bounds.clear();
      bounds.add_key(h, kw, bad);
      if (slot > 0) bounds.add_old(h, *q, *q_hi);
      *q = bounds.low(h);
      *q_hi = bounds.high(h);
    }
  }
}

// Rows back: a thread to eight channels of a token's key and value.
struct ReadParams {
  evconv_read_args a;
  int dp, log, pieces;  // vectors of a row
  int len;              // tokens of every sequence, or -1
  int64_t block0;
};

template <bool BF16, bool FP4>
__global__ __launch_bounds__(256) void cache_read(ReadParams p) {
  const evconv_read_args& a = p.a;
  const evconv_cache& c = a.cache;
  const int64_t t = p.block0 + blockIdx.x;  // a workgroup to a token
  const Piece piece = find_piece(a.tokens, t, p.len, 1, 1, 0);
  const int within = (int)t - piece.first;
  if (within < 0 || within >= piece.count) return;
  const int64_t position = (int64_t)a.tokens.past[piece.seq] + within;
  const int from = position < 0 ? -1 : page_of(c, a.tokens, piece.seq, position >> p.log);
  const int slot = (int)(position & (c.page - 1));
  for (int i = threadIdx.x; i < c.heads * p.pieces; i += blockDim.x) {
    const int head = i / p.pieces, ch = i % p.pieces * 8, left = min(c.d - ch, 8);
    float k[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = v[j] = 0.0f;
    if (from >= 0) {
      const int64_t row = ((int64_t)from * c.heads + head) * c.page + slot, column = ((int64_t)from * c.heads + head) * p.dp + ch;
      if constexpr (FP4) {
        const unsigned w = *(const unsigned*)((const char*)c.k + row * (p.dp / 2) + ch / 2);
        const float ks = c.k_scale[row], vs = c.v_scale[row];
        auto value = [](unsigned code) __attribute__((always_inline)) {
          const int e = code >> 1 & 3, f = code & 1;
          const float m = e ? (float)((2 + f) << (e - 1)) * 0.5f : 0.5f * (float)f;
          return code & 8 ? -m : m;
        };
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          k[j] = value(w >> (4 * j) & 15) * ks;
          v[j] = value((unsigned)((const uint8_t*)c.v)[(column + j) * (c.page / 2) + slot / 2] >> (slot % 2 * 4) & 15) * vs;
        }
      } else {
        load_run<true, 8, true>(c.k, row * p.dp + ch, 8, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = load_one<true>(c.v, (column + j) * c.page + slot);
      }
    }
    const int64_t at = (t * c.heads + head) * c.d + ch;
    for (int j = 0; j < left; ++j) {
      store_one<BF16>(a.k, at + j, k[j]);
      store_one<BF16>(a.v, at + j, v[j]);
    }
  }
}

template <bool BF16, bool FP4, int MODE, int LANES>
void start_append(AppendParams p, int64_t blocks, hipStream_t s) {
  if (p.single) {
    const int64_t blocks_single = (p.a.tokens.n_tokens + 64 / LANES - 1) / (64 / LANES) * p.roles, most = kMostThreads / 64;
    for (; p.block0 < blocks_single; p.block0 += most)
      append_single<BF16, FP4, MODE, LANES><<<(unsigned)std::min(most, blocks_single - p.block0), 64, 0, s>>>(p);
    return;
  }
  const size_t lds = 2 * sizeof(float) * (kPiece * (p.a.rot / 2) + p.dp) + 4 * p.dp * value_row(FP4);
  const int64_t most = kMostThreads / 256;
  for (; p.block0 < blocks; p.block0 += most)
    cache_append<BF16, FP4, MODE, LANES><<<(unsigned)std::min(most, blocks - p.block0), 256, lds, s>>>(p);
}
// Lanes of a row: the power of two that holds its channels by sixteens.
template <bool BF16, bool FP4, int MODE>
void start_append(const AppendParams& p, int64_t blocks, hipStream_t s) {
  if (p.dp <= 32) start_append<BF16, FP4, MODE, 2>(p, blocks, s);
  else if (p.dp <= 64) start_append<BF16, FP4, MODE, 4>(p, blocks, s);
  else if (p.dp <= 128) start_append<BF16, FP4, MODE, 8>(p, blocks, s);
  else start_append<BF16, FP4, MODE, 16>(p, blocks, s);
}
template <bool BF16, bool FP4>
void start_append(const AppendParams& p, bool vec, int64_t blocks, hipStream_t s) {
  if (vec && p.a.rot && p.a.pairs == EVCONV_PAIRS_NEIGHBOURS) start_append<BF16, FP4, kNeighbours>(p, blocks, s);
  else if (vec && p.a.rot % 16 == 0) start_append<BF16, FP4, kHalves>(p, blocks, s);
  else start_append<BF16, FP4, kAnyRows>(p, blocks, s);
}

}  // namespace

void launch_cache_append(const evconv_append_args& a, bool vec, hipStream_t s) {
  AppendParams p{};
  p.a = a;
  p.dp = cache_channels(a.cache.d);
  p.log = __builtin_ctz(a.cache.page);
  p.per_channel = 1.0 / a.cache.d;
  const evconv_tokens& t = a.tokens;
  p.per = t.seq_offsets ? -1 : (int)((t.n_tokens / t.n_seq + a.cache.page - 2) / a.cache.page) + 1;
  p.roles = a.heads_q + a.cache.heads;
  p.single = !t.seq_offsets && t.n_tokens == t.n_seq;
  const int64_t pages = p.per >= 0 ? (int64_t)p.per * t.n_seq : t.n_tokens / a.cache.page + 2 * (int64_t)t.n_seq;
  // Workgroups of a page: as many as fill the chip a few times over, each with whole rounds of roles for its four waves.  (More compute the
  // angles more often; 8 x 4096 tokens of 40 roles, us: 3 groups 275, 5 237, 10 247.)
  const int64_t rounds = (p.roles + 3) / 4;
  p.per_group = 4 * (int)std::max<int64_t>(1, std::min(rounds, rounds * pages / 2048));
  p.groups = (p.roles + p.per_group - 1) / p.per_group;
  const int64_t blocks = pages * p.groups;
  const bool fp4 = a.cache.kind == EVCONV_CACHE_FP4;
  if (a.dtype == EVCONV_BF16) fp4 ? start_append<true, true>(p, vec, blocks, s) : start_append<true, false>(p, vec, blocks, s);
  else fp4 ? start_append<false, true>(p, vec, blocks, s) : start_append<false, false>(p, vec, blocks, s);
}

void launch_cache_read(const evconv_read_args& a, hipStream_t s) {
  ReadParams p{};
  p.a = a;
  p.dp = cache_channels(a.cache.d);
  p.log = __builtin_ctz(a.cache.page);
  p.pieces = (a.cache.d + 7) / 8;
  p.len = a.tokens.seq_offsets ? -1 : (int)(a.tokens.n_tokens / a.tokens.n_seq);
  const bool fp4 = a.cache.kind == EVCONV_CACHE_FP4, bf16 = a.dtype == EVCONV_BF16;
  const int64_t most = kMostThreads / 256;
  for (; p.block0 < a.tokens.n_tokens; p.block0 += most) {
    const unsigned grid = (unsigned)std::min(most, a.tokens.n_tokens - p.block0);
    if (bf16) fp4 ? cache_read<true, true><<<grid, 256, 0, s>>>(p) : cache_read<true, false><<<grid, 256, 0, s>>>(p);
    else fp4 ? cache_read<false, true><<<grid, 256, 0, s>>>(p) : cache_read<false, false><<<grid, 256, 0, s>>>(p);
  }
}

}  // namespace evk
