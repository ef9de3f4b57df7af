// Appending to a paged cache (evconv_cache_append) and reading it back (evconv_cache_read) on gfx950.
//
// A workgroup takes the call's tokens of one page, in pieces of 32 slots, and a group of the heads; of a piece it computes the
// rotation's cosines and sines once, in LDS, for all its heads (in 64 bits: some 150 instructions an angle, which 40 heads that
// did it for themselves would spend twice the copy's time on).  A wave then takes a head at a time: eight channels to a
// lane, 64 / lanes tokens at once.  Whole pages belong to one workgroup, so that bounds and half-filled bytes are read, changed and
// written by one wave.  Bound by the rows' bytes; for single tokens by the chain of a launch, a search, a read, two sums and a write.
#include <algorithm>

#include "cache_device.h"

namespace evk {
namespace {

constexpr int kPiece = 32;  // slots that are dealt with at once

struct AppendParams {
  evconv_append_args a;
  int dp, log;      // padded channels, log2 of the page
  int lanes;        // of a row: the power of two that holds dp / 8
  int per;          // pages that a sequence of equal lengths can reach, or -1
  int roles;        // heads of queries and of keys with their values together
  int groups;       // workgroups that share the roles of a page
  int64_t block0;   // first workgroup of this launch
  bool pairs_wide;  // partners of rotated channels in whole vectors
};

__device__ __forceinline__ double lanes_sum(double v, int lanes) {
  for (int d = 1; d < lanes; d *= 2) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ unsigned lanes_max(unsigned v, int lanes) {
  for (int d = 1; d < lanes; d *= 2) v = max(v, (unsigned)__shfl_xor((int)v, d));
  return v;
}

// 1 / sqrt(m) rounded to fp32, of m in 64 bits (positive): the hardware's estimate and two terms of the series of its error e,
// y (1 + e / 2 + 3 e^2 / 8), which leaves 2^-60.
__device__ __forceinline__ float inverse_root(double m) {
  if (!(m > 1e-37 && m < 1e37)) return (float)(1.0 / sqrt(m));
  const double y = (double)__builtin_amdgcn_rsqf((float)m);
  const double e = 1.0 - m * y * y;
  return (float)(y + y * e * (0.5 + 0.375 * e));
}

// Norm and rotation of eight channels from `ch` on of one row.  No contraction: each product and sum is rounded by itself, so that
// the codes of a 4-bit row do not depend on how the compiler joins them.
template <bool BF16, bool VEC>
__device__ __forceinline__ void head_row(const AppendParams& p, const void* src, int64_t at, int ch, int left, const float* weight, const float* cosines,
                                         const float* sines, float (&x)[8]) {
#pragma clang fp contract(off)
  load_run<BF16, 8, VEC>(src, at + ch, left, x);
  const int rot = p.a.rot, half = rot / 2;
  float scale = 1.0f;
  if (weight) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += (double)x[j] * (double)x[j];
    sum = lanes_sum(sum, p.lanes);
    scale = inverse_root(sum / (double)p.a.cache.d + (double)p.a.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) x[j] = x[j] * scale * weight[ch + j];
  }
  if (ch >= rot) return;
  if (p.a.pairs == EVCONV_PAIRS_NEIGHBOURS) {
#pragma unroll
    for (int j = 0; j < 8; j += 2)
      if (ch + j < rot) {
        const float c = cosines[(ch + j) / 2], s = sines[(ch + j) / 2], u = x[j], v = x[j + 1];
        x[j] = u * c - v * s;
        x[j + 1] = v * c + u * s;
      }
    return;
  }
  if (p.pairs_wide) {  // a vector is of one half
    const bool low = ch < half;
    const int other = low ? ch + half : ch - half, f = low ? ch : other;
    float y[8];
    load_run<BF16, 8, VEC>(src, at + other, 8, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (weight) y[j] = y[j] * scale * weight[other + j];
      const float c = cosines[f + j], s = sines[f + j];
      const float xc = x[j] * c, ys = y[j] * s;
      x[j] = low ? xc - ys : xc + ys;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (ch + j >= rot) break;
    const bool low = ch + j < half;
    const int other = low ? ch + j + half : ch + j - half, f = low ? ch + j : other;
    float y = load_one<BF16>(src, at + other);
    if (weight) y = y * scale * weight[other];
    const float xc = x[j] * cosines[f], ys = y * sines[f];
    x[j] = low ? xc - ys : xc + ys;
  }
}

// Largest magnitude's bits of a row, over its lanes
__device__ __forceinline__ unsigned row_largest(const float (&x)[8], int lanes) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
  return lanes_max(m, lanes);
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

template <bool BF16, bool FP4, bool VEC>
__global__ __launch_bounds__(256) void cache_append(AppendParams p) {
  extern __shared__ char s_mem[];
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
  const int rows = 64 / p.lanes, row = lane / p.lanes, ch = lane % p.lanes * 8, left = d - ch;
  float* const s_cos = (float*)s_mem;
  float* const s_sin = s_cos + kPiece * half;
  char* const s_v = s_mem + 2 * sizeof(float) * kPiece * half + wave * p.dp * value_row(FP4);
  const int per_group = (p.roles + p.groups - 1) / p.groups, role_end = min((group + 1) * per_group, p.roles);
  for (int64_t sub = begin & ~(int64_t)(kPiece - 1); sub < end; sub += kPiece) {
    const int64_t from = max(sub, begin);
    const int count = (int)(min(sub + kPiece, end) - from), token = piece.first + (int)(from - past);
    const int slot = (int)(from & (c.page - 1));
    __syncthreads();  // (the last piece's angles have been read)
    for (int i = threadIdx.x; i < count * half; i += blockDim.x) {
      const int r = i / half, f = i - r * half;
      double s, co;
      sincos((double)(a.positions ? a.positions[token + r] : from + r) * (double)a.freqs[f], &s, &co);
      s_cos[i] = (float)co;
      s_sin[i] = (float)s;
    }
    __syncthreads();
    for (int role = group * per_group + wave; role < role_end; role += waves) {
      if (role < a.heads_q) {  // ---- a head of the queries
        for (int r0 = 0; r0 < count; r0 += rows) {
          const int r = r0 + row;
          const bool live = r < count;
          const int64_t t = token + (live ? r : 0);
          float x[8];
          head_row<BF16, VEC>(p, a.q.data, t * a.q.token_stride + role * a.q.head_stride, ch, live ? left : 0, a.q_norm, s_cos + (live ? r : 0) * half,
                              s_sin + (live ? r : 0) * half, x);
          store_row<VEC>(a.q_out, t * a.q_out_token_stride + role * a.q_out_head_stride, ch, live ? left : 0, x, BF16);
        }
        continue;
      }
      // ---- a head of the keys and the values
      if (to < 0) continue;
      const int head = role - a.heads_q;
      const int64_t at = ((int64_t)to * c.heads + head) * c.page;  // tokens before this head's of the page
      float lo[8], hi[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) lo[j] = INFINITY, hi[j] = -INFINITY;
      for (int r0 = 0; r0 < count; r0 += rows) {
        const int r = r0 + row;
        const bool live = r < count;
        const int64_t t = token + (live ? r : 0);
        float x[8], v[8];
        load_run<BF16, 8, VEC>(a.v.data, t * a.v.token_stride + head * a.v.head_stride + ch, live ? left : 0, v);
        head_row<BF16, VEC>(p, a.k.data, t * a.k.token_stride + head * a.k.head_stride, ch, live ? left : 0, a.k_norm, s_cos + (live ? r : 0) * half,
                            s_sin + (live ? r : 0) * half, x);
        const unsigned big_k = row_largest(x, p.lanes), big_v = row_largest(v, p.lanes);
        const bool bad = big_k >= kNoBf16 || (!FP4 && big_v >= kNoBf16);
        if (bad)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < left) x[j] = NAN;
        const bool there = live && ch < p.dp;
        if constexpr (FP4) {
          const unsigned k4 = codes_of(x, big_k), v4 = codes_of(v, big_v);
          if (there) {
            *(unsigned*)((char*)c.k + (at + slot + r) * (p.dp / 2) + ch / 2) = k4;
#pragma unroll
            for (int j = 0; j < 8; ++j) s_v[(ch + j) * value_row(true) + slot % kPiece + r] = (char)(v4 >> (4 * j) & 15);
            if (ch == 0) {
              c.k_scale[at + slot + r] = scale_of(big_k);
              c.v_scale[at + slot + r] = scale_of(big_v);
            }
          }
        } else if (there) {
          *(uint4*)((uint16_t*)c.k + (at + slot + r) * p.dp + ch) =
              make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            unsigned w = pack_bf16(v[j], v[j + 1]);
            if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;  // (no value of v that is not finite)
            if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
            if (count == kPiece) {
              *(uint16_t*)(s_v + (ch + j) * value_row(false) + 2 * r) = (uint16_t)w;
              *(uint16_t*)(s_v + (ch + j + 1) * value_row(false) + 2 * r) = (uint16_t)(w >> 16);
            } else {
              uint16_t* const q = (uint16_t*)c.v + ((int64_t)to * c.heads + head) * p.dp * c.page + (int64_t)(ch + j) * c.page + slot + r;
              q[0] = (uint16_t)w;
              q[c.page] = (uint16_t)(w >> 16);
            }
          }
        }
        if (live)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float k = bf16_low(pack_bf16(x[j], 0.0f));  // (as the cache in bf16 has it; a NaN stays in both bounds)
            if (k < lo[j] || k != k) lo[j] = k;
            if (k > hi[j] || k != k) hi[j] = k;
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
      }
      lds_turn();
      // ---- bounds: over the piece's tokens, then with what the page had unless it begins here
      if (c.bounds) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          for (int s = p.lanes; s < 64; s *= 2) {
            const float l = __shfl_xor(lo[j], s), h = __shfl_xor(hi[j], s);
            if (l < lo[j] || l != l) lo[j] = l;
            if (h > hi[j] || h != h) hi[j] = h;
          }
        if (row == 0 && ch < p.dp) {
          uint4* const q = (uint4*)((uint16_t*)c.bounds + (((int64_t)to * c.heads + head) * 2) * p.dp + ch);
          uint4* const q_hi = (uint4*)((uint16_t*)q + p.dp);
          if (slot > 0) {
            float old[8];
            load_run<true, 8, true>(q, 0, 8, old);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (old[j] < lo[j] || old[j] != old[j]) lo[j] = old[j];
            load_run<true, 8, true>(q_hi, 0, 8, old);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (old[j] > hi[j] || old[j] != old[j]) hi[j] = old[j];
          }
          *q = make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(lo[4], lo[5]), pack_bf16(lo[6], lo[7]));
          *q_hi = make_uint4(pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]), pack_bf16(hi[4], hi[5]), pack_bf16(hi[6], hi[7]));
        }
      }
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

template <bool BF16, bool FP4>
void start_append(AppendParams p, bool vec, int64_t blocks, hipStream_t s) {
  const size_t lds = 2 * sizeof(float) * kPiece * (p.a.rot / 2) + 4 * p.dp * value_row(FP4);
  const int64_t most = kMostThreads / 256;
  for (; p.block0 < blocks; p.block0 += most) {
    const unsigned grid = (unsigned)std::min(most, blocks - p.block0);
    if (vec) cache_append<BF16, FP4, true><<<grid, 256, lds, s>>>(p);
    else cache_append<BF16, FP4, false><<<grid, 256, lds, s>>>(p);
  }
}

}  // namespace

void launch_cache_append(const evconv_append_args& a, bool vec, hipStream_t s) {
  AppendParams p{};
  p.a = a;
  p.dp = cache_channels(a.cache.d);
  p.log = __builtin_ctz(a.cache.page);
  p.lanes = 1;
  while (p.lanes * 8 < p.dp) p.lanes *= 2;
  const evconv_tokens& t = a.tokens;
  p.per = t.seq_offsets ? -1 : (int)((t.n_tokens / t.n_seq + a.cache.page - 2) / a.cache.page) + 1;
  p.roles = a.heads_q + a.cache.heads;
  p.pairs_wide = vec && a.rot % 16 == 0;
  const int64_t pages = p.per >= 0 ? (int64_t)p.per * t.n_seq : t.n_tokens / a.cache.page + 2 * (int64_t)t.n_seq;
  // Workgroups of a page: as many as fill the chip a few times over, with a role at least for each of their waves.
  p.groups = (int)std::max<int64_t>(1, std::min<int64_t>((p.roles + 3) / 4, 2048 / std::max<int64_t>(pages, 1)));
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
