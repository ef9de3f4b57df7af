// Attention over a paged cache for few rows (evconv_cache_attend): single tokens of streams, a few of them, chosen pages.
//
// A workgroup takes up to 16 rows (tokens x query heads that share a key head) and one stretch of the tokens they see; each
// of its four waves takes every fourth tile of it, with statistics and sums of its own, joined in LDS at the end.  Keys and values go from
// memory to the registers of the matrix instructions without LDS: S' = K Q' has the tile's tokens in rows, and which
// token a row stands for is free, so they are dealt out such that the lane which holds the weights of eight tokens is the one whose
// operand of O' = V' P' wants them: no weight changes its lane.  v lies with its channels in rows for that.  The next
// tile's keys are requested once this one's are multiplied, its values likewise.
//   The running maximum is raised only when a score exceeds it by 2^8 (weights are then at most 2^8 and the sums far
// from fp32's end): a tile costs one comparison for the whole wave instead of a reduction and a product of all sums.
//   Codes of 4 bits are bf16 numbers without their scale (one instruction for two); the scale of a key multiplies its scores, that of a
// value its weights.
//   Bound by the bytes of the cache: one token of 32 heads on 8 over 262144 in bf16 5.8 TB/s, 64 tokens over up to 16384 in 4 bits 4.2 TB/s
// (there half of the time is vector and matrix instructions, of which 16 rows would take no more than the four there are).  Tiles in 4 bits of
// 64 tokens instead of 128, which leave registers for a third wave of a SIMD: 158 -> 121 us; table entries a tile ahead: 158 -> 143.
#pragma once

#include "cache_device.h"

namespace evk {
namespace {

constexpr float kRaise = 8.0f;  // log2 of the largest weight
constexpr int kNowhere = 0x3fffffff;  // position of a token that nobody sees

__device__ __forceinline__ b16x8 codes_to_bf16(unsigned w) {
  union {
    b16x2 two[4];
    b16x8 all;
  } u;
  u.two[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
  u.two[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
  u.two[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
  u.two[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
  return u.all;
}

// Zeros in place of those of eight bf16 values whose place is outside [begin, end).
__device__ __forceinline__ b16x8 keep_range(b16x8 v, int begin, int end) {
  uint4 u = __builtin_bit_cast(uint4, v);
  unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < begin || j >= end) w[j / 2] &= j % 2 ? 0x0000ffffu : 0xffff0000u;
  return __builtin_bit_cast(b16x8, make_uint4(w[0], w[1], w[2], w[3]));
}

// What a row (token of the call, query head) sees: positions [lo, hi).
__device__ __forceinline__ void seen_by(const AttendParams& p, int64_t past, int within, int& lo, int& hi) {
  const int64_t position = past + within;
  const int64_t end = p.a.causal ? position + 1 : past;
  hi = (int)max((int64_t)0, min(end, p.most));
  lo = p.a.window ? (int)min(max(position + 1 - p.a.window, (int64_t)0), (int64_t)hi) : 0;
}

// Where the stretches of a workgroup's rows begin, of the first position that its first row sees.
__device__ __forceinline__ int stretch_base(int lo) { return lo & ~127; }
// What a workgroup does with what it found of a row in stretch `split`: 0 nothing, 1 the output, 2 a part of it.
__device__ __forceinline__ int fate_of(int lo, int hi, int base, int split, int chunk) {
  if (hi <= lo) return split == 0;
  const int s0 = (lo - base) / chunk, s1 = (hi - 1 - base) / chunk;
  return split < s0 || split > s1 ? 0 : s0 == s1 ? 1 : 2;
}

template <bool FP4, int GROUPS, bool BF16, int DP, bool LIST>
__global__ __launch_bounds__(256, DP > 128 ? 1 : (DP <= 64 ? 3 : 2) + (FP4 && BF16)) void attend_rows(AttendParams p, int64_t unit0) {
  constexpr int PARTS = BF16 ? 1 : 3, WPARTS = BF16 ? 2 : 3, STEPS = DP / 32, VT = DP / 16;
  constexpr int MINE = 8 * GROUPS, TOK = 4 * MINE;  // tokens of a lane's weights, of a tile (which lies in one page)
  constexpr int KW = FP4 ? STEPS : 4 * STEPS;  // 32-bit words of a lane's part of a key
  __shared__ float s_o[4][16][DP + 4];
  __shared__ float s_stat[4][16][2];
  __shared__ int s_row[16][3];  // token, query head, what becomes of it: 0 nothing, 1 output, 2 part
  __shared__ __align__(16) float s_scale[FP4 ? 4 : 1][2][FP4 ? TOK : 4];
  const evconv_attend_args& a = p.a;
  const evconv_cache& c = a.cache;
  const evconv_tokens& tk = a.tokens;
  const int64_t u = unit0 + blockIdx.x;
  const int head = (int)(u % c.heads), split = blockIdx.y;
  const int64_t unit = u / c.heads;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  // ---- the rows
  int seq, token, within, rows_left;  // of row 0 of this tile: its token; rows from there on
  int64_t row0;
  if constexpr (LIST) {
    token = (int)(unit / p.rows.tiles);
    const Piece piece = find_piece(tk, token, tk.seq_offsets ? -1 : (int)(tk.n_tokens / tk.n_seq), 1, 1, 0);
    seq = piece.seq;
    within = token - piece.first;
    if (within < 0 || within >= piece.count) return;
    row0 = unit % p.rows.tiles * 16;
    rows_left = p.share - (int)row0;
  } else {
    seq = (int)unit;
    int count = (int)(tk.n_tokens / tk.n_seq);
    token = seq * count;
    if (tk.seq_offsets) {
      token = offset_of(tk, seq);
      count = offset_of(tk, seq + 1) - token;
    }
    row0 = within = 0;
    if (count <= 0 || (int64_t)count * p.share > p.few) return;
    rows_left = count * p.share;
  }
  const int past = tk.past[seq];
  const int64_t r = row0 + n;
  const bool live = n < rows_left;
  const int step = LIST ? 0 : (int)(r / p.share);
  const int my_token = token + (live ? step : 0), q_head = head * p.share + (live ? (int)(LIST ? r : r - (int64_t)step * p.share) : 0);
  int lo = 0, hi = 0;
  if (live) seen_by(p, past, within + step, lo, hi);
  int hi_max = hi, hi_min = live ? hi : INT32_MAX, lo_min = live ? lo : INT32_MAX, lo_max = lo;
#pragma unroll
  for (int s = 1; s < 16; s *= 2) {
    hi_max = max(hi_max, __shfl_xor(hi_max, s));
    hi_min = min(hi_min, __shfl_xor(hi_min, s));
    lo_min = min(lo_min, __shfl_xor(lo_min, s));
    lo_max = max(lo_max, __shfl_xor(lo_max, s));
  }
  const int base0 = LIST ? 0 : stretch_base(__shfl(lo, 0));
  int64_t begin = base0 + (int64_t)split * p.rows.chunk, end = begin + p.rows.chunk;
  int fate;
  if constexpr (LIST) {
    end = min(end, (int64_t)a.count << p.log);
    fate = p.rows.splits == 1 ? 1 : 2;
  } else {
    begin = max(begin, (int64_t)lo_min);
    end = min(end, (int64_t)hi_max);
    fate = fate_of(lo, hi, base0, split, p.rows.chunk);
  }
  if (!live) fate = 0;
  if (!__any(fate)) return;  // (alike in all waves)
  if (wave == 0 && g == 0) {
    s_row[n][0] = my_token;
    s_row[n][1] = q_head;
    s_row[n][2] = fate;
  }
  begin &= ~(int64_t)(TOK - 1);  // (stretches are whole tiles)
  // ---- where tokens lie: table entries (with chosen pages: from the list) two tiles ahead, pages one, so that no request waits for them
  const int* const list = LIST ? a.selected + ((int64_t)token * c.heads + head) * a.count : nullptr;
  const int* const table = tk.table + seq * tk.table_stride;
  auto entry_at = [&](int64_t base) __attribute__((always_inline)) -> int {
    const int64_t i = base >> p.log;
    if constexpr (LIST) return i < a.count ? __builtin_amdgcn_readfirstlane(list[i]) : -1;
    return (int)i;
  };
  auto page_at = [&](int entry) __attribute__((always_inline)) -> int { return entry >= 0 && entry < tk.width ? table[entry] : -1; };
  int64_t at_page = 0;                               // heads before this one's of the tile's page
  int slot = 0, real = kNowhere;                     // the tile's place in it, its first token's position
  int next_entry = -1, next_page = -1, entry = -1;   // of the next tile, of the one after it
  auto use_next = [&](int64_t base) __attribute__((always_inline)) {  // the next tile's place, and requests for those behind it
    const int page = __builtin_amdgcn_readfirstlane(next_page);
    const bool there = page >= 0 && page < c.n_pages;
    at_page = (int64_t)(there ? page : 0) * c.heads + head;  // (of a page that is not there the first one's tokens are read, and not seen)
    slot = (int)(base & (c.page - 1));
    real = there ? (next_entry << p.log) + slot : kNowhere;
    next_entry = entry;
    next_page = page_at(entry);
    entry = entry_at(base + 8 * TOK);
  };
  unsigned kw[2 * GROUPS][KW];
  unsigned vw[VT][FP4 ? GROUPS : 4];
  float ks, vs;  // scales of the token of the tile whose number is the lane's (of 32 tokens: lanes 32 and up have none)
  // (addresses: what is alike in the wave, what the lane adds to it, constants)
  const unsigned lane_k = FP4 ? (MINE * (n >> 2) + (n & 3)) * (DP / 2) + g * (DP / 8) : ((MINE * (n >> 2) + (n & 3)) * DP + 8 * g) * 2;
  const unsigned lane_v = FP4 ? (unsigned)(n * c.page + MINE * g) / 2 : (unsigned)(n * c.page + MINE * g) * 2;
  auto load_scales = [&](const float* scales, float& to) __attribute__((always_inline)) {
    to = scales[at_page * c.page + slot + (lane & (TOK - 1))];
  };
  auto load_k = [&]() __attribute__((always_inline)) {
    const char* const tile = (const char*)c.k + (at_page * c.page + slot) * (FP4 ? DP / 2 : DP * 2);
#pragma unroll
    for (int i = 0; i < 2 * GROUPS; ++i) {
      const char* const from = tile + (8 * (i / 2) + 4 * (i % 2)) * (FP4 ? DP / 2 : DP * 2) + lane_k;
      if constexpr (!FP4) {
#pragma unroll
        for (int st = 0; st < STEPS; ++st) *(uint4*)&kw[i][4 * st] = *(const uint4*)(from + 64 * st);
      } else if constexpr (STEPS % 4 == 0) {
#pragma unroll
        for (int w = 0; w < STEPS; w += 4) *(uint4*)&kw[i][w] = *(const uint4*)(from + 4 * w);
      } else if constexpr (STEPS % 2 == 0) {
#pragma unroll
        for (int w = 0; w < STEPS; w += 2) *(uint2*)&kw[i][w] = *(const uint2*)(from + 4 * w);
      } else {
#pragma unroll
        for (int w = 0; w < STEPS; ++w) kw[i][w] = *(const unsigned*)(from + 4 * w);
      }
    }
    if constexpr (FP4) load_scales(c.k_scale, ks);
  };
  auto load_v = [&]() __attribute__((always_inline)) {
    const char* const tile = (const char*)c.v + (FP4 ? (at_page * DP * c.page + slot) / 2 : (at_page * DP * c.page + slot) * 2);
#pragma unroll
    for (int i = 0; i < VT; ++i) {
      const char* const from = tile + (FP4 ? (int64_t)i * 8 * c.page : (int64_t)i * 32 * c.page) + lane_v;
      if constexpr (!FP4) *(uint4*)vw[i] = *(const uint4*)from;
      else if constexpr (GROUPS == 2) *(uint2*)vw[i] = *(const uint2*)from;
      else vw[i][0] = *(const unsigned*)from;
    }
    if constexpr (FP4) load_scales(c.v_scale, vs);
  };
  int64_t base = begin + wave * TOK;
  int seen_real = kNowhere;
  if (base < end) {
    next_entry = entry_at(base);
    next_page = page_at(next_entry);
    entry = entry_at(base + 4 * TOK);
    use_next(base);
    seen_real = real;
    load_k();
    load_v();
  }
  // ---- the queries as operands: channels as the keys' lanes have them
  b16x8 q[STEPS][PARTS];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    const int ch = FP4 ? g * (DP / 4) + 8 * st : 32 * st + 8 * g;
    const int64_t at = (int64_t)my_token * a.q.token_stride + q_head * a.q.head_stride + ch;
    float x[8];
    if (p.vec) load_run<BF16, 8, true>(a.q.data, at, live ? c.d - ch : 0, x);
    else load_run<BF16, 8, false>(a.q.data, at, live ? c.d - ch : 0, x);
    split8<PARTS>(x, q[st]);
  }
  f32x4 o[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i) o[i] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;
  for (; base < end; base += 4 * TOK) {
    const int64_t next = base + 4 * TOK;
    // ---- scores
    float x[GROUPS][8];
    if constexpr (FP4) {
      lds_turn();
      s_scale[wave][0][lane & (TOK - 1)] = ks;
      s_scale[wave][1][lane & (TOK - 1)] = vs;
      lds_turn();
    }
#pragma unroll
    for (int i = 0; i < 2 * GROUPS; ++i) {
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        b16x8 k;
        if constexpr (FP4) k = codes_to_bf16(kw[i][st]);
        else k = __builtin_bit_cast(b16x8, *(uint4*)&kw[i][4 * st]);
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[st][part], acc, 0, 0, 0);
      }
      if constexpr (FP4) acc *= *(const f32x4*)&s_scale[wave][0][MINE * g + 8 * (i / 2) + 4 * (i % 2)];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i / 2][4 * (i % 2) + j] = acc[j];
    }
    int next_real = kNowhere;
    if (next < end) {
      use_next(next);
      next_real = real;
      load_k();
    }
    // ---- what is not seen
    const int first = seen_real + MINE * g;  // of the lane's weights
    const bool whole = seen_real >= lo_max && seen_real + TOK <= hi_min;
    if (!whole)
#pragma unroll
      for (int s = 0; s < GROUPS; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int t = first + 8 * s + j;
          if (t < lo || t >= hi) x[s][j] = -INFINITY;
        }
    // ---- the running maximum
    float top = x[0][0];
#pragma unroll
    for (int s = 0; s < GROUPS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, x[s][j]);
    top *= p.scale2;
    if (__any(top > m + kRaise)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float raised = fmaxf(m, top);
      const float factor = m == raised ? 1.0f : __builtin_amdgcn_exp2f(m - raised);
      m = raised;
      l *= factor;
#pragma unroll
      for (int i = 0; i < VT; ++i) o[i] *= factor;
    }
    const float off = m == -INFINITY ? 0.0f : m;
    // ---- weights, sums
#pragma unroll
    for (int s = 0; s < GROUPS; ++s) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = __builtin_amdgcn_exp2f(fmaf(x[s][j], p.scale2, -off));
        l += w[j];
      }
      if constexpr (FP4) {
        const f32x4 v0 = *(const f32x4*)&s_scale[wave][1][MINE * g + 8 * s], v1 = *(const f32x4*)&s_scale[wave][1][MINE * g + 8 * s + 4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float scale = j < 4 ? v0[j & 3] : v1[j & 3];
          const int t = first + 8 * s + j;
          w[j] = whole || (t >= lo && t < hi) ? w[j] * scale : 0.0f;
        }
      }
      b16x8 weights[WPARTS];  // (bf16 calls too: the second half of their bits costs nothing beside the cache's bytes)
      split8<WPARTS>(w, weights);
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        b16x8 v;
        if constexpr (FP4) {
          v = codes_to_bf16(vw[i][s]);
        } else {
          v = __builtin_bit_cast(b16x8, *(uint4*)vw[i]);
          if (!whole) v = keep_range(v, lo_min - first, hi_max - first);
        }
#pragma unroll
        for (int part = WPARTS - 1; part >= 0; --part) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, weights[part], o[i], 0, 0, 0);
      }
    }
    if (next < end) load_v();
    seen_real = next_real;
  }
  // ---- the four waves' sums
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int i = 0; i < VT; ++i) *(f32x4*)&s_o[wave][n][16 * i + 4 * g] = o[i];
  if (g == 0) {
    s_stat[wave][n][0] = m;
    s_stat[wave][n][1] = l;
  }
  __syncthreads();
  const int64_t rows = tk.n_tokens * a.heads_q;
  for (int i = threadIdx.x; i < 16 * DP; i += 256) {
    const int row = i / DP, ch = i % DP, what = s_row[row][2];
    if (what == 0 || (what == 1 && ch >= c.d)) continue;
    float big = -INFINITY, sum = 0.0f, total = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) big = fmaxf(big, s_stat[w][row][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = s_stat[w][row][0], factor = mw == big ? 1.0f : __builtin_amdgcn_exp2f(mw - big);
      sum += factor * s_o[w][row][ch];
      total += factor * s_stat[w][row][1];
    }
    const int64_t token_out = s_row[row][0];
    const int head_out = s_row[row][1];
    if (what == 1) {
      store_one<BF16>(a.o, token_out * a.o_token_stride + head_out * a.o_head_stride + ch, total == 0.0f ? 0.0f : sum / total);
    } else {
      const int64_t at = (int64_t)split * rows + token_out * a.heads_q + head_out;
      p.part[at * DP + ch] = sum;
      if (ch == 0) {
        p.stat[2 * at] = big;
        p.stat[2 * at + 1] = total;
      }
    }
  }
}

template <bool FP4, int GROUPS, bool BF16, int DP>
void start_tiles(const AttendParams& p, hipStream_t s) {
  const int64_t units = p.rows.units * p.a.cache.heads;
  const int64_t most = std::min<int64_t>(kMostThreads / 256 / p.rows.splits, INT32_MAX);
  for (int64_t at = 0; at < units; at += most) {
    const dim3 grid((unsigned)std::min(most, units - at), (unsigned)p.rows.splits);
    if (p.a.selected) attend_rows<FP4, GROUPS, BF16, DP, true><<<grid, 256, 0, s>>>(p, at);
    else attend_rows<FP4, GROUPS, BF16, DP, false><<<grid, 256, 0, s>>>(p, at);
  }
}
// Tiles of 64 tokens in 4 bits, which have the bytes of 16 in bf16, where a page holds them.
template <bool FP4, bool BF16, int DP>
void start_rows(const AttendParams& p, hipStream_t s) {
  if constexpr (FP4)
    if (p.a.cache.page >= 64) return start_tiles<true, 2, BF16, DP>(p, s);
  start_tiles<FP4, 1, BF16, DP>(p, s);
}

template <bool FP4, bool BF16>
void start_rows(const AttendParams& p, hipStream_t s) {
  switch (p.dp) {
    case 32: return start_rows<FP4, BF16, 32>(p, s);
    case 64: return start_rows<FP4, BF16, 64>(p, s);
    case 96: return start_rows<FP4, BF16, 96>(p, s);
    case 128: return start_rows<FP4, BF16, 128>(p, s);
    case 192: return start_rows<FP4, BF16, 192>(p, s);
    default: return start_rows<FP4, BF16, 256>(p, s);
  }
}

}  // namespace
}  // namespace evk
