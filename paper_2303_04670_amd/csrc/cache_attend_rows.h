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
//   Bound by the bytes of the cache.
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

// What a workgroup does with what it found of such a row in stretch `split`: 0 nothing, 1 the output, 2 a part of it.
__device__ __forceinline__ int fate_of(int lo, int hi, int split, int chunk) {
  if (hi <= lo) return split == 0;
  const int s0 = lo / chunk, s1 = (hi - 1) / chunk;
  return split < s0 || split > s1 ? 0 : s0 == s1 ? 1 : 2;
}

template <bool FP4, bool BF16, int DP, bool LIST>
__global__ __launch_bounds__(256) void attend_rows(AttendParams p, int64_t unit0) {
  constexpr int PARTS = BF16 ? 1 : 3, STEPS = DP / 32, VT = DP / 16, GROUPS = FP4 ? 4 : 1, TOK = 32 * GROUPS;
  constexpr int KW = FP4 ? STEPS : 4 * STEPS;  // 32-bit words of a lane's part of a key
  __shared__ float s_o[4][16][DP + 4];
  __shared__ float s_stat[4][16][2];
  __shared__ int s_row[16][3];  // token, query head, what becomes of it: 0 nothing, 1 output, 2 part
  __shared__ float s_scale[FP4 ? 4 : 1][2][FP4 ? 128 : 1];
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
    if (count <= 0 || (int64_t)count * p.share > kFewRows) return;
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
  int64_t begin = (int64_t)split * p.rows.chunk, end = begin + p.rows.chunk;
  int fate;
  if constexpr (LIST) {
    end = min(end, (int64_t)a.count << p.log);
    fate = p.rows.splits == 1 ? 1 : 2;
  } else {
    begin = max(begin, (int64_t)lo_min);
    end = min(end, (int64_t)hi_max);
    fate = fate_of(lo, hi, split, p.rows.chunk);
  }
  if (!live) fate = 0;
  if (!__any(fate)) return;  // (alike in all waves)
  if (wave == 0 && g == 0) {
    s_row[n][0] = my_token;
    s_row[n][1] = q_head;
    s_row[n][2] = fate;
  }
  begin &= ~(int64_t)(TOK - 1);
  // ---- where tokens lie
  const int* const list = LIST ? a.selected + ((int64_t)token * c.heads + head) * a.count : nullptr;
  auto look = [&](int64_t base, int& page, int& real) __attribute__((always_inline)) {  // of 32 tokens from `base` on
    const int64_t entry = base >> p.log;
    const int slot = (int)(base & (c.page - 1));
    if constexpr (LIST) {
      const int e = entry < a.count ? list[entry] : -1;
      page = e < 0 ? -1 : page_of(c, tk, seq, e);
      real = page < 0 ? kNowhere : (e << p.log) + slot;
    } else {
      page = page_of(c, tk, seq, entry);
      real = page < 0 ? kNowhere : (int)base;
    }
    page = max(page, 0);  // (of a page that is not there the first one's are read, and not seen)
  };
  const int gk = FP4 ? n >> 2 : 0, gv = FP4 ? g : 0;
  int page_k, page_v, real_k, real_v, slot_k, slot_v;
  auto find_tile = [&](int64_t base) __attribute__((always_inline)) {
    look(base + 32 * gv, page_v, real_v);
    slot_v = (int)((base + 32 * gv) & (c.page - 1));
    if constexpr (FP4) {
      look(base + 32 * gk, page_k, real_k);
      slot_k = (int)((base + 32 * gk) & (c.page - 1));
    } else {
      page_k = page_v, slot_k = slot_v;
    }
  };
  unsigned kw[2 * GROUPS][KW];
  uint4 vw[VT];
  float2 ks, vs;
  auto load_k = [&]() __attribute__((always_inline)) {
    const int64_t at = ((int64_t)page_k * c.heads + head) * c.page + slot_k;
#pragma unroll
    for (int i = 0; i < 2 * GROUPS; ++i) {
      const int t = (FP4 ? 8 * (i / 2) : 8 * (n >> 2)) + 4 * (i % 2) + (n & 3);
      if constexpr (FP4) {
        const char* const q = (const char*)c.k + (at + t) * (DP / 2) + g * (DP / 8);
        if constexpr (STEPS % 4 == 0) {
#pragma unroll
          for (int w = 0; w < STEPS; w += 4) *(uint4*)&kw[i][w] = *(const uint4*)(q + 4 * w);
        } else if constexpr (STEPS % 2 == 0) {
#pragma unroll
          for (int w = 0; w < STEPS; w += 2) *(uint2*)&kw[i][w] = *(const uint2*)(q + 4 * w);
        } else {
#pragma unroll
          for (int w = 0; w < STEPS; ++w) kw[i][w] = *(const unsigned*)(q + 4 * w);
        }
      } else {
        const uint16_t* const q = (const uint16_t*)c.k + (at + t) * DP + 8 * g;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) *(uint4*)&kw[i][4 * st] = *(const uint4*)(q + 32 * st);
      }
    }
    if constexpr (FP4) {
      const int64_t at_v = ((int64_t)page_v * c.heads + head) * c.page + slot_v + 2 * n;
      ks = *(const float2*)(c.k_scale + at_v);
    }
  };
  auto load_v = [&]() __attribute__((always_inline)) {
    const int64_t at = ((int64_t)page_v * c.heads + head) * DP;
#pragma unroll
    for (int i = 0; i < VT; ++i) {
      if constexpr (FP4) vw[i] = *(const uint4*)((const char*)c.v + ((at + 16 * i + n) * c.page + slot_v) / 2);
      else vw[i] = *(const uint4*)((const uint16_t*)c.v + (at + 16 * i + n) * c.page + slot_v + 8 * g);
    }
    if constexpr (FP4) vs = *(const float2*)(c.v_scale + ((int64_t)page_v * c.heads + head) * c.page + slot_v + 2 * n);
  };
  int64_t base = begin + wave * TOK;
  int seen_real = kNowhere;
  if (base < end) {
    find_tile(base);
    seen_real = real_v;
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
      *(float2*)&s_scale[wave][0][2 * lane] = ks;
      *(float2*)&s_scale[wave][1][2 * lane] = vs;
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
      if constexpr (FP4) acc *= *(const f32x4*)&s_scale[wave][0][32 * g + 8 * (i / 2) + 4 * (i % 2)];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i / 2][4 * (i % 2) + j] = acc[j];
    }
    const int real = real_v;
    int next_real = kNowhere;
    if (next < end) {
      find_tile(next);
      next_real = real_v;
      load_k();
    }
    (void)real;
    // ---- what is not seen
    const int first = FP4 ? seen_real : seen_real + 8 * g;  // of this lane's weights
    const bool whole = __all(seen_real >= lo_max && seen_real + 32 <= hi_min);
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
        const f32x4 v0 = *(const f32x4*)&s_scale[wave][1][32 * g + 8 * s], v1 = *(const f32x4*)&s_scale[wave][1][32 * g + 8 * s + 4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float scale = j < 4 ? v0[j & 3] : v1[j & 3];
          const int t = first + 8 * s + j;
          w[j] = whole || (t >= lo && t < hi) ? w[j] * scale : 0.0f;
        }
      }
      b16x8 weights[PARTS];
      split8<PARTS>(w, weights);
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        b16x8 v;
        if constexpr (FP4) {
          const unsigned words[4] = {vw[i].x, vw[i].y, vw[i].z, vw[i].w};
          v = codes_to_bf16(words[s]);
        } else {
          v = __builtin_bit_cast(b16x8, vw[i]);
          if (!whole) v = keep_range(v, lo_min - first, hi_max - first);
        }
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, weights[part], o[i], 0, 0, 0);
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

template <bool FP4, bool BF16, int DP>
void start_rows(const AttendParams& p, hipStream_t s) {
  const int64_t units = p.rows.units * p.a.cache.heads;
  const int64_t most = std::min<int64_t>(kMostThreads / 256 / p.rows.splits, INT32_MAX);
  for (int64_t at = 0; at < units; at += most) {
    const dim3 grid((unsigned)std::min(most, units - at), (unsigned)p.rows.splits);
    if (p.a.selected) attend_rows<FP4, BF16, DP, true><<<grid, 256, 0, s>>>(p, at);
    else attend_rows<FP4, BF16, DP, false><<<grid, 256, 0, s>>>(p, at);
  }
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
