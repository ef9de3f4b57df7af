// Attention over a paged cache for many rows (evconv_cache_attend): pieces of sequences.
//
// A workgroup takes 128 rows (64 in fp32; rows are tokens x query heads that share a key head, so these share its keys) and goes over
// the tokens they see, a tile at a time: keys and values come into LDS while the tile before is being worked on, in 16-byte pieces whose places
// are permuted within a row such that the operands' reads meet no bank twice; codes of 4 bits are turned into bf16 on the way, once for
// all waves.  A wave has 16 or 32 rows of its own, with S' = K Q' and O' = V' P' as cache_attend_rows.h has them: weights stay in the lane that
// made them.  Few workgroups over many tokens share a row's tokens and join what they found.
//   8 sequences of 4096 tokens, 16 heads on 4 of 128 in bf16: 584 us, 940 TFLOP/s, where a large library product reaches 1215; matrix
// instructions in 42 % of the cycles, vector ones (exponentials a third of them) in as many.  Operands read ahead instead of where they are wanted 710 -> 661 us,
// addresses made once 661 -> 624, priority to the matrix instructions 624 -> 611.  512 tokens on 32768 in 4 bits: 175 us, 790 TFLOP/s.
#pragma once

#include "cache_attend_rows.h"

namespace evk {
namespace {

template <int DP>
struct PieceTile {
  static constexpr int kTokens = DP > 128 ? 32 : 64, kHalves = kTokens / 32;
  static constexpr int kBytes = kTokens * DP * 2;  // of keys, and of values
  static constexpr int kPlaces = DP / 8;           // 16-byte pieces of a key
  // Where piece `c` of token t's key is, and piece `c` of a channel's tokens
  static __device__ __forceinline__ int key_at(int t, int c) {
    constexpr int mask = kPlaces % 16 == 0 ? 15 : kPlaces % 8 == 0 ? 7 : 3;
    return t * kPlaces + (c ^ (((t & 3) | (t >> 3 & 3) << 2) & mask));
  }
  static __device__ __forceinline__ int value_at(int channel, int c) {
    return kTokens == 64 ? channel * 8 + (c ^ (channel & 7)) : channel * 4 + (c ^ (channel >> 1 & 3));
  }
};

template <bool V>
struct Whole {
  static constexpr bool value = V;
};

template <bool FP4, bool BF16, int DP>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attend_pieces(AttendParams p, int64_t block0) {
  using Tile = PieceTile<DP>;
  // (weights of bf16 calls are rounded to bf16, by up to 2^-8 of themselves as the output is: 8 x 4096 tokens are 0.0022 of the norm off instead
  // of 0.0016, and take 594 us instead of 756 with two parts, 512 tokens on 32768 in 4 bits 193 instead of 233)
  constexpr int PARTS = BF16 ? 1 : 3, CT = BF16 ? 2 : 1, ROWS = BF16 ? kPieceRowsBf16 : kPieceRowsF32, STEPS = DP / 32, VT = DP / 16, TT = Tile::kTokens, HALVES = Tile::kHalves;
  extern __shared__ __align__(16) char s_mem[];
  char* const s_k = s_mem;
  char* const s_v = s_mem + 2 * Tile::kBytes;
  float* const s_scale = (float*)(s_mem + 4 * Tile::kBytes);  // [2][keys, values][TT]
  const evconv_attend_args& a = p.a;
  const evconv_cache& c = a.cache;
  const evconv_tokens& tk = a.tokens;
  const int64_t block = block0 + blockIdx.x;
  const int head = (int)(block % c.heads), split = blockIdx.y;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  // ---- the rows: of equal lengths the last pieces first, which see the most
  const int64_t number = p.pieces.units - 1 - block / c.heads;
  Piece piece;
  if (p.pieces.tiles >= 0) {
    piece.seq = (int)(number % tk.n_seq);
    piece.at = (int)(number / tk.n_seq);
    piece.count = (int)(tk.n_tokens / tk.n_seq);
    piece.first = piece.seq * piece.count;
  } else {
    piece = find_piece(tk, number, -1, p.share, ROWS, 1);
  }
  const int64_t total = (int64_t)piece.count * p.share, row0 = (int64_t)piece.at * ROWS;
  if (piece.at < 0 || row0 >= total || total <= p.few) return;
  const int past = tk.past[piece.seq];
  // (rows of a sequence may pass 32 bits: they are counted from the workgroup's first one on)
  const int last = (int)min(total - row0, (int64_t)ROWS) - 1;
  const int token0 = (int)(row0 / p.share), rest0 = (int)(row0 - (int64_t)token0 * p.share);
  auto token_of = [&](int row) __attribute__((always_inline)) { return token0 + (rest0 + row) / p.share; };
  int lo_min, hi_max, other;
  seen_by(p, past, token0, lo_min, other);
  seen_by(p, past, token_of(last), other, hi_max);
  const int chunk = p.pieces.chunk;
  const int base0 = stretch_base(lo_min);
  const int64_t begin = max(base0 + (int64_t)split * chunk, (int64_t)lo_min) & ~(int64_t)(TT - 1), end = min(base0 + (int64_t)(split + 1) * chunk, (int64_t)hi_max);
  if (begin >= end && split != 0) return;
  // of this wave: its first and last row, what all of them and what any of them sees
  const int wave_row = wave * 16 * CT;
  const bool working = wave_row <= last;
  int wave_lo_min = 0, wave_hi_min = 0, wave_lo_max = 0, wave_hi_max = 0;
  if (working) {
    seen_by(p, past, token_of(wave_row), wave_lo_min, wave_hi_min);
    seen_by(p, past, token_of(min(wave_row + 16 * CT - 1, last)), wave_lo_max, wave_hi_max);
  }
  int lo[CT], hi[CT], token[CT], q_head[CT];
  bool live[CT];
  b16x8 q[CT][STEPS][PARTS];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int r = wave_row + 16 * ct + n;
    live[ct] = r <= last;
    const int within = live[ct] ? token_of(r) : 0;
    token[ct] = piece.first + within;
    q_head[ct] = head * p.share + (live[ct] ? rest0 + r - (within - token0) * p.share : 0);
    lo[ct] = hi[ct] = 0;
    if (live[ct]) seen_by(p, past, within, lo[ct], hi[ct]);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int ch = 32 * st + 8 * g;
      const int64_t at = (int64_t)token[ct] * a.q.token_stride + q_head[ct] * a.q.head_stride + ch;
      float x[8];
      if (p.vec) load_run<BF16, 8, true>(a.q.data, at, live[ct] ? c.d - ch : 0, x);
      else load_run<BF16, 8, false>(a.q.data, at, live[ct] ? c.d - ch : 0, x);
      split8<PARTS>(x, q[ct][st]);
    }
  }
  // ---- a tile into LDS.  Addresses: where the halves' tokens begin is alike for all lanes, what a lane adds to it the same for every tile
  // (the permutation is its own inverse: what a lane writes to its place is what it finds by it).
  int real[HALVES];
  const char *k_at[HALVES], *v_at[HALVES];
  int64_t scale_at[HALVES];
  uint4 k_new, v_new;
  float scale_new;
  constexpr int kLoads = Tile::kBytes / 4096;  // of keys and of values, by each wave
  unsigned k_lane[kLoads], v_lane;             // bytes; keys: from their half's first on; values: of the first load
  const int v_part = Tile::value_at((wave * 64 + lane) / (TT / 8), lane % (TT / 8)) - (wave * 64 + lane) / (TT / 8) * (TT / 8);
  if constexpr (!FP4) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int place = (4 * i + wave) * 64 + lane, t = place / Tile::kPlaces;
      k_lane[i] = 2 * (t % 32 * DP + 8 * (Tile::key_at(t, place % Tile::kPlaces) - t * Tile::kPlaces));
    }
    v_lane = 2 * ((wave * 64 + lane) / (TT / 8) * c.page + 8 * (v_part % 4));
  } else {
    const int i = threadIdx.x;
    k_lane[0] = i / (DP / 32) % 32 * (DP / 2) + 16 * (i % (DP / 32));
    v_lane = i / HALVES * c.page / 2;
  }
  int ahead[HALVES];  // table entries of the next tile: looked up a tile before they are wanted
  const int* const table = tk.table + piece.seq * tk.table_stride;
  auto look_ahead = [&](int64_t base) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < HALVES; ++h) ahead[h] = table[min((base + 32 * h) >> p.log, (int64_t)tk.width - 1)];
  };
  auto find_tile = [&](int64_t base) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const int64_t at = base + 32 * h;
      const int entry = __builtin_amdgcn_readfirstlane(ahead[h]), found = (at >> p.log) < tk.width && entry < c.n_pages ? entry : -1;
      const int slot = (int)(at & (c.page - 1));
      real[h] = found < 0 ? kNowhere : (int)at;
      const int64_t heads = (int64_t)max(found, 0) * c.heads + head;  // (of a page that is not there the first one's tokens are read, and not seen)
      scale_at[h] = heads * c.page + slot;
      k_at[h] = (const char*)c.k + scale_at[h] * (FP4 ? DP / 2 : DP * 2);
      v_at[h] = (const char*)c.v + (FP4 ? (heads * DP * c.page + slot) / 2 : (heads * DP * c.page + slot) * 2);
    }
  };
  const int wave_of = __builtin_amdgcn_readfirstlane(wave);
  auto request = [&](int buffer) __attribute__((always_inline)) {
    if constexpr (!FP4) {
      auto copy = [&](const char* from, char* to) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
      };
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        char* const to = s_k + buffer * Tile::kBytes + (4 * i + wave_of) * 1024;
        // (a load's keys are of one half, but for rows of 12 pieces)
        const int first = (4 * i + wave) * 64, t0 = first / Tile::kPlaces, t1 = (first + 63) / Tile::kPlaces;
        if (HALVES == 1 || t1 < 32) copy(k_at[0] + k_lane[i], to);
        else if (t0 >= 32) copy(k_at[HALVES - 1] + k_lane[i], to);
        else copy((first + lane < 32 * Tile::kPlaces ? k_at[0] : k_at[HALVES - 1]) + k_lane[i], to);
      }
      const int64_t step = (int64_t)(256 / (TT / 8)) * 2 * c.page;  // (channels of a load by all waves: whole periods of the permutation)
      const char* const lane_at = (HALVES == 1 || v_part < 4 ? v_at[0] : v_at[HALVES - 1]) + v_lane;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) copy(lane_at + i * step, s_v + buffer * Tile::kBytes + (4 * i + wave_of) * 1024);
    } else {
      // (values, not places of arrays, to choose between: those would lie in memory)
      const int i = threadIdx.x, t = i % TT;
      const char *const k0 = k_at[0], *const k1 = k_at[HALVES - 1], *const v0 = v_at[0], *const v1 = v_at[HALVES - 1];
      const int64_t s0 = scale_at[0], s1 = scale_at[HALVES - 1];
      const float *const ks = c.k_scale, *const vs = c.v_scale;
      if (i < TT * DP / 32) k_new = *(const uint4*)((HALVES == 1 || i < 32 * (DP / 32) ? k0 : k1) + k_lane[0]);
      if (i < DP * HALVES) v_new = *(const uint4*)((i % HALVES == 0 ? v0 : v1) + v_lane);
      if (i < 2 * TT) scale_new = (i < TT ? ks : vs)[(HALVES == 1 || t < 32 ? s0 : s1) + t % 32];
    }
  };
  auto deliver = [&](int buffer) __attribute__((always_inline)) {  // codes into LDS as bf16
    if constexpr (FP4) {
      const int i = threadIdx.x;
      const unsigned kw[4] = {k_new.x, k_new.y, k_new.z, k_new.w}, vw[4] = {v_new.x, v_new.y, v_new.z, v_new.w};
      if (i < TT * DP / 32) {
        const int t = i / (DP / 32), part = i % (DP / 32);
#pragma unroll
        for (int j = 0; j < 4; ++j) *(b16x8*)(s_k + buffer * Tile::kBytes + 16 * Tile::key_at(t, 4 * part + j)) = codes_to_bf16(kw[j]);
      }
      if (i < DP * HALVES) {
        const int channel = i / HALVES, h = i % HALVES;
#pragma unroll
        for (int j = 0; j < 4; ++j) *(b16x8*)(s_v + buffer * Tile::kBytes + 16 * Tile::value_at(channel, 4 * h + j)) = codes_to_bf16(vw[j]);
      }
      if (i < 2 * TT) s_scale[buffer * 2 * TT + i] = scale_new;
    }
  };
  auto turn = [&]() __attribute__((always_inline)) {  // what was requested is there, for all waves
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  f32x4 o[CT][VT];
  float m[CT], l[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m[ct] = -INFINITY;
    l[ct] = 0.0f;
#pragma unroll
    for (int i = 0; i < VT; ++i) o[ct][i] = f32x4{0, 0, 0, 0};
  }
  // A tile that is in LDS: operands are read a step before the products that want them, values' while the weights are made.
  auto work = [&](const int (&at)[HALVES], int buffer, auto is_whole) __attribute__((always_inline)) {
    constexpr bool whole = decltype(is_whole)::value;
    const char* const keys = s_k + buffer * Tile::kBytes;
    const char* const values = s_v + buffer * Tile::kBytes;
    const float* const scales = s_scale + buffer * 2 * TT;
    auto read_keys = [&](int i, b16x8 (&k)[STEPS]) __attribute__((always_inline)) {
      const int t = 32 * (i / 2) + 8 * (n >> 2) + 4 * (i % 2) + (n & 3);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) k[st] = *(const b16x8*)(keys + 16 * Tile::key_at(t, 4 * st + g));
    };
    auto read_value = [&](int h, int i) __attribute__((always_inline)) { return *(const b16x8*)(values + 16 * Tile::value_at(16 * i + n, 4 * h + g)); };
    __builtin_amdgcn_s_setprio(1);  // (matrix instructions first: the other wave of the SIMD has vector ones meanwhile)
    // ---- scores
    float x[CT][HALVES][8];
    constexpr int AHEAD = DP > 192 ? 0 : 1;  // (keys of 256 channels: there are no registers for two rows of operands)
    b16x8 k[1 + AHEAD][STEPS];
    if (AHEAD) read_keys(0, k[0]);
#pragma unroll
    for (int i = 0; i < 2 * HALVES; ++i) {
      if (i + AHEAD < 2 * HALVES) read_keys(i + AHEAD, k[(i + AHEAD) & AHEAD]);
      f32x4 acc[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) acc[ct] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < STEPS; ++st)
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i & AHEAD][st], q[ct][st][part], acc[ct], 0, 0, 0);
      if constexpr (FP4) {
        const f32x4 scale = *(const f32x4*)(scales + 32 * (i / 2) + 8 * g + 4 * (i % 2));
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) acc[ct] *= scale;
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[ct][i / 2][4 * (i % 2) + j] = acc[ct][j];
    }
    b16x8 v[VT];
#pragma unroll
    for (int i = 0; i < VT; ++i) v[i] = read_value(0, i);
    __builtin_amdgcn_sched_barrier(0);  // (requested here, not where they are wanted)
    __builtin_amdgcn_s_setprio(0);
    // ---- what is not seen
    if constexpr (!whole)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int t = at[h] + 8 * g + j;
            if (t < lo[ct] || t >= hi[ct]) x[ct][h][j] = -INFINITY;
          }
    // ---- the running maxima
    float top[CT];
    bool raise = false;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      top[ct] = x[ct][0][0];
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) top[ct] = fmaxf(top[ct], x[ct][h][j]);
      top[ct] *= p.scale2;
      raise = raise || top[ct] > m[ct] + kRaise;
    }
    if (__any(raise))
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        top[ct] = fmaxf(top[ct], __shfl_xor(top[ct], 16));
        top[ct] = fmaxf(top[ct], __shfl_xor(top[ct], 32));
        const float raised = fmaxf(m[ct], top[ct]);
        const float factor = m[ct] == raised ? 1.0f : __builtin_amdgcn_exp2f(m[ct] - raised);
        m[ct] = raised;
        l[ct] *= factor;
#pragma unroll
        for (int i = 0; i < VT; ++i) o[ct][i] *= factor;
      }
    // ---- weights, sums
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      b16x8 weights[CT][PARTS];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const float off = m[ct] == -INFINITY ? 0.0f : m[ct];
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          w[j] = __builtin_amdgcn_exp2f(fmaf(x[ct][h][j], p.scale2, -off));
          l[ct] += w[j];
        }
        if constexpr (FP4) {
          const f32x4 s0 = *(const f32x4*)(scales + TT + 32 * h + 8 * g), s1 = *(const f32x4*)(scales + TT + 32 * h + 8 * g + 4);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float scale = j < 4 ? s0[j & 3] : s1[j & 3];
            const int t = at[h] + 8 * g + j;
            w[j] = whole || (t >= lo[ct] && t < hi[ct]) ? w[j] * scale : 0.0f;
          }
        }
        split8<PARTS>(w, weights[ct]);
      }
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        b16x8 value = v[i];
        if (h + 1 < HALVES) v[i] = read_value(h + 1, i);
        if constexpr (!FP4 && !whole) value = keep_range(value, wave_lo_min - (at[h] + 8 * g), wave_hi_max - (at[h] + 8 * g));
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) o[ct][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, weights[ct][part], o[ct][i], 0, 0, 0);
      }
      __builtin_amdgcn_s_setprio(0);
    }
  };
  if (begin < end) {
    look_ahead(begin);
    find_tile(begin);
    request(0);
    look_ahead(begin + TT);
    deliver(0);
    turn();
  }
  int buffer = 0;
  for (int64_t base = begin; base < end; base += TT, buffer ^= 1) {
    int at[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) at[h] = real[h];
    const bool more = base + TT < end;
    if (more) {
      find_tile(base + TT);
      request(buffer ^ 1);
      look_ahead(base + 2 * TT);
    }
    // (a tile that no row of the wave sees: the others' diagonal)
    if (working && base < wave_hi_max && base + TT > wave_lo_min) {
      bool whole = true;
#pragma unroll
      for (int h = 0; h < HALVES; ++h) whole = whole && at[h] >= wave_lo_max && at[h] + 32 <= wave_hi_min;
      if (whole) work(at, buffer, Whole<true>{});
      else work(at, buffer, Whole<false>{});
    }
    if (more) deliver(buffer ^ 1);
    turn();
  }
  if (!working) return;
  // ---- out
  const int64_t rows = tk.n_tokens * a.heads_q;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    l[ct] += __shfl_xor(l[ct], 16);
    l[ct] += __shfl_xor(l[ct], 32);
    const int fate = live[ct] ? fate_of(lo[ct], hi[ct], base0, split, chunk) : 0;
    if (fate == 1) {
      const float inverse = l[ct] == 0.0f ? 0.0f : 1.0f / l[ct];
      const int64_t at = (int64_t)token[ct] * a.o_token_stride + q_head[ct] * a.o_head_stride;
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        const int ch = 16 * i + 4 * g;
        const f32x4 y = o[ct][i] * inverse;
        if (p.vec_o) {
          if (ch >= c.d) continue;
          if (BF16) *(uint2*)((uint16_t*)a.o + at + ch) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
          else *(f32x4*)((float*)a.o + at + ch) = y;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (ch + j < c.d) store_one<BF16>(a.o, at + ch + j, y[j]);
        }
      }
    } else if (fate == 2) {
      const int64_t at = (int64_t)split * rows + (int64_t)token[ct] * a.heads_q + q_head[ct];
#pragma unroll
      for (int i = 0; i < VT; ++i) *(f32x4*)(p.part + at * DP + 16 * i + 4 * g) = o[ct][i];
      if (g == 0) {
        p.stat[2 * at] = m[ct];
        p.stat[2 * at + 1] = l[ct];
      }
    }
  }
}

template <bool FP4, bool BF16, int DP>
void start_pieces(const AttendParams& p, hipStream_t s) {
  using Tile = PieceTile<DP>;
  const size_t lds = 4 * Tile::kBytes + (FP4 ? 4 * Tile::kTokens * sizeof(float) : 0);
  const int64_t blocks = p.pieces.units * p.a.cache.heads, most = std::min<int64_t>(kMostThreads / 256 / p.pieces.splits, INT32_MAX);
  for (int64_t at = 0; at < blocks; at += most)
    attend_pieces<FP4, BF16, DP><<<dim3((unsigned)std::min(most, blocks - at), (unsigned)p.pieces.splits), 256, lds, s>>>(p, at);
}

template <bool FP4, bool BF16>
void start_pieces(const AttendParams& p, hipStream_t s) {
  switch (p.dp) {
    case 32: return start_pieces<FP4, BF16, 32>(p, s);
    case 64: return start_pieces<FP4, BF16, 64>(p, s);
    case 96: return start_pieces<FP4, BF16, 96>(p, s);
    case 128: return start_pieces<FP4, BF16, 128>(p, s);
    case 192: return start_pieces<FP4, BF16, 192>(p, s);
    default: return start_pieces<FP4, BF16, 256>(p, s);
  }
}

}  // namespace
}  // namespace evk
