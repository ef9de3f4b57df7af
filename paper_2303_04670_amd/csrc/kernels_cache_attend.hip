// Attention over a paged cache (evconv_cache_attend): how a call is cut into launches, and the join of what several workgroups
// found of a row.  The kernels: cache_attend_rows.h, cache_attend_pieces.h.
#include <algorithm>

#include "cache_attend_rows.h"

namespace evk {
namespace {

// What a row's stretches gave, o = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i: T threads to a row (many stretches: a workgroup; few: a
// wave, which meets no barrier; 8192 rows of 8 stretches 24 us by workgroups, 11 by waves), `groups` workgroups to a token's heads (many
// tokens, of which most may have one stretch: one).  Which stretches a row has follows from what it sees; a row with one was written by the
// kernel itself.
template <bool BF16, int T>
__global__ __launch_bounds__(256) void attend_join(AttendParams p, int groups, int64_t block0) {
  __shared__ __align__(16) float s_sum[1024];
  __shared__ float s_total[256];
  const evconv_attend_args& a = p.a;
  const evconv_tokens& tk = a.tokens;
  const int64_t block = block0 + blockIdx.x;
  const int64_t token = block / groups;
  const Piece piece = find_piece(tk, token, tk.seq_offsets ? -1 : (int)(tk.n_tokens / tk.n_seq), 1, 1, 0);
  const int within = (int)(token - piece.first);
  if (within < 0 || within >= piece.count) return;
  const bool few = (int64_t)piece.count * p.share <= p.few;
  const int past = tk.past[piece.seq], chunk = few ? p.rows.chunk : p.pieces.chunk;
  int lo, hi;
  seen_by(p, past, within, lo, hi);
  if (!a.selected && hi - lo <= 1) return;  // (no stretch, or one)
  const int64_t rows = tk.n_tokens * a.heads_q;
  constexpr int ROWS = 256 / T;
  const int lane = threadIdx.x & 63, t = threadIdx.x % T;
  float* const sums = s_sum + threadIdx.x / T * 4 * T;
  float* const totals = s_total + threadIdx.x / T * T;
  auto turn = [&]() __attribute__((always_inline)) {
    if constexpr (T == 64) lds_turn();
    else __syncthreads();
  };
  // four channels to a thread, the rest of the threads to other stretches
  const int quads = p.dp / 4, beside = T / quads, mine = t / quads, ch = t % quads * 4;
  for (int head = (int)(block % groups) * ROWS + threadIdx.x / T; head < a.heads_q; head += groups * ROWS) {
    const int64_t row = token * a.heads_q + head;
    int s0 = 0, s1 = p.rows.splits - 1;
    if (!a.selected) {
      // (the tile of rows that the workgroup had: its first row's token)
      constexpr int kTile = BF16 ? kPieceRowsBf16 : kPieceRowsF32;
      const int64_t in_group = (int64_t)within * p.share + head % p.share;
      int first, other;
      seen_by(p, past, few ? 0 : (int)(in_group / kTile * kTile / p.share), first, other);
      const int base = stretch_base(first);
      s0 = (lo - base) / chunk;
      s1 = (hi - 1 - base) / chunk;
      if (s0 == s1) continue;
    }
    float big = -INFINITY;
    for (int s = s0 + lane; s <= s1; s += 64) big = fmaxf(big, p.stat[2 * (s * rows + row)]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) big = fmaxf(big, __shfl_xor(big, d));
    f32x4 sum = {0, 0, 0, 0};
    float total = 0.0f;
    if (mine < beside) {
#pragma unroll 4
      for (int s = s0 + mine; s <= s1; s += beside) {
        const int64_t at = s * rows + row;
        const float m = p.stat[2 * at], factor = m == big ? 1.0f : __builtin_amdgcn_exp2f(m - big);
        total += factor * p.stat[2 * at + 1];
        sum += factor * *(const f32x4*)(p.part + at * p.dp + ch);
      }
    }
    turn();  // (the last head's sums have been read)
    *(f32x4*)&sums[4 * t] = sum;
    totals[t] = total;
    turn();
    for (int c = t; c < a.cache.d; c += T) {
      float o = 0.0f, all = 0.0f;
      for (int i = 0; i < beside; ++i) {
        o += sums[i * p.dp + c];
        all += totals[i * quads];
      }
      store_one<BF16>(a.o, token * a.o_token_stride + head * a.o_head_stride + c, all == 0.0f ? 0.0f : o / all);
    }
  }
}

template <bool BF16, int T>
void start_join(const AttendParams& p, hipStream_t s) {
  const int groups = p.a.tokens.n_tokens < 1024 ? (p.a.heads_q * T + 255) / 256 : 1;
  const int64_t blocks = p.a.tokens.n_tokens * groups, most = kMostThreads / 256;
  for (int64_t at = 0; at < blocks; at += most) attend_join<BF16, T><<<(unsigned)std::min(most, blocks - at), 256, 0, s>>>(p, groups, at);
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t plan_attend(AttendParams& p) {
  const evconv_attend_args& a = p.a;
  const evconv_tokens& t = a.tokens;
  p.dp = cache_channels(a.cache.d);
  p.log = __builtin_ctz(a.cache.page);
  p.share = a.heads_q / a.cache.heads;
  p.most = (int64_t)t.width * a.cache.page;
  if (a.max_len) p.most = std::min(p.most, a.max_len);
  p.scale2 = a.scale * 1.44269504f;
  const bool fp4 = a.cache.kind == EVCONV_CACHE_FP4;
  const int64_t len = t.n_tokens / t.n_seq;
  // Stretches of `extent` tokens for `units` workgroups a stretch: so many that there are `wanted` workgroups, but none shorter than `least`.
  auto cut = [&](AttendWay& way, int64_t extent, int64_t least, int64_t wanted) {
    const int64_t workgroups = std::max<int64_t>(way.units * a.cache.heads, 1);
    int64_t chunk = std::max(least, (int64_t)((double)workgroups * extent / wanted));
    chunk = std::max(chunk, (extent + 65534) / 65535);  // (a grid's second size)
    way.chunk = (int)std::min<int64_t>((chunk + 127) / 128 * 128, 1 << 30);
    way.splits = (int)std::max<int64_t>((extent + way.chunk - 1) / way.chunk, 1);
  };
  p.rows = p.pieces = AttendWay{0, -1, 128, 1};
  if (a.selected) {
    p.rows.tiles = (p.share + kFewRows - 1) / kFewRows;
    p.rows.units = t.n_tokens * p.rows.tiles;
    cut(p.rows, (int64_t)a.count * a.cache.page, 256, 2048);
  } else {
    // (a workgroup's rows are of so many tokens at most, and its stretches begin up to 127 before the first that they see)
    auto seen = [&](int64_t tokens) { return a.window ? std::min<int64_t>(p.most, (int64_t)a.window + tokens + 127) : p.most; };
    // (lengths of their own, many rows on average: the few short ones do not get a launch of their own)
    p.few = t.seq_offsets && t.n_tokens * p.share >= 64 * (int64_t)t.n_seq ? 0 : kFewRows;
    if (p.few && (t.seq_offsets || len * p.share <= kFewRows)) {
      p.rows.units = t.n_seq;
      cut(p.rows, seen(kFewRows), fp4 ? 1024 : 512, 2048);
    }
    const int rows = a.dtype == EVCONV_BF16 ? kPieceRowsBf16 : kPieceRowsF32;
    if (t.seq_offsets) {
      if (t.n_tokens * p.share > p.few) p.pieces.units = t.n_tokens * p.share / rows + t.n_seq;
    } else if (len * p.share > kFewRows) {
      p.pieces.tiles = (int)((len * p.share + rows - 1) / rows);
      p.pieces.units = (int64_t)t.n_seq * p.pieces.tiles;
    }
    // (a workgroup for every CU is enough where it has its rows' tokens to itself: the join costs more than a half-filled last round)
    if (p.pieces.units) cut(p.pieces, seen(rows), p.pieces.units * a.cache.heads >= 256 ? std::max<int64_t>(p.most, 1) : 512, 512);
  }
  const int splits = std::max(p.rows.splits, p.pieces.splits);
  if (splits == 1) return 0;
  const size_t rows = (size_t)t.n_tokens * a.heads_q * splits;
  return up(rows * 2 * sizeof(float)) + rows * p.dp * sizeof(float);
}

void place_attend(AttendParams& p, char* workspace) {
  p.stat = (float*)workspace;
  p.part = (float*)(workspace + up((size_t)p.a.tokens.n_tokens * p.a.heads_q * std::max(p.rows.splits, p.pieces.splits) * 2 * sizeof(float)));
}

void launch_attend(const AttendParams& p, hipStream_t s) {
  const bool fp4 = p.a.cache.kind == EVCONV_CACHE_FP4;
  if (p.rows.units) fp4 ? launch_attend_rows_fp4(p, s) : launch_attend_rows_bf16(p, s);
  if (p.pieces.units) fp4 ? launch_attend_pieces_fp4(p, s) : launch_attend_pieces_bf16(p, s);
  if (p.rows.splits == 1 && p.pieces.splits == 1) return;
  const bool few = std::max(p.rows.splits, p.pieces.splits) <= 16;
  if (p.a.dtype == EVCONV_BF16) few ? start_join<true, 64>(p, s) : start_join<true, 256>(p, s);
  else few ? start_join<false, 64>(p, s) : start_join<false, 256>(p, s);
}

}  // namespace evk
