// Choosing pages of a paged cache (evconv_cache_select) on gfx950, in two launches: the scores of all pages, and of each query and
// key head the highest ones.
//
// Scores are taken in 64 bits: which of two pages is chosen is then the formula's answer and not that of an order of additions.  A wave
// holds the bounds of a few pages per lane as 64-bit values, eight channels to a lane, and goes over the query heads that share
// them, whose values come from LDS; so the conversions are made once for all heads.
#include <algorithm>

#include "cache_choice.h"
#include "cache_device.h"

namespace evk {
namespace {

constexpr int kHeads = 16;  // query heads whose values are in LDS at once
constexpr int kHeld = 2;    // pages that a lane holds
constexpr int kRounds = 2;  // of a workgroup

// Unsigned numbers in the order of the floats, all above 0: that is the mark of a page that cannot be chosen.
__device__ __forceinline__ unsigned key_of(float score) {
  if (score != score) return kNotANumber;
  const unsigned u = __float_as_uint(score + 0.0f);  // (no negative zero)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Query {
  int seq, token;
  int64_t last;  // page of the query's own position, -1: it sees none
};
__device__ __forceinline__ Query find_query(const SelectParams& p, int64_t token) {
  const evconv_tokens& tk = p.a.tokens;
  const Piece piece = find_piece(tk, token, p.len, 1, 1, 0);
  const int64_t within = token - piece.first;
  if (within < 0 || within >= piece.count) return {-1, 0, -1};
  const int64_t position = min((int64_t)tk.past[piece.seq] + within, p.most - 1);
  return {piece.seq, (int)token, position < 0 ? -1 : position >> p.log};
}

// `v` of the lane that the pattern names, within rows of 16 lanes
template <int PATTERN>
__device__ __forceinline__ double of_lane(double v) {
  const uint2 u = __builtin_bit_cast(uint2, v);
  uint2 w;
  w.x = (unsigned)__builtin_amdgcn_update_dpp(0, (int)u.x, PATTERN, 0xf, 0xf, false);
  w.y = (unsigned)__builtin_amdgcn_update_dpp(0, (int)u.y, PATTERN, 0xf, 0xf, false);
  return __builtin_bit_cast(double, w);
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kTurn4 = 0x124, kTurn8 = 0x128;  // lanes l ^ 1, l ^ 2 (of four), l - 4, l - 8 (of 16, round)

// Sums over LANES neighbouring lanes of two values; lane l has that of value l & 1.
template <int LANES>
__device__ __forceinline__ double pages_sum(const double (&v)[2], int lane) {
  const bool odd = lane & 1;
  double s = (odd ? v[1] : v[0]) + of_lane<kSwap1>(odd ? v[0] : v[1]);
  s += of_lane<kSwap2>(s);
  if constexpr (LANES == 8) s += __shfl_xor(s, 4);
  if constexpr (LANES >= 16) {
    s += of_lane<kTurn4>(s);
    s += of_lane<kTurn8>(s);
  }
  if constexpr (LANES == 32) s += __shfl_xor(s, 16);
  return s;
}

// A workgroup goes over kRounds times 4 kHeld GROUPS pages: its start (whose the query is, its values as 64-bit numbers) costs as much as a
// round, and the next one's bounds are on their way while one is added up.  us for 16 streams of up to 2048 pages, 8 key heads / one of 15626,
// 4, with four pages to a lane: 1 round 25.6 / 13.2, 2 26.9 / 12.4, 4 28.2 / 15.6; 2 rounds with two pages, which leave room for twice the waves,
// 23.9 / 12.3.  Bound by 64-bit instructions and the start: the bounds are 60 MB / 32 MB.
template <bool BF16, int DP>
__global__ __launch_bounds__(256) void score_pages(SelectParams p, int blocks, int64_t block0) {
  constexpr int LANES = DP <= 32 ? 4 : DP <= 64 ? 8 : DP <= 128 ? 16 : 32, GROUPS = 64 / LANES, ROUND = 4 * kHeld * GROUPS;
  // min(q, 0), max(q, 0): of a lane's eight channels two at a time, neighbouring lanes next to each other
  __shared__ double2 s_q[kHeads][2][4][DP / 8];
  const evconv_select_args& a = p.a;
  const evconv_cache& c = a.cache;
  const int64_t unit = (block0 + blockIdx.x) / blocks, token = unit / c.heads;
  const int head = (int)(unit - token * c.heads);
  const Query query = find_query(p, token);
  const int64_t first_page = (block0 + blockIdx.x - unit * blocks) * (kRounds * ROUND);
  if (query.seq < 0 || first_page > query.last) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, group = lane / LANES, ch = lane % LANES * 8;
  const int rounds = (int)min((int64_t)kRounds, (query.last - first_page) / ROUND + 1);
  auto page_number = [&](int round, int i) __attribute__((always_inline)) { return first_page + round * ROUND + (wave * kHeld + i) * GROUPS + group; };
  int held[kHeld];         // pages of the round whose bounds are requested next
  bool there[kHeld];       // whether those of the round that was requested are there
  uint4 low[kHeld], high[kHeld];
  auto look = [&](int round) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int64_t at = page_number(round, i);
      held[i] = at <= query.last ? page_of(c, a.tokens, query.seq, at) : -1;
    }
  };
  auto request = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      there[i] = held[i] >= 0;
      const uint16_t* const row = (const uint16_t*)c.bounds + ((int64_t)max(held[i], 0) * c.heads + head) * 2 * DP + min(ch, DP - 8);
      low[i] = *(const uint4*)row;
      high[i] = *(const uint4*)(row + DP);
    }
  };
  look(0);
  request();
  if (rounds > 1) look(1);
  for (int round = 0; round < rounds; ++round) {
    double lo[kHeld][8], hi[kHeld][8];
    bool is_there[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const unsigned l[4] = {low[i].x, low[i].y, low[i].z, low[i].w}, h[4] = {high[i].x, high[i].y, high[i].z, high[i].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        lo[i][j] = (double)(j % 2 ? bf16_high(l[j / 2]) : bf16_low(l[j / 2]));
        hi[i][j] = (double)(j % 2 ? bf16_high(h[j / 2]) : bf16_low(h[j / 2]));
      }
      is_there[i] = there[i];
    }
    if (round + 1 < rounds) {
      request();
      if (round + 2 < rounds) look(round + 2);
    }
    double best = -INFINITY;  // of the page whose sums come to this lane
    bool bad = false;
    for (int h0 = 0; h0 < p.share; h0 += kHeads) {
      const int heads = min(p.share - h0, kHeads);
      if (round == 0 || p.share > kHeads) {
        __syncthreads();
        for (int i = threadIdx.x; i < heads * DP; i += 256) {
          const int h = i / DP, x = i % DP;
          const int64_t from = token * a.q.token_stride + (int64_t)(head * p.share + h0 + h) * a.q.head_stride + x;
          const double v = x < c.d ? (double)load_one<BF16>(a.q.data, from) : 0.0;
          ((double*)&s_q[h][0][x % 8 / 2][x / 8])[x % 2] = v > 0.0 ? 0.0 : v;  // (a NaN is in both)
          ((double*)&s_q[h][1][x % 8 / 2][x / 8])[x % 2] = v < 0.0 ? 0.0 : v;
        }
        __syncthreads();
      }
      for (int h = 0; h < heads; ++h) {
        double sum[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) sum[i] = 0.0;
        if (ch < DP)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const double2 neg = s_q[h][0][j][ch / 8], pos = s_q[h][1][j][ch / 8];
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
              sum[i] = fma(neg.x, lo[i][2 * j], fma(pos.x, hi[i][2 * j], sum[i]));
              sum[i] = fma(neg.y, lo[i][2 * j + 1], fma(pos.y, hi[i][2 * j + 1], sum[i]));
            }
          }
        const double score = pages_sum<LANES>(sum, lane);
        bad = bad || score != score;
        best = fmax(best, score);
      }
    }
    if (lane % LANES < 2) {
      const int i = lane & 1;
      const int64_t page = page_number(round, i);
      const bool here = i == 0 ? is_there[0] : is_there[1];
      if (page <= query.last) {
        const bool forced = page < a.first || page > query.last - a.last;
        p.score[unit * p.pages + page] = !here ? 0u : forced ? kForced : bad ? kNotANumber : key_of((float)best);
      }
    }
  }
}

// Sums over the threads of a workgroup of what stands before each of them, of two numbers at once; `all`: of all.
struct Two {
  int a, b;
};
__device__ __forceinline__ Two sums_before(Two v, Two* s_wave, Two* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  Two before = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int a = __shfl_up(before.a, d), b = __shfl_up(before.b, d);
    if (lane >= d) before.a += a, before.b += b;
  }
  __syncthreads();  // (the last sums have been read)
  if (lane == 63) s_wave[wave] = before;
  __syncthreads();
  Two others{0, 0};
  *all = Two{0, 0};
  for (int w = 0; w < waves; ++w) {
    const Two x = s_wave[w];
    if (w < wave) others.a += x.a, others.b += x.b;
    all->a += x.a, all->b += x.b;
  }
  return {others.a + before.a - v.a, others.b + before.b - v.b};
}
// Least and largest of a value over the threads of a workgroup.
__device__ __forceinline__ void range_of(unsigned& lo, unsigned& hi, unsigned (*s_range)[2]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    lo = min(lo, (unsigned)__shfl_xor((int)lo, d));
    hi = max(hi, (unsigned)__shfl_xor((int)hi, d));
  }
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) s_range[wave][0] = lo, s_range[wave][1] = hi;
  __syncthreads();
  for (int w = 0; w < waves; ++w) lo = min(lo, s_range[w][0]), hi = max(hi, s_range[w][1]);
}

// The `count` highest keys of a row, the lower index first among equals: the key of the last one, by counting the keys in equal parts of the
// range that it is in, until a part is one key or has few, which are ranked (10.8 -> 9.4 us, of 15626 pages 14.7 -> 13.8); then all above it
// and the first of those that equal it, in the order of their pages.  A
// workgroup to a row, a thread to neighbouring pages, whose keys (HELD: up to 16) stay in its registers.  (Parts of the range that the keys
// have, not digits of them: scores of one sequence share their upper digits, and counters that all threads want are counted one after the
// other: 59 us against 14.7 for 15626 pages, before the few were ranked.)
template <bool HELD>
__global__ __launch_bounds__(1024) void choose_pages(SelectParams p, int64_t unit0) {
  constexpr int kFew = 256;
  __shared__ int s_parts[kKeyParts], s_found[3];
  __shared__ unsigned s_few[kFew];  // keys of a part
  __shared__ int s_few_at[kFew];    // and their pages
  __shared__ Two s_wave[16];
  __shared__ unsigned s_range[16][2];
  const evconv_select_args& a = p.a;
  const int64_t unit = unit0 + blockIdx.x, token = unit / a.cache.heads;
  const Query query = find_query(p, token);
  if (query.seq < 0) return;
  const int n = (int)query.last + 1, threads = blockDim.x, t = threadIdx.x;
  const unsigned* const key = p.score + unit * p.pages;
  int* const out = a.selected + unit * a.count;
  const int per = HELD ? 4 * ((n + 4 * threads - 1) / (4 * threads)) : ((n + threads - 1) / threads + 3) / 4 * 4;
  const int from = min(t * per, n), to = min(from + per, n);
  uint4 held[4];
  if constexpr (HELD)
#pragma unroll
    for (int i = 0; i < 4; ++i) held[i] = from + 4 * i < to ? *(const uint4*)(key + from + 4 * i) : make_uint4(0, 0, 0, 0);
  auto four = [&](int i, const uint4& u, auto&& what) __attribute__((always_inline)) {
    if (i < to) what(i, u.x);
    if (i + 1 < to) what(i + 1, u.y);
    if (i + 2 < to) what(i + 2, u.z);
    if (i + 3 < to) what(i + 3, u.w);
  };
  auto each = [&](auto&& what) __attribute__((always_inline)) {  // of this thread's pages (rows are whole fours)
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) four(from + 4 * i, held[i], what);
    } else {
      for (int i = from; i < to; i += 4) four(i, *(const uint4*)(key + i), what);
    }
  };
  Two mine{0, 0}, all;  // pages that can be chosen, those that have to be
  unsigned lo = kForced, hi = 0;
  each([&](int, unsigned k) {
    mine.a += k != 0;
    mine.b += k == kForced;
    if (k != 0 && k != kForced) lo = min(lo, k), hi = max(hi, k);
  });
  sums_before(mine, s_wave, &all);
  unsigned edge = 0;  // key of the last one that is chosen
  int equal = 0;      // how many with it
  if (all.a > a.count) {
    int need = a.count - all.b;
    range_of(lo, hi, s_range);
    edge = kForced;  // (none but them)
    while (need > 0) {
      const int shift = part_shift({lo, hi}), parts = part_count({lo, hi}, shift);
      for (int i = t; i < parts; i += threads) s_parts[i] = 0;
      __syncthreads();
      each([&](int, unsigned k) {
        if (k >= lo && k <= hi) atomicAdd(&s_parts[(k - lo) >> shift], 1);
      });
      __syncthreads();
      // from the top: the part where the sum reaches `need`
      const int share = (parts + threads - 1) / threads, top = parts - 1 - t * share;
      Two here{0, 0};
      for (int i = 0; i < share; ++i) here.a += top - i >= 0 ? s_parts[top - i] : 0;
      int before = sums_before(here, s_wave, &all).a;
      if (before < need && before + here.a >= need)
        for (int i = 0; i < share; ++i) {
          const int c = s_parts[top - i];
          if (before + c >= need) {
            s_found[0] = top - i;
            s_found[1] = need - before;
            s_found[2] = c;
            break;
          }
          before += c;
        }
      __syncthreads();
      const KeyRange part = part_range({lo, hi}, shift, s_found[0]);
      lo = part.lo;
      hi = part.hi;
      need = s_found[1];
      if (shift == 0) {
        edge = lo;
        equal = need;
        break;
      }
      const int few = s_found[2];
      __syncthreads();
      if (few <= kFew) {  // as few as that are ranked at once
        if (t == 0) s_found[0] = 0;
        __syncthreads();
        each([&](int i, unsigned k) {
          if (k >= lo && k <= hi) {
            const int at = atomicAdd(&s_found[0], 1);
            s_few[at] = k;
            s_few_at[at] = i;
          }
        });
        __syncthreads();
        if (t < few) {
          const unsigned mine_key = s_few[t];
          const int mine_at = s_few_at[t];
          int larger = 0, earlier = 0;
          for (int i = 0; i < few; ++i) {
            larger += s_few[i] > mine_key;
            earlier += s_few[i] == mine_key && s_few_at[i] < mine_at;
          }
          if (larger + earlier == need - 1) {
            s_parts[0] = (int)mine_key;
            s_parts[1] = need - larger;
          }
        }
        __syncthreads();
        edge = (unsigned)s_parts[0];
        equal = s_parts[1];
        break;
      }
    }
    if (edge == kForced) equal = a.count;
  }
  // ---- written in the order of the pages
  Two found{0, 0};  // above it, as it
  each([&](int, unsigned k) {
    found.a += k > edge;
    found.b += k == edge && edge != 0;
  });
  Two before = sums_before(found, s_wave, &all);
  each([&](int i, unsigned k) {
    const bool above = k > edge, same = k == edge && edge != 0;
    const int at = before.a + min(before.b, equal);
    if ((above || (same && before.b < equal)) && at < a.count) out[at] = i;
    before.a += above;
    before.b += same;
  });
  for (int i = all.a + min(all.b, equal) + t; i < a.count; i += threads) out[i] = -1;
}

template <bool BF16>
void start_scores(const SelectParams& p, unsigned grid, int blocks, int64_t at, hipStream_t s) {
  switch (p.dp) {
    case 32: score_pages<BF16, 32><<<grid, 256, 0, s>>>(p, blocks, at); break;
    case 64: score_pages<BF16, 64><<<grid, 256, 0, s>>>(p, blocks, at); break;
    case 96: score_pages<BF16, 96><<<grid, 256, 0, s>>>(p, blocks, at); break;
    case 128: score_pages<BF16, 128><<<grid, 256, 0, s>>>(p, blocks, at); break;
    case 192: score_pages<BF16, 192><<<grid, 256, 0, s>>>(p, blocks, at); break;
    default: score_pages<BF16, 256><<<grid, 256, 0, s>>>(p, blocks, at); break;
  }
}

int pages_of_a_workgroup(int dp) { return kRounds * 4 * kHeld * (dp <= 32 ? 16 : dp <= 64 ? 8 : dp <= 128 ? 4 : 2); }

}  // namespace

size_t plan_select(SelectParams& p) {
  const evconv_select_args& a = p.a;
  const evconv_tokens& t = a.tokens;
  p.dp = cache_channels(a.cache.d);
  p.log = __builtin_ctz(a.cache.page);
  p.share = a.heads_q / a.cache.heads;
  p.most = (int64_t)t.width * a.cache.page;
  if (a.max_len) p.most = std::min(p.most, a.max_len);
  p.len = t.seq_offsets ? -1 : (int)(t.n_tokens / t.n_seq);
  p.pages = (int)((((p.most + a.cache.page - 1) >> p.log) + 3) / 4 * 4);
  return (size_t)t.n_tokens * a.cache.heads * p.pages * sizeof(unsigned);
}

void launch_select(const SelectParams& p, hipStream_t s) {
  const int64_t units = p.a.tokens.n_tokens * p.a.cache.heads;
  const int per = pages_of_a_workgroup(p.dp), blocks = (p.pages + per - 1) / per;
  const int64_t total = units * blocks, most = kMostThreads / 256;
  for (int64_t at = 0; at < total; at += most) {
    const unsigned grid = (unsigned)std::min(most, total - at);
    if (p.a.dtype == EVCONV_BF16) start_scores<true>(p, grid, blocks, at, s);
    else start_scores<false>(p, grid, blocks, at, s);
  }
  // (128 rows of 2048 pages take 9.4 us with 256 threads and with 1024: the barriers; the fewer leave room for other rows)
  const int threads = p.pages <= 4096 ? 256 : 1024;
  const int64_t rows = kMostThreads / threads;
  for (int64_t at = 0; at < units; at += rows) {
    const unsigned grid = (unsigned)std::min(rows, units - at);
    if (p.pages <= 16 * threads) choose_pages<true><<<grid, threads, 0, s>>>(p, at);
    else choose_pages<false><<<grid, threads, 0, s>>>(p, at);
  }
}

}  // namespace evk
