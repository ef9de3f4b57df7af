// The gated delta rule in chunks, one launch (bf16 keys of up to 128 channels; formulas and precision: kernels_delta.hip).
//
// A workgroup owns a sequence's value head and NC strips of 16 state columns, a wave each (a consumer), and goes
// through the chunks; two pairs of further waves (producers) take turns at preparing the chunks ahead: T and P, which do
// not depend on the state.  Nothing that is computed once leaves the compute unit: keys and queries are read once into LDS
// (the transposed operand K' comes from the same rows by transposing LDS reads), T and P go from producer to
// consumer through a ring of three slots, S, R and D stay in their lanes (kernels_delta.hip: place).
//
// A step of the chip full of workgroups (heads of 128 x 128) takes 9 us, 18 thousand cycles, of which a SIMD spends 9 to 11 thousand on
// vector instructions (parts of S, R and D, exponentials, T's substitution) and 7 thousand on matrix instructions: together the step.
// They hardly run beside each other, for all waves meet once a step, so that the two consumers of a SIMD split at the same time and
// multiply at the same time; beside each other the same instructions would fit into 11 thousand.  8 sequences of 4096 tokens and
// 32 heads: 0.55 ms, where the rows and states alone would take 0.16; prepared by a launch of its own they took 3.6.
// Measured without gain: a pair of producers instead of two in workgroups of four strips; more priority to half of the consumers (slower).
//
// In step c (all waves meet once per step) the consumers apply chunk c and bring in the rows of chunk c + 1; a pair of producers
// computes K K', Q K' and A of chunk c + 2, the other pair T of chunk c + 1.
#include <algorithm>

#include "delta_device.h"

namespace evk {
namespace {

constexpr int kStrideA = 68;  // floats between the rows of A and T: rows of a load instruction in different banks

// Orders what lanes of one wave hand to each other through LDS (which serves a wave's requests in order).
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }

template <int DKP, int NC>
struct FusedShape {
  static constexpr int kSteps = DKP / 32;
  static constexpr int kOffP = kTri * 3 * kFrag, kOffScal = kOffP + kTri * 2 * kFrag, kSlot = kOffScal + 5 * C * 4;
  static constexpr int kRows = C * DKP * 2;  // bytes of a chunk's K (or Q)
  static constexpr int kOffK = 3 * kSlot, kOffTemp = kOffK + 4 * kRows, kBytes = kOffTemp + 2 * 3 * C * 4;
  static constexpr int kThreads = (NC + 4) * 64;
  static_assert(C * kStrideA * 4 <= kOffP && kBytes <= 160 * 1024, "LDS");
};
// Place of the 16-byte piece c of row `row` of K (Q) in LDS: the 16 rows of an operand load, and the four rows of a
// transposing one, in different banks.
template <int DKP>
__device__ __forceinline__ int at_rows(int row, int c) {
  const int f = DKP == 128 ? (row & 3) << 2 | (row >> 3 & 3) : (row >> 1 & 1) << 2 | (row >> 3 & 3);
  return row * DKP * 2 + ((c ^ f) << 4);
}

// Addresses: a part that is the same for a whole wave (64 bits, scalar registers) and a lane's bytes (32 bits).
// A value that is the same for a whole wave, kept out of the compiler's sight: it would otherwise add a lane's part once
// before the loop and hold dozens of 64-bit addresses in vector registers through it.
// (Global by type: the compiler could not tell any more, and loads that may be LDS wait for LDS, too.)
#define EVK_GLOBAL __attribute__((address_space(1)))
__device__ __forceinline__ EVK_GLOBAL char* uniform(const void* q) {
  EVK_GLOBAL char* r = (EVK_GLOBAL char*)q;
  asm volatile("" : "+s"(r));
  return r;
}
// base + a lane's bytes, by an instruction that adds the two itself (the extension to 64 bits has to be in sight of it)
template <class T>
__device__ __forceinline__ EVK_GLOBAL T* lane_at(const void* base, unsigned lane_bytes) {
  asm volatile("" : "+v"(lane_bytes));
  return (EVK_GLOBAL T*)(uniform(base) + lane_bytes);
}
// This wave's lane, likewise out of sight: what is derived from it is computed where it is used, not kept for all of a loop.
__device__ __forceinline__ int own_lane() {
  int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));  // (not of the thread's index, which would be)
  asm volatile("" : "+v"(lane));
  return lane;
}
// Eight bf16 of a row as they are, the first of `left` that the row has from there on
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
template <bool VEC>
__device__ __forceinline__ u32x4 load_raw(const char* base, unsigned lane_bytes, int left) {
  u32x4 u = {0, 0, 0, 0};
  if (left <= 0) return u;
  if (VEC) {
    u = *lane_at<const u32x4>(base, lane_bytes);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) u[j / 2] |= (unsigned)*lane_at<const uint16_t>(base + j * 2, lane_bytes) << (j % 2 * 16);
    __builtin_amdgcn_sched_barrier(0);
  }
  return u;
}
// Whether one of eight bf16 is not finite, as bits 15 and 31 of the result
__device__ __forceinline__ unsigned not_finite(const u32x4& u) {
  unsigned r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= (u[i] & 0x7f807f80u) + 0x00800080u;
  return r & 0x80008000u;
}
// Rows of a head: of a chunk's first token, and the bytes from token to token
struct Rows {
  const char* at;
  int step;
  __device__ __forceinline__ void next(int chunks) { at += (int64_t)chunks * C * step; }
};
__device__ __forceinline__ Rows rows_of(const evconv_heads& h, int size, int head, int64_t token) {
  return {(const char*)h.data + (token * h.token_stride + head * h.head_stride) * size, (int)h.token_stride * size};
}

// What a producer reads.
template <bool VEC>
struct Source {
  Rows k, q, gate, beta;
  int d_k, left;          // tokens from the first of k on
  float a_scale, dt_bias;
  bool gate_bf16;
};
// What it holds of a chunk ahead of its turn: block b of an operand is the tokens place(b, .), so that a pair of blocks spans
// 32 tokens.
template <int DKP>
struct Ahead {
  b16x8 k[4][DKP / 32], q[2][DKP / 32];
  float gate, beta;  // as they are in memory
};
template <int DKP, bool VEC>
__device__ __forceinline__ void request_blocks(const Rows& r, int d_k, int left, int block0, b16x8 (*to)[DKP / 32], int blocks) {
  const int lane = own_lane(), m = lane & 15, g = lane >> 4;
  if (VEC && d_k == DKP) {
    // (loads under conditions of their own would be waited for one by one: tokens behind the end are the last one again, whose
    // rows of A and P count for nothing)
#pragma unroll
    for (int b = 0; b < blocks; ++b) {
      const unsigned at = (unsigned)(min(place(block0 + b, m), left - 1) * r.step + 16 * g);
#pragma unroll
      for (int s = 0; s < DKP / 32; ++s) to[b][s] = *lane_at<const b16x8>(r.at + 64 * s, at);
    }
    return;
  }
#pragma unroll
  for (int b = 0; b < blocks; ++b)
#pragma unroll
    for (int s = 0; s < DKP / 32; ++s)
      to[b][s] = __builtin_bit_cast(b16x8, load_raw<VEC>(r.at + 64 * s, (unsigned)(place(block0 + b, m) * r.step + 16 * g), place(block0 + b, m) < left ? d_k - 32 * s - 8 * g : 0));
}
// Row blocks of A and P that each of the two producers of a chunk computes: as many products each.
__device__ __forceinline__ constexpr int row_block(int role, int n) { return role == 0 ? 3 * n : 1 + n; }
template <int DKP, bool VEC, bool TRANS, int ROLE>
__device__ __forceinline__ void request_ahead(const Source<VEC>& f, Ahead<DKP>& to) {
  request_blocks<DKP, VEC>(f.k, f.d_k, f.left, 0, to.k, 4);
  if (!TRANS) request_blocks<DKP, VEC>(f.q, f.d_k, f.left, row_block(ROLE, 0), to.q, 1);
  const int t = own_lane();
  const EVK_GLOBAL char *const gates = uniform(f.gate.at), *const betas = uniform(f.beta.at);
  unsigned at_g = (unsigned)(t * f.gate.step), at_b = (unsigned)(t * f.beta.step);
  asm volatile("" : "+v"(at_g), "+v"(at_b));
  to.gate = to.beta = 0.0f;
  if (t < f.left) {
    if (f.gate_bf16) {
      to.gate = bf16_low(*(const EVK_GLOBAL uint16_t*)(gates + at_g));
      to.beta = bf16_low(*(const EVK_GLOBAL uint16_t*)(betas + at_b));
    } else {
      to.gate = *(const EVK_GLOBAL float*)(gates + at_g);
      to.beta = *(const EVK_GLOBAL float*)(betas + at_b);
    }
  }
}

// First half of a chunk's preparation, by two waves: A (fp32, in the place of T), P, the factors of the rows.
template <int DKP, bool VEC, bool TRANS, int ROLE>
__device__ __forceinline__ void prepare_products(const DeltaParams& p, char* slot, float* temp, const Source<VEC>& f, int left, Ahead<DKP>& x) {
  typedef FusedShape<DKP, 8> F;
  constexpr int STEPS = F::kSteps;
  const evconv_delta_args& a = p.a;
  const int lane = own_lane(), m = lane & 15, g = lane >> 4;
  float* const s_a = (float*)slot;
  float* const scal = (float*)(slot + F::kOffScal);
  float *const s_hi = temp, *const s_lo = temp + C, *const s_rk = temp + 2 * C;
  if (!TRANS) request_blocks<DKP, VEC>(f.q, f.d_k, left, row_block(ROLE, 1), &x.q[1], 1);
  // ---- a token to a lane: sums of log2 decays, as two floats each, so that differences keep their bits
  Gates gate = {0.0f, 0.0f};
  if (lane < left) gate = gates_from(a.flags & EVCONV_DELTA_RAW_GATES, x.gate, x.beta, f.a_scale, f.dt_bias);
  double sum = (double)gate.g * 1.44269504088896340736;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double other = __shfl_up(sum, d);
    if (lane >= d) sum += other;
  }
  const float hi = (float)sum, lo = isfinite(hi) ? (float)(sum - (double)hi) : 0.0f;
  s_hi[lane] = hi;
  s_lo[lane] = lo;
  // ---- norms: diagonals of K K' and Q Q', which lanes with m / 4 == g hold
  const bool normalize = a.flags & EVCONV_DELTA_NORMALIZE;
  auto diagonal = [&](const b16x8 (&v)[STEPS]) __attribute__((always_inline)) {
    f32x4 u = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[s], v[s], u, 0, 0, 0);
    return m & 2 ? (m & 1 ? u[3] : u[2]) : (m & 1 ? u[1] : u[0]);
  };
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const float u = diagonal(x.k[b]);
    if (m >> 2 == g) s_rk[place(b, m)] = u;
  }
  wave_order();
  // A token whose row of A cannot be finite: from the first one on the rows are NaN, by their beta, and zero in A, whose
  // zeros would otherwise carry them to rows above them.  (A sum of squares bounds the products of its key.)
  const float square = s_rk[lane];
  const uint64_t wrong = __ballot(!(fabsf(square) < INFINITY) || !(fabsf(gate.beta) < INFINITY) || !(fabsf(hi) < INFINITY));
  const int bad = wrong ? (int)__builtin_ctzll(wrong) : C;
  const float rk = normalize ? 1.0f / norm_of(square) : 1.0f;
  s_rk[lane] = rk;
  const float beta_rk = lane < bad ? gate.beta * rk : 0.0f;
  __builtin_amdgcn_sched_barrier(0);
  // ---- rows 16 at a time
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int bi = row_block(ROLE, n), i = place(bi, m);
    const b16x8 (&q)[STEPS] = x.q[n];
    wave_order();
    const float hi_i = s_hi[i], lo_i = s_lo[i], br = __shfl(beta_rk, i);
    const bool good = i < bad;
    float rq = a.scale;
    if (!TRANS) {
      if (normalize) rq = a.scale / norm_of(__shfl(diagonal(q), (m >> 2) << 4 | m));
      if (g == 0) scal[2 * C + i] = rq * __builtin_amdgcn_exp2f(hi_i);
    }
    // a lane holds of block j the row i = place(bi, m) of A and P, columns j0 .. j0 + 3
#pragma unroll
    for (int pair = 0; pair < 1 + (bi >> 1); ++pair) {
      const bool below = pair < bi >> 1;  // all of these columns are of earlier tokens
      // there e^{G_i - G_j} is a factor of the row times one of the column, both of token 31's distance
      const float hi_m = s_hi[31], lo_m = s_lo[31];
      float bru = br, rqu = rq;
      if (below) {
        const float u = __builtin_amdgcn_exp2f((hi_i - hi_m) + (lo_i - lo_m));
        bru *= u;
        rqu *= u;
      }
      f32x4 kk[2], kq[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) kk[h] = kq[h] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          kk[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.k[2 * pair + h][s], x.k[bi][s], kk[h], 0, 0, 0);
          if (!TRANS) kq[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.k[2 * pair + h][s], q[s], kq[h], 0, 0, 0);
        }
      float v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j0 = place(2 * pair + h, 4 * g);
        const f32x4 hi_j = *(const f32x4*)(s_hi + j0), lo_j = *(const f32x4*)(s_lo + j0), rk_j = *(const f32x4*)(s_rk + j0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = rk_j[e] * __builtin_amdgcn_exp2f(below ? (hi_m - hi_j[e]) + (lo_m - lo_j[e]) : (hi_i - hi_j[e]) + (lo_i - lo_j[e]));
          // (selected, not multiplied: what is above the diagonal, or of bad rows, may be anything)
          kk[h][e] = good && (below || j0 + e < i) ? bru * w * kk[h][e] : 0.0f;
          v[4 * h + e] = below || j0 + e <= i ? rqu * w * kq[h][e] : 0.0f;
        }
        *(f32x4*)(s_a + i * kStrideA + j0) = kk[h];
      }
      if (!TRANS) {
        b16x8 out[2];
        split8(v, out);
#pragma unroll
        for (int part = 0; part < 2; ++part) *(b16x8*)(slot + F::kOffP + (tri(bi, pair) * 2 + part) * kFrag + lane * 16) = out[part];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (ROLE == 0) {
    const double last = __shfl(sum, 63);
    scal[lane] = lane < bad ? gate.beta : NAN;
    scal[C + lane] = gate.beta * rk * __builtin_amdgcn_exp2f(hi);
    scal[3 * C + lane] = rk * __builtin_amdgcn_exp2f((float)(last - sum));
    scal[4 * C + lane] = __builtin_amdgcn_exp2f((float)last);
  }
}

// Second half: T = (I + A)^-1 in A's place (the method: delta_prepare), then as left operands.
template <int DKP>
__device__ __forceinline__ void prepare_inverse(char* slot) {
  const int lane = own_lane(), m = lane & 15, g = lane >> 4;
  float* const t = (float*)slot;
  {
    // diagonal block g, column m
    float x[16];
    const float* const at = t + g * 16 * kStrideA + g * 16;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float sum = i == m ? 1.0f : 0.0f;
#pragma unroll
      for (int l = 0; l < i; ++l) sum = fmaf(-at[i * kStrideA + l], x[l], sum);
      x[i] = sum;
      if (i & 1) __builtin_amdgcn_sched_barrier(0);
    }
    wave_order();
#pragma unroll
    for (int i = 0; i < 16; ++i) t[(g * 16 + i) * kStrideA + g * 16 + m] = x[i];
    wave_order();
  }
  // a 16 x 16 block of X Y, n blocks of 16 deep; blocks by their row and column
  auto product = [&](f32x4& acc, int xr, int xc, int yr, int yc, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < n * 16; c += 4)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(t[(xr * 16 + m) * kStrideA + xc * 16 + c + g], t[(yr * 16 + c + g) * kStrideA + yc * 16 + m], acc, 0, 0, 0);
  };
  auto put = [&](const f32x4& v, int r, int c, float sign) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[(r * 16 + 4 * g + i) * kStrideA + c * 16 + m] = sign * v[i];
  };
  const f32x4 zero = {0, 0, 0, 0};
  {
    f32x4 x[2] = {zero, zero}, y[2] = {zero, zero};
#pragma unroll
    for (int h = 0; h < 2; ++h) product(x[h], 2 * h + 1, 2 * h, 2 * h, 2 * h, 1);
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) put(x[h], 2 * h + 1, 2 * h, 1.0f);
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) product(y[h], 2 * h + 1, 2 * h + 1, 2 * h + 1, 2 * h, 1);
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h) put(y[h], 2 * h + 1, 2 * h, -1.0f);
    wave_order();
  }
  {
    f32x4 x[2][2] = {{zero, zero}, {zero, zero}}, y[2][2] = {{zero, zero}, {zero, zero}};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      product(x[r][0], 2 + r, 0, 0, 0, 2);
      product(x[r][1], 2 + r, 1, 1, 1, 1);  // (the block above T11's diagonal is zero)
    }
    wave_order();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < 2; ++c) put(x[r][c], 2 + r, c, 1.0f);
    wave_order();
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      product(y[0][c], 2, 2, 2, c, 1);
      product(y[1][c], 3, 2, 2, c, 2);
    }
    wave_order();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < 2; ++c) put(y[r][c], 2 + r, c, -1.0f);
    wave_order();
  }
  float v[kTri][8];
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int f = 0; f < kTri; ++f) {
    const int b = f < 2 ? f : 2 + (f - 2) / 2, s = f < 2 ? 0 : (f - 2) % 2;
    const int row = place(b, m), col = 32 * s + 8 * g;
    const f32x4 u = *(const f32x4*)(t + row * kStrideA + col), w = *(const f32x4*)(t + row * kStrideA + col + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[f][e] = e < 4 ? u[e] : w[e - 4];  // (zeros above the diagonal are there)
  }
  wave_order();
#pragma unroll
  for (int f = 0; f < kTri; ++f) {
    b16x8 out[3];
    split8(v[f], out);
#pragma unroll
    for (int part = 0; part < 3; ++part) *(b16x8*)(slot + (f * 3 + part) * kFrag + lane * 16) = out[part];
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The instructions since the last scheduling barrier in turns: a matrix instruction, then `vector` vector instructions, which run
// beside it.
template <int MATRIX, int VECTOR>
__device__ __forceinline__ void beside() {
#pragma unroll
  for (int i = 0; i < MATRIX; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// All waves of a workgroup; what they wrote to LDS is there behind it.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A producer: every other chunk; the first half of chunk x in step x - 2, the second in step x - 1 (ROLE 0; the other
// one of the pair has nothing to do there).
template <int DKP, int NC, bool VEC, bool TRANS, int ROLE>
__device__ __forceinline__ void produce(const DeltaParams& p, char* s_mem, const Span& span, int chunks, int x, int head, int hk) {
  typedef FusedShape<DKP, NC> F;
  const evconv_delta_args& a = p.a;
  float* const temp = (float*)(s_mem + F::kOffTemp) + ROLE * 3 * C;
  int left = chunks + 2;  // steps to come
  if (x == 1) {
    meet();
    --left;
  }
  __builtin_amdgcn_s_setprio(2);  // (the consumers wait for it)
  Source<VEC> f;
  f.gate_bf16 = a.gate_dtype == EVCONV_BF16;
  // (where it has no further chunk it requests its last, or the sequence's last, once more: every request is for tokens that exist)
  const int from = min(x, chunks - 1);
  const int64_t first = span.first + (int64_t)from * C;
  f.k = rows_of(a.k, 2, hk, first);
  f.q = rows_of(a.q, 2, hk, first);
  f.gate = rows_of(a.gate, f.gate_bf16 ? 2 : 4, head, first);
  f.beta = rows_of(a.beta, f.gate_bf16 ? 2 : 4, head, first);
  f.d_k = a.d_k;
  f.left = span.len - from * C;
  f.a_scale = a.flags & EVCONV_DELTA_RAW_GATES ? a.a_scale[head] : 0.0f;
  f.dt_bias = a.flags & EVCONV_DELTA_RAW_GATES ? a.dt_bias[head] : 0.0f;
  Ahead<DKP> ahead;
  request_ahead<DKP, VEC, TRANS, ROLE>(f, ahead);
#pragma unroll 1
  for (; left > 0; x += 2) {
    char* const slot = s_mem + x % 3 * F::kSlot;
    if (x < chunks) prepare_products<DKP, VEC, TRANS, ROLE>(p, slot, temp, f, f.left, ahead);
    meet();
    if (--left == 0) break;
    const int on = x + 2 < chunks ? 2 : 0;
    f.k.next(on);
    f.q.next(on);
    f.gate.next(on);
    f.beta.next(on);
    f.left -= on * C;
    request_ahead<DKP, VEC, TRANS, ROLE>(f, ahead);
    if (ROLE == 0 && x < chunks) prepare_inverse<DKP>(slot);
    meet();
    --left;
  }
}

// Few heads and long sequences: segments of a sequence side by side (p.segs of p.seg_chunks chunks).  What a segment does to the
// state it starts from is S -> M S + N, so a first launch (TRANS: no outputs) runs the segments from zero, which gives N, and
// with the columns of the unit matrix as further columns of a state and no values, which gives M (the first
// segment from the given state; the last one is not needed); delta_join goes through them; the second launch runs
// every segment from its start.
template <int DKP, int NC, bool VEC, bool TRANS>
__global__ __launch_bounds__((NC + 4) * 64) void delta_fused(DeltaParams p) {
  typedef FusedShape<DKP, NC> F;
  constexpr int STEPS = F::kSteps, PIECES = 2 * C * (DKP / 8) / (NC * 64);
  extern __shared__ __align__(16) char s_mem[];
  const evconv_delta_args& a = p.a;
  const int strips_v = (a.d_v + 15) / 16, strips = strips_v + (TRANS ? (a.d_k + 15) / 16 : 0), parts = (strips + NC - 1) / NC;
  const int part = blockIdx.x % parts, segs = TRANS ? p.segs - 1 : p.segs, seg = blockIdx.x / parts % segs;
  const int64_t pair = blockIdx.x / parts / segs;
  const int seq = (int)(pair / a.heads_v), head = (int)(pair % a.heads_v), hk = head / p.share;
  Span span = span_of(p, seq);
  if (span.len <= p.short_len) return;
  {
    const int64_t skip = (int64_t)seg * p.seg_chunks * C;
    if (span.len <= skip + (TRANS ? p.seg_chunks * C : 0)) return;  // (TRANS: nothing behind it)
    if (TRANS && seg == 0 && part * NC >= strips_v) return;
    span.first += (int)skip;
    span.len -= (int)skip;
  }
  const bool last = span.len <= p.seg_chunks * C;
  span.len = min(span.len, p.seg_chunks * C);
  const int chunks = (span.len + C - 1) / C;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= NC) {  // a producer
    const int which = wave - NC;
    if (which < 2) produce<DKP, NC, VEC, TRANS, 0>(p, s_mem, span, chunks, which & 1, head, hk);
    else produce<DKP, NC, VEC, TRANS, 1>(p, s_mem, span, chunks, which & 1, head, hk);
    return;
  }
  const int strip = part * NC + wave;
  const bool unit_columns = TRANS && strip >= strips_v;
  const bool works = strip < strips && !(unit_columns && seg == 0);
  const int64_t at = state_at(p, seq, head);
  const int ld = TRANS ? strips * 16 : (strips_v + (a.d_k + 15) / 16) * 16;  // floats between the rows of p.trans
  float* const trans = p.trans + (pair * p.segs + seg) * a.d_k * (int64_t)ld;  // N, M; behind delta_join N is the next segment's start
  float* const start0 = p.start0 + pair * a.d_k * (int64_t)(strips_v * 16);    // (the first segment's: its place may be state_out's)
  f32x4 S[2 * STEPS];
  {
    const int lane = own_lane(), col = strip * 16 + (lane & 15), g = lane >> 4;
    const float* from = a.state_in ? a.state_in + at : nullptr;
    int width = a.d_v;
    bool there = at >= 0 && a.state_in && col < a.d_v;
    if (TRANS) there &= seg == 0;
    else if (seg || !last) {
      from = seg ? p.trans + (pair * p.segs + seg - 1) * a.d_k * (int64_t)ld : start0;
      width = seg ? ld : strips_v * 16;
      there = strip < strips_v;
    }
#pragma unroll
    for (int b = 0; b < 2 * STEPS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = place(b, 4 * g + i);
        S[b][i] = there && row < a.d_k ? ((const EVK_GLOBAL float*)from)[row * width + col] : unit_columns && row == col - strips_v * 16 ? 1.0f : 0.0f;
      }
    if (TRANS && seg == 0 && works)
#pragma unroll
      for (int b = 0; b < 2 * STEPS; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = place(b, 4 * g + i);
          if (row < a.d_k) start0[row * strips_v * 16 + col] = S[b][i];
        }
#pragma unroll
    for (int b = 0; b < 2 * STEPS; ++b) asm volatile("" : "+v"(S[b]));  // (waited for here, or the loop would wait in every turn)
  }
  const int64_t before = span.first - (int64_t)C;
  Rows k_rows = rows_of(a.k, 2, hk, before), q_rows = rows_of(a.q, 2, hk, before);  // of chunk c + 1
  Rows v_rows = rows_of(a.v, 2, head, before);
  Rows o_rows = {(const char*)a.o + ((before - C) * a.o_token_stride + head * a.o_head_stride) * 2, (int)a.o_token_stride * 2};  // of c
  u32x4 value[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};  // this lane's part of v, see `unit`
  constexpr int HALF = PIECES / 2, PIECE_ROWS = NC * 64 / (DKP / 8);  // K's pieces, then Q's; rows of one round of them
  // The chunk's values as left operands: 16 bytes of a token's row to a lane, of blocks 2 p and 2 p + 1 of tokens (their columns as
  // the contraction's first and last 16 places).  A product with half a unit matrix brings them into the layout of results,
  // and o's values back out of it: two loads and four stores a chunk where lanes' own places would take 16 of two bytes each.
  // (Not where some value is not finite: the zeros would carry it to others.)
  auto unit = [](int lane, int half) __attribute__((always_inline)) {
    const int n = lane & 15, at = (n >> 1) - 4 * (lane >> 4) + 8 * half;  // which pair of this lane's places has the one
    const unsigned one = n & 1 ? 0x3f800000u : 0x3f80u;
    u32x4 u;
#pragma unroll
    for (int d = 0; d < 4; ++d) u[d] = at == d ? one : 0u;
    return __builtin_bit_cast(b16x8, u);
  };
#pragma unroll 1
  for (int c = -2; c < chunks; ++c) {
    const int64_t token0 = span.first + (int64_t)c * C;
    const int count = min(span.len - c * C, C);
    const char* const slot = s_mem + (c + 3) % 3 * F::kSlot;
    const float* const scal = (const float*)(slot + F::kOffScal);
    const char* const rows = s_mem + F::kOffK + (c & 1) * 2 * F::kRows;
    const bool now = c >= 0 && works, more = c + 1 >= 0 && c + 1 < chunks;
    // ---- rows of the next chunk, into the buffer that the last step has done with
    if (more) {
      const int left = span.len - (c + 1) * C, lane = own_lane();
      char* const to = s_mem + F::kOffK + ((c + 1) & 1) * 2 * F::kRows;
      if (VEC && a.d_k == DKP) {
        // straight into LDS, a wave 64 neighbouring places, which at_rows' exclusive or makes those of other pieces of the row.
        // (A token behind the end is the last one again: its rows of R and D are zero.)
#pragma unroll
        for (int i = 0; i < (TRANS ? HALF : PIECES); ++i) {
          const Rows& r = i < HALF ? k_rows : q_rows;
          const int first = i % HALF * PIECE_ROWS + wave * (512 / DKP), row = first + lane / (DKP / 8), at = lane % (DKP / 8) * 16;
          const int piece = at ^ (at_rows<DKP>(row, 0) - row * DKP * 2);
          __builtin_amdgcn_global_load_lds(lane_at<const u32x4>(r.at, (unsigned)(min(row, left - 1) * r.step + piece)),
                                           (__attribute__((address_space(3))) void*)(to + (i < HALF ? 0 : F::kRows) + first * DKP * 2), 16, 0, 0);
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < (TRANS ? HALF : PIECES); ++i) {
          const Rows& r = i < HALF ? k_rows : q_rows;
          const int row = i % HALF * PIECE_ROWS + wave * (512 / DKP) + lane / (DKP / 8), piece = lane % (DKP / 8);
          *(u32x4*)(to + (i < HALF ? 0 : F::kRows) + at_rows<DKP>(row, piece)) =
              load_raw<VEC>(r.at, (unsigned)(row * r.step + piece * 16), row < left ? a.d_k - piece * 8 : 0);
        }
      }
    }
    f32x4 R[4], O[4];
    if (now) {
      // ---- K S and Q S
      const int lane = own_lane(), n = lane & 15, g = lane >> 4;
      const int at_k = at_rows<DKP>(place(0, n), g);
#pragma unroll
      for (int b = 0; b < 4; ++b) R[b] = O[b] = f32x4{0, 0, 0, 0};
      b16x8 Sp[2][3];
      auto split_s = [&](int s) __attribute__((always_inline)) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = S[2 * s][i];
          v[4 + i] = S[2 * s + 1][i];
        }
        split8(v, Sp[s & 1]);
      };
      split_s(0);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        // (operands requested together: left alone, each read would be waited for by itself)
        const char* const at_s = rows + (at_k ^ (s << 6));  // (another piece of the row, by exclusive or; blocks of rows by addition)
        b16x8 k[4][1], q[4][1];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          k[b][0] = *(const b16x8*)(at_s + place(b, 0) * DKP * 2);
          if (!TRANS) q[b][0] = *(const b16x8*)(at_s + F::kRows + place(b, 0) * DKP * 2);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (s + 1 < STEPS) split_s(s + 1);
        mfma_parts<2, 4>(R, k, Sp[s & 1]);
        if (!TRANS) mfma_parts<1, 4>(O, q, Sp[s & 1]);
        beside<TRANS ? 12 : 20, 2>();
      }
      // ---- R = beta v - beta e^G K S;  e^G Q S   (behind the sequence's end all of them are zero)
      const b16x8 half[2] = {unit(lane, 0), unit(lane, 1)};
      const bool plain_v = !__ballot((not_finite(value[0]) | not_finite(value[1])) != 0);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t0 = place(b, 4 * g);  // this lane's tokens: t0 .. t0 + 3
        f32x4 v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, value[b >> 1]), half[b & 1], f32x4{0, 0, 0, 0}, 0, 0, 0);
        if (!plain_v)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = t0 + i < count && strip * 16 + n < a.d_v ? load_one<true>(a.v.data, (token0 + t0 + i) * a.v.token_stride + head * a.v.head_stride + strip * 16 + n) : 0.0f;
        const f32x4 beta = *(const f32x4*)(scal + t0), kf = *(const f32x4*)(scal + C + t0), qf = *(const f32x4*)(scal + 2 * C + t0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          R[b][i] = beta[i] * v[i] - kf[i] * R[b][i];
          O[b][i] *= qf[i];
        }
        if (b & 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
    // ---- values of the next chunk
    if (more && works && !unit_columns) {
      const int left = span.len - (c + 1) * C;
      const int lane = own_lane(), m = lane & 15, g = lane >> 4, own = strip * 16 + (g & 1) * 8;
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        const int t = 32 * pair + place(g >> 1, m);
        if (VEC) value[pair] = *lane_at<const u32x4>(v_rows.at, (unsigned)(min(t, left - 1) * v_rows.step + (own < a.d_v ? own : 0) * 2));
        else value[pair] = load_raw<VEC>(v_rows.at, (unsigned)(t * v_rows.step + own * 2), t < left ? a.d_v - own : 0);
      }
    }
    int first_bad = C;
    f32x4 D[4];
    if (now) {
      const int lane = own_lane(), g = lane >> 4;
      auto frag = [&](int off) __attribute__((always_inline)) { return *(const b16x8*)(slot + lane * 16 + off); };
      // ---- D = T R; a second time, without the columns' rows from the first bad one on, where some value is not finite
      auto apply_t = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 4; ++b) D[b] = f32x4{0, 0, 0, 0};
        b16x8 Rp[2][3], t[2][3];
        auto split_r = [&](int s) __attribute__((always_inline)) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = R[2 * s][i];
            v[4 + i] = R[2 * s + 1][i];
          }
          split8(v, Rp[s]);
        };
        auto read_t = [&](int b0, int s) __attribute__((always_inline)) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int part = 0; part < 3; ++part) t[b][part] = frag((tri(b0 + b, s) * 3 + part) * kFrag);
          __builtin_amdgcn_sched_barrier(0);
        };
        read_t(0, 0);
        split_r(0);
        __builtin_amdgcn_sched_barrier(0);
        split_r(1);
        mfma_parts<2, 2>(D, t, Rp[0]);
        beside<12, 4>();
        read_t(2, 0);
        mfma_parts<2, 2>(D + 2, t, Rp[0]);
        read_t(2, 1);
        mfma_parts<2, 2>(D + 2, t, Rp[1]);
        __builtin_amdgcn_sched_barrier(0);
      };
      apply_t();
      uint64_t wrong = 0;  // (a value of R that is not finite, or that a bf16 rounds to infinity, is in D too)
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) wrong |= __ballot(!(fabsf(D[b][i]) < kBf16Overflow));
      if (wrong) {
        cut_columns(R, bad_values(R), first_bad, g);
        apply_t();
        cut_columns(D, bad_values(D), first_bad, g);
      }
    }
    if (now) {
      const int lane = own_lane(), n = lane & 15, g = lane >> 4;
      auto frag = [&](int off) __attribute__((always_inline)) { return *(const b16x8*)(slot + lane * 16 + off); };
      // ---- O += P D;  S = e^G S + K' (w D)
      const float decay = scal[4 * C];
      const int at_t = at_rows<DKP>(8 * g + (n >> 2), n & 3);
      b16x8 pp[4][2], kt[STEPS][1], Dp[2], Dw[3];
      // tokens 32 s + 8 g .. + 7 of the channels place(b, .): two transposing reads of four tokens
      auto read_k = [&](int s, int b0) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < STEPS; ++b) {
          const char* const q = rows + (at_t ^ (((b0 + b) >> 1) << 6)) + 32 * s * DKP * 2 + ((b0 + b) & 1) * 8;
          typedef short s16x4 __attribute__((ext_vector_type(4)));
          typedef short s16x8 __attribute__((ext_vector_type(8)));
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)q);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q + 4 * DKP * 2));
          kt[b][0] = __builtin_bit_cast(b16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      };
      auto read_p = [&](int s) __attribute__((always_inline)) {
        if (!TRANS)
#pragma unroll
          for (int b = 2 * s; b < 4; ++b)
#pragma unroll
            for (int part = 0; part < 2; ++part) pp[b][part] = frag(F::kOffP + (tri(b, s) * 2 + part) * kFrag);
      };
      auto split_d = [&](int s) __attribute__((always_inline)) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = D[2 * s][i];
          v[4 + i] = D[2 * s + 1][i];
        }
        split8(v, Dp);
      };
      auto split_w = [&](int s) __attribute__((always_inline)) {
        const f32x4 w0 = *(const f32x4*)(scal + 3 * C + place(2 * s, 4 * g)), w1 = *(const f32x4*)(scal + 3 * C + place(2 * s + 1, 4 * g));
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = D[2 * s][i] * w0[i];
          v[4 + i] = D[2 * s + 1][i] * w1[i];
        }
        split8(v, Dw);
      };
      // (vector instructions in turns with matrix instructions that do not need them)
      read_p(0);
      __builtin_amdgcn_sched_barrier(0);
      if (!TRANS) split_d(0);
      __builtin_amdgcn_sched_barrier(0);
      split_w(0);
#pragma unroll
      for (int b = 0; b < 2 * STEPS; ++b) S[b] *= decay;
      if (!TRANS) mfma_parts<1, 4>(O, pp, Dp);
      beside<12, 6>();
      read_k(0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (!TRANS) split_d(1);
      mfma_parts<2, STEPS>(S, kt, Dw);
      beside<3 * STEPS, 3>();
      read_k(0, STEPS);
      read_p(1);
      __builtin_amdgcn_sched_barrier(0);
      mfma_parts<2, STEPS>(S + STEPS, kt, Dw);
      if (!TRANS) mfma_parts<1, 2>(O + 2, pp + 2, Dp);
      __builtin_amdgcn_sched_barrier(0);
      read_k(1, 0);
      split_w(1);
      __builtin_amdgcn_sched_barrier(0);
      mfma_parts<2, STEPS>(S, kt, Dw);
      __builtin_amdgcn_sched_barrier(0);
      read_k(1, STEPS);
      __builtin_amdgcn_sched_barrier(0);
      mfma_parts<2, STEPS>(S + STEPS, kt, Dw);
      __builtin_amdgcn_sched_barrier(0);
      if (__ballot(first_bad < C)) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (place(b, 4 * g) + i >= first_bad) O[b][i] = NAN;
        if (first_bad < C)
#pragma unroll
          for (int b = 0; b < 2 * STEPS; ++b) S[b] = f32x4{NAN, NAN, NAN, NAN};
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the next chunk's rows are in LDS (o's stores, which come now, are not waited for)
    if (!TRANS && now) {
      const int lane = own_lane(), n = lane & 15, g = lane >> 4;
      // ---- o, rounded; transposed by unit matrices (as left operand, so that a lane gets a token's neighbouring columns)
      const b16x8 part_of[2] = {unit(lane, 0), unit(lane, 1)};
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          u[i] = pack_bf16(O[2 * pair][2 * i], O[2 * pair][2 * i + 1]);
          u[2 + i] = pack_bf16(O[2 * pair + 1][2 * i], O[2 * pair + 1][2 * i + 1]);
        }
        if (__ballot(not_finite(u) != 0)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int t = 32 * pair + 8 * g + i;
            if (t < count && strip * 16 + n < a.d_v)
              ((uint16_t*)a.o)[(token0 + t) * a.o_token_stride + head * a.o_head_stride + strip * 16 + n] = (uint16_t)(u[i / 2] >> (i % 2 * 16));
          }
          continue;
        }
        const int own = strip * 16 + 4 * g;  // this lane's columns: own .. own + 3
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const f32x4 w = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, u), part_of[half], f32x4{0, 0, 0, 0}, 0, 0, 0);
          const int t = 32 * pair + 16 * half;  // + n: this lane's token
          const char* const q = o_rows.at + t * o_rows.step;
          const unsigned at = (unsigned)(n * o_rows.step + own * 2);
          if (t + n < count) {
            if (VEC) {
              if (own < a.d_v) *lane_at<u32x2>(q, at) = u32x2{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])};
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (own + i < a.d_v) *lane_at<uint16_t>(q + i * 2, at) = (uint16_t)pack_bf16(w[i], 0.0f);
            }
          }
        }
      }
    }
    k_rows.next(1);
    q_rows.next(1);
    v_rows.next(1);
    o_rows.next(1);
    meet();
  }
  float* const out = TRANS ? trans : at >= 0 && a.state_out && last ? a.state_out + at : nullptr;
  if (out && works) {
    const int lane = own_lane(), col = strip * 16 + (lane & 15), g = lane >> 4, width = TRANS ? ld : a.d_v;
    EVK_GLOBAL float* const to = (EVK_GLOBAL float*)uniform(out);
    if (TRANS || col < a.d_v)
#pragma unroll
      for (int b = 0; b < 2 * STEPS; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = place(b, 4 * g + i);
          if (row < a.d_k) to[row * width + col] = S[b][i];
        }
  }
}

// The states that the segments start from: N_j becomes M_j (the start of segment j) + N_j, for one segment after the other.  A
// workgroup has 16 columns of one head, its waves DKP / 64 blocks of 16 rows each; fp32 matrix instructions, the next M on its way.
template <int DKP>
__global__ __launch_bounds__(256) void delta_join(DeltaParams p) {
  constexpr int BLOCKS = DKP / 64, DEEP = DKP / 16;
  __shared__ float s_state[DKP][17];
  const evconv_delta_args& a = p.a;
  const int strips_v = (a.d_v + 15) / 16, ld = (strips_v + (a.d_k + 15) / 16) * 16;
  const int strip = blockIdx.x % strips_v;
  const int64_t pair = blockIdx.x / strips_v;
  const Span span = span_of(p, (int)(pair / a.heads_v));
  const int segs = (span.len + p.seg_chunks * C - 1) / (p.seg_chunks * C);
  if (span.len <= p.short_len || segs < 3) return;  // (N of the first segment is the second one's start)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4, col = strip * 16 + m;
  auto segment = [&](int j) { return p.trans + (pair * p.segs + j) * a.d_k * (int64_t)ld; };
  f32x4 S[BLOCKS], N[BLOCKS], M[BLOCKS][DEEP];
  auto request = [&](int j) __attribute__((always_inline)) {
    const float* const q = segment(j);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int row0 = (wave * BLOCKS + b) * 16;
#pragma unroll
      for (int d = 0; d < DEEP; ++d)  // columns 16 d + 4 g .. + 3 of row m (behind d_k they are zero up to whole 16)
        M[b][d] = row0 + m < a.d_k && 16 * d < a.d_k ? *(const f32x4*)(q + (row0 + m) * ld + strips_v * 16 + 16 * d + 4 * g) : f32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) N[b][i] = row0 + 4 * g + i < a.d_k ? q[(row0 + 4 * g + i) * ld + col] : 0.0f;
    }
  };
  {
    const float* const q = segment(0);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = (wave * BLOCKS + b) * 16 + 4 * g + i;
        S[b][i] = row < a.d_k ? q[row * ld + col] : 0.0f;
      }
  }
  request(1);
  for (int j = 1; j < segs - 1; ++j) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_state[(wave * BLOCKS + b) * 16 + 4 * g + i][m] = S[b][i];
    __syncthreads();
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) S[b] = N[b];
#pragma unroll
    for (int d = 0; d < DEEP; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = s_state[16 * d + 4 * g + e][m];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) S[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(M[b][d][e], x, S[b], 0, 0, 0);
      }
    __syncthreads();
    if (j + 1 < segs - 1) request(j + 1);
    float* const q = segment(j);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = (wave * BLOCKS + b) * 16 + 4 * g + i;
        if (row < a.d_k) q[row * ld + col] = S[b][i];
      }
  }
}

// Consumer waves of a workgroup.
int delta_fused_waves(const DeltaParams& p) { return p.vec && p.vec_v && p.a.d_v <= 64 ? 4 : 8; }
template <int DKP, int NC, bool VEC, bool TRANS>
void start_pass(const DeltaParams& p, hipStream_t s) {
  typedef FusedShape<DKP, NC> F;
  const int strips = (p.a.d_v + 15) / 16 + (TRANS ? (p.a.d_k + 15) / 16 : 0), parts = (strips + NC - 1) / NC;
  const int64_t grid = (int64_t)p.a.n_seq * p.a.heads_v * (TRANS ? p.segs - 1 : p.segs) * parts;
  delta_fused<DKP, NC, VEC, TRANS><<<(unsigned)grid, F::kThreads, F::kBytes, s>>>(p);
}
template <int DKP, int NC, bool VEC>
void start(const DeltaParams& p, hipStream_t s) {
  if (p.segs > 1) {
    start_pass<DKP, NC, VEC, true>(p, s);
    launch_delta_join(p, s);
  }
  start_pass<DKP, NC, VEC, false>(p, s);
}
template <int DKP>
void start_keys(const DeltaParams& p, hipStream_t s) {
  if (!p.vec || !p.vec_v) start<DKP, 8, false>(p, s);
  else if (delta_fused_waves(p) == 8) start<DKP, 8, true>(p, s);
  else start<DKP, 4, true>(p, s);
}
}  // namespace

bool delta_fused_supported(const DeltaParams& p) {
  // (a lane's bytes into a chunk are 32 bits)
  auto near = [](int64_t stride) { return stride >= 0 && stride <= 1 << 23; };
  return p.a.dtype == EVCONV_BF16 && p.a.d_k <= 128 && near(p.a.q.token_stride) && near(p.a.k.token_stride) &&
         near(p.a.v.token_stride) && near(p.a.o_token_stride) && near(p.a.gate.token_stride) && near(p.a.beta.token_stride);
}

int64_t delta_fused_threads(const DeltaParams& p) {
  const int waves = delta_fused_waves(p), strips = (p.a.d_v + 15) / 16 + (p.segs > 1 ? (p.a.d_k + 15) / 16 : 0);  // (with the first pass' strips of keys)
  return (int64_t)p.a.n_seq * p.a.heads_v * p.segs * ((strips + waves - 1) / waves) * (waves + 4) * 64;
}

// A workgroup of the unsplit launch per head and eight (four) strips; where they leave most of the chip idle and sequences are
// long, segments, as many as give every compute unit one, of four chunks at least.  Three segments cost what they save: every
// chunk is worked on twice, the first time with twice the columns.  us, whole and in segments, heads of 128 x 128 / 64 x 64:
//                                    bf16                              fp32
//   1 sequence of 4 heads,   800       107, 90 / 69, 56                  137, 125 / 85, 72
//                           1024       130, 90 / 83, 56                  161, 127 / 99, 74
//                           4096       483, 135 / 303, 70                533, 169 / 331, 91
//   1 sequence of 32 heads, 2048       257, 155 / 158, 89                364, 269 / 207, 118
//                          32768      4040, 1399 / 2444, 818            5862, 2961 / 3611, 1457
//   2 sequences of 32 heads, 8192     1025, 714 / 604, 421              1760, 1512 / 1081, 764
//   3 (three segments)                1031, 1287 / 622, 775             2034, 2521 / 1225, 1271
//   4 (two)                           1033, 1004 / 625, 571             2306, 2426 / 1375, 1388
size_t plan_delta_segments(DeltaParams& p, bool fused) {
  const int waves = fused ? delta_fused_waves(p) : 8, strips_v = (p.a.d_v + 15) / 16, parts = (strips_v + waves - 1) / waves;
  const int64_t pairs = (int64_t)p.a.n_seq * p.a.heads_v, groups = pairs * parts;
  const int64_t most = p.len >= 0 ? (p.len + C - 1) / C : p.a.n_tokens / C + 1;                          // chunks of a sequence
  const int64_t sum = p.len >= 0 ? most * p.a.n_seq : p.a.n_tokens / C + p.a.n_seq;                      // of all
  p.segs = 1;
  p.seg_chunks = (int)most;
  if ((!fused && (p.a.dtype != EVCONV_F32 || p.a.d_k > 128)) || groups >= 128 || sum / p.a.n_seq < 12) return 0;
  const int64_t chunks = std::max<int64_t>(4, (sum * p.a.heads_v * parts + 255) / 256), segs = (most + chunks - 1) / chunks;
  const int64_t state = (int64_t)p.a.d_k * (strips_v + (p.a.d_k + 15) / 16) * 16 * 4, start = (int64_t)p.a.d_k * strips_v * 16 * 4;
  const int64_t bytes = pairs * (segs * state + start);
  if (segs < 4 || bytes > 2ll << 30 || pairs * segs * parts * 8 >= 1ll << 31) return 0;
  p.segs = (int)segs;
  p.seg_chunks = (int)chunks;
  return (size_t)bytes;
}
void place_delta_segments(DeltaParams& p, char* workspace) {
  const int strips_v = (p.a.d_v + 15) / 16;
  p.trans = (float*)workspace;
  p.start0 = p.trans + (int64_t)p.a.n_seq * p.a.heads_v * p.segs * p.a.d_k * (strips_v + (p.a.d_k + 15) / 16) * 16;
}

void launch_delta_join(const DeltaParams& p, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)p.a.n_seq * p.a.heads_v * ((p.a.d_v + 15) / 16));
  if (p.dkp <= 64) delta_join<64><<<grid, 256, 0, s>>>(p);
  else delta_join<128><<<grid, 256, 0, s>>>(p);
}
void launch_delta_fused(const DeltaParams& p, hipStream_t s) {
  if (p.dkp == 64) start_keys<64>(p, s);
  else start_keys<128>(p, s);
}

}  // namespace evk
