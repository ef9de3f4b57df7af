// Device code that the kernels of the gated delta rule share (kernels_delta.hip, kernels_delta_fused.hip).
#pragma once

#include "ops_device.h"
#include "ops_kernels.h"

namespace evk {
namespace {

constexpr int C = kDeltaChunk;
constexpr int kFrag = 1024;            // bytes of one matrix-core operand: 64 lanes x 8 bf16
constexpr int kTri = 6;                // 16 x 32 blocks of a 64 x 64 matrix that a lower triangle reaches
constexpr float kLeastLog = -1e5f;     // log decays are not below: e^x is 0, and differences of sums stay finite
constexpr float kBf16Overflow = 3.3961775e38f;  // the smallest value that rounds to an infinite bf16

__host__ __device__ constexpr int parts_in(bool f32) { return f32 ? 3 : 1; }    // of keys and queries
__host__ __device__ constexpr int parts_out(bool f32) { return f32 ? 3 : 2; }   // of what reaches o only

struct Span { int first, len; };
__device__ __forceinline__ Span span_of(const DeltaParams& p, int seq) {
  if (p.len >= 0) return {seq * p.len, p.len};
  const int n = (int)p.a.n_tokens;
  const int a = min(max(p.a.seq_offsets[seq], 0), n), b = min(max(p.a.seq_offsets[seq + 1], 0), n);
  return {a, max(b - a, 0)};
}
// First chunk slot of a long sequence (one in chunks): no two sequences' slots meet, and none is behind slots_total (plan_delta).  Of
// lengths of their own, behind s.first / C and one for every long sequence that can stand before this one: at most seq, and at most
// s.first / (kDeltaShortRagged + 1).  (From one long sequence to the next the first grows by len / C and the second by one at least.)
__device__ __forceinline__ int first_slot(const DeltaParams& p, const Span& s, int seq) {
  return p.len >= 0 ? seq * ((p.len + C - 1) / C) : s.first / C + min(seq, s.first / (kDeltaShortRagged + 1));
}

// Offset of a sequence's state, or -1: it has none.
__device__ __forceinline__ int64_t state_at(const DeltaParams& p, int seq, int head) {
  const int slot = p.a.slots ? p.a.slots[seq] : seq;
  if (slot < 0 || slot >= p.a.n_slots) return -1;
  return ((int64_t)slot * p.a.heads_v + head) * p.a.d_k * p.a.d_v;
}

struct Gates { float g, beta; };
// from what is in memory
__device__ __forceinline__ Gates gates_from(bool raw, float gate, float beta, float a_scale, float dt_bias) {
  Gates r = {gate, beta};
  if (raw) {
    const float x = gate + dt_bias;
    r.g = -a_scale * (x > 20.0f ? x : log1pf(expf(x)));
    r.beta = 1.0f / (1.0f + expf(-beta));
  }
  if (r.g < kLeastLog) r.g = kLeastLog;
  return r;
}
__device__ __forceinline__ Gates gates_of(const DeltaParams& p, int64_t token, int head) {
  const bool bf16 = p.a.gate_dtype == EVCONV_BF16, raw = p.a.flags & EVCONV_DELTA_RAW_GATES;
  return gates_from(raw, load_any(p.a.gate.data, token * p.a.gate.token_stride + head * p.a.gate.head_stride, bf16),
                    load_any(p.a.beta.data, token * p.a.beta.token_stride + head * p.a.beta.head_stride, bf16),
                    raw ? p.a.a_scale[head] : 0.0f, raw ? p.a.dt_bias[head] : 0.0f);
}

// What a row is divided by, from its sum of squares; NaN beyond fp32: the division would make it zeros.
__device__ __forceinline__ float norm_of(float squares) { return squares < INFINITY ? sqrtf(squares + 1e-6f) : NAN; }

// Operands of the 16 x 16 x 32 matrix instruction: a lane (m = lane % 16, g = lane / 16) holds row m of the left
// operand (column m of the right one) at the contraction's places 8 g .. 8 g + 7, and column m, rows
// 4 g .. 4 g + 3 of the result.  Let block b of a result's rows hold, at its row 4 g + i, the row
//   place(b, 4 g + i) = 32 (b / 2) + 8 g + 4 (b % 2) + i.
// Then the eight values that a lane has of blocks 2 s and 2 s + 1 are the ones that it needs as right operand
// at step s of a contraction over those rows: S, R and D go from result to operand without leaving
// their lane.  K, Q, K', T and P are laid out for that by delta_prepare.
__host__ __device__ __forceinline__ int place(int block, int m) { return 32 * (block >> 1) + 8 * (m >> 2) + 4 * (block & 1) + (m & 3); }
// Index of T's (P's) 16 x 32 block of result block b and contraction step s.
__device__ __forceinline__ constexpr int tri(int b, int s) { return b < 2 ? b : 2 + (b - 2) * 2 + s; }

// Bits of this lane's 16 values that are not finite, or that a bf16 rounds to infinity
__device__ __forceinline__ unsigned bad_values(const f32x4 (&x)[4]) {
  unsigned bad = 0;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!(fabsf(x[b][i]) < kBf16Overflow)) bad |= 1u << (b * 4 + i);
  return bad;
}
// A value that is not finite would reach earlier tokens through the zeros of T and P: what follows a column's first such
// token (which: bits of this lane's 16 values that are not) is left out of the products, and made NaN behind them.
__device__ __forceinline__ void cut_columns(f32x4 (&x)[4], unsigned which, int& first_bad, int g) {
  int first = first_bad;
#pragma unroll
  for (int b = 3; b >= 0; --b)
#pragma unroll
    for (int i = 3; i >= 0; --i)
      if (which >> (b * 4 + i) & 1) first = min(first, place(b, 4 * g) + i);
  first = min(first, __shfl_xor(first, 16));
  first = min(first, __shfl_xor(first, 32));
  first_bad = first;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (place(b, 4 * g) + i >= first) x[b][i] = 0.0f;
}

}  // namespace
}  // namespace evk
