// The gated delta rule (evconv_delta_rule) on gfx950.
//
// With S a d_k x d_v matrix per sequence and value head, a token does
//   S = e^g S;  d = beta (v - S'k);  S += k d';  o = scale S'q.
// The columns of S never meet, so a wave owns a strip of columns for a whole sequence.
//
// Few tokens (delta_step): token by token, the strip in registers.
//
// Long sequences: 64 tokens (a chunk) at a time.  With G_i the sum of g up to token i of the chunk, S the state
// before it, and the rows d_i of D unknown, the recurrence says
//   d_i = beta_i (v_i - e^{G_i} S'k_i - sum_{j<i} e^{G_i-G_j} (k_i k_j) d_j)
// so (I + A) D = R with A_ij = beta_i e^{G_i-G_j} k_i k_j below the diagonal and R_i = beta_i (v_i - e^{G_i} S'k_i):
//   D = T R, T = (I + A)^-1;  O = scale (e^G Q S + P D), P_ij = e^{G_i-G_j} q_i k_j for j <= i;
//   S_next = e^{G_63} S + sum_j k_j (e^{G_63-G_j} d_j)'.
// T and P do not depend on S: delta_prepare computes them for all chunks at once; delta_chain goes
// through a sequence's chunks with what is left, products with S, D and R.
//
// Precision: the state is fp32.  bf16 keys and queries enter products as they are (their norms are factors of
// rows, applied to the sums), everything else that reaches the state as three bf16 parts, which hold
// 24 bits; outputs of bf16 calls are summed from two parts.  G is summed in 64 bits: the difference of two
// sums over a chunk would lose the bits that its exponential needs.
#include <algorithm>
#include <type_traits>

#include "delta_device.h"

namespace evk {
namespace {

// ---- token by token -------------------------------------------------------------------------------
// A wave: one sequence, one head, 32 columns; 8 lanes x 4 columns across, 8 groups of ROWS rows down.
// o needs S'q after the update, which is e^g (S'q before it) + (k q) d: one pass over the strip gives both
// products, one reduction over the groups sums them.
// Bound by the state's bytes, read once and written once: 256 sequences of 16 heads of 128 x 128 (537 MB) in
// 104 us, the 5.2 TB/s of a large copy.
// ONE: every sequence has one token; otherwise the next token is on its way while one is applied.
template <bool BF16, int ROWS, bool VEC, bool ONE>
__global__ __launch_bounds__(256) void delta_step(DeltaParams p) {
  const evconv_delta_args& a = p.a;
  const int lane = threadIdx.x & 63;
  const int blocks = (a.d_v + 31) / 32;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int block = (int)(wave % blocks);
  const int head = (int)(wave / blocks % a.heads_v);
  const int64_t seq64 = wave / blocks / a.heads_v;
  if (seq64 >= a.n_seq) return;
  const int seq = (int)seq64;
  const Span s = span_of(p, seq);
  if (s.len > p.short_len) {  // (delta_prepare's: its chunk slots are told whose they are)
    if (p.slot_seq && head == 0 && block == 0)
      for (int i = lane, slot0 = first_slot(p, s, seq); i < (s.len + C - 1) / C; i += 64) p.slot_seq[slot0 + i] = seq;
    return;
  }
  const int64_t at = state_at(p, seq, head);
  const int row0 = (lane >> 3) * ROWS, col = block * 32 + (lane & 7) * 4;
  f32x4 S[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    S[i] = f32x4{0, 0, 0, 0};
    if (at >= 0 && a.state_in && row0 + i < a.d_k) {
      const float* q = a.state_in + at + (int64_t)(row0 + i) * a.d_v + col;
      if (VEC) {
        if (col < a.d_v) S[i] = *(const f32x4*)q;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < a.d_v) S[i][j] = q[j];
      }
    }
  }
  const int hk = head / p.share;
  struct Token {
    float k[ROWS], q[ROWS], v[4], gate, beta;
  };
  const bool raw = a.flags & EVCONV_DELTA_RAW_GATES, gate_bf16 = a.gate_dtype == EVCONV_BF16;
  const float a_scale = raw ? a.a_scale[head] : 0.0f, dt_bias = raw ? a.dt_bias[head] : 0.0f;
  auto load = [&](int t, Token& x) __attribute__((always_inline)) {
    const int64_t token = s.first + t;
    load_run<BF16, ROWS, VEC>(a.k.data, token * a.k.token_stride + hk * a.k.head_stride + row0, a.d_k - row0, x.k);
    load_run<BF16, ROWS, VEC>(a.q.data, token * a.q.token_stride + hk * a.q.head_stride + row0, a.d_k - row0, x.q);
    load_run<BF16, 4, false>(a.v.data, token * a.v.token_stride + head * a.v.head_stride + col, a.d_v - col, x.v);
    x.gate = load_any(a.gate.data, token * a.gate.token_stride + head * a.gate.head_stride, gate_bf16);
    x.beta = load_any(a.beta.data, token * a.beta.token_stride + head * a.beta.head_stride, gate_bf16);
  };
  Token next;
  if (s.len > 0) load(0, next);
  for (int t = 0; t < (ONE ? min(s.len, 1) : s.len); ++t) {
    const int64_t token = s.first + t;
    const Token now = next;
    if (!ONE && t + 1 < s.len) load(t + 1, next);
    const float(&k)[ROWS] = now.k, (&q)[ROWS] = now.q, (&v)[4] = now.v;
    const Gates gate = gates_from(raw, now.gate, now.beta, a_scale, dt_bias);
    const float decay = expf(gate.g);
    float sum[11];  // S'k, S'q (four columns each), kq, kk, qq
#pragma unroll
    for (int j = 0; j < 11; ++j) sum[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[j] = fmaf(S[i][j], k[i], sum[j]);
        sum[4 + j] = fmaf(S[i][j], q[i], sum[4 + j]);
      }
      sum[8] = fmaf(k[i], q[i], sum[8]);
      sum[9] = fmaf(k[i], k[i], sum[9]);
      sum[10] = fmaf(q[i], q[i], sum[10]);
    }
#pragma unroll
    for (int d = 8; d < 64; d *= 2)
#pragma unroll
      for (int j = 0; j < 11; ++j) sum[j] += __shfl_xor(sum[j], d);
    float rk = 1.0f, rq = a.scale;
    if (a.flags & EVCONV_DELTA_NORMALIZE) {
      rk = 1.0f / norm_of(sum[9]);
      rq = a.scale / norm_of(sum[10]);
    }
    float out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float d = gate.beta * (v[j] - decay * (rk * sum[j]));
      const float dk = rk * d;
      out[j] = rq * (decay * sum[4 + j] + sum[8] * dk);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) S[i][j] = fmaf(k[i], dk, decay * S[i][j]);
    }
    if (lane < 8) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < a.d_v) store_one<BF16>(a.o, token * a.o_token_stride + head * a.o_head_stride + col + j, out[j]);
    }
  }
  if (at >= 0 && a.state_out) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (row0 + i < a.d_k) {
        float* q = a.state_out + at + (int64_t)(row0 + i) * a.d_v + col;
        if (VEC) {
          if (col < a.d_v) *(f32x4*)q = S[i];
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (col + j < a.d_v) q[j] = S[i][j];
        }
      }
  }
}

// ---- chunks: what does not depend on the state ------------------------------------------------------
// Eight values of a token's row from column c on, as bf16 parts
template <bool F32, bool VEC>
__device__ __forceinline__ void load_parts(const evconv_heads& h, int head, int d, int64_t token, bool live, int c, b16x8 (&out)[parts_in(F32)]) {
  float v[8];
  load_run<!F32, 8, VEC>(h.data, token * h.token_stride + head * h.head_stride + c, live ? d - c : 0, v);
  split8(v, out);
}

template <bool F32, bool VEC>
__global__ __launch_bounds__(256, 3) void delta_prepare(DeltaParams p) {
  constexpr int PI = parts_in(F32), PO = parts_out(F32);
  const evconv_delta_args& a = p.a;
  __shared__ float s_a[C][C + 1], s_t[C][C + 1];  // (P takes A's place)
  __shared__ double s_g[C];
  __shared__ float s_beta[C], s_rk[C], s_rq[C];
  __shared__ int s_bad;  // first token whose row of A is not finite
  const int slot = blockIdx.x / a.heads_v, head = blockIdx.x % a.heads_v, hk = head / p.share;
  // Whose slot it is: delta_step has written that down for every chunk of the long sequences.  What stands there of a slot that is
  // nobody's may be anything, and is taken only where it is the truth.
  const int seq = p.len >= 0 ? slot / ((p.len + C - 1) / C) : p.slot_seq[slot];
  if ((unsigned)seq >= (unsigned)a.n_seq) return;
  const Span span = span_of(p, seq);
  const int chunk = slot - first_slot(p, span, seq);
  if (span.len <= p.short_len || chunk < 0 || chunk * C >= span.len) return;
  const int64_t token0 = span.first + chunk * C;
  const int count = min(span.len - chunk * C, C);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, g = lane >> 4;

  // ---- gates and norms of the tokens
  if (wave == 0) {
    Gates gate = {0.0f, 0.0f};
    if (lane < count) gate = gates_of(p, token0 + lane, head);
    double sum = gate.g;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    s_g[lane] = sum;
    s_beta[lane] = gate.beta;
  }
  for (int i = tid; i < C * C; i += 256) s_t[i / C][i % C] = 0.0f;
  if (tid == 0) s_bad = C;

  // ---- K K' and Q K', a wave 16 tokens' rows of them, and the diagonal of Q Q'
  f32x4 kk[4], qk[4], qq = {0, 0, 0, 0};
#pragma unroll
  for (int b = 0; b < 4; ++b) kk[b] = qk[b] = f32x4{0, 0, 0, 0};
  {
    const int row = wave * 16 + m;
    for (int c = 0; c < p.dkp; c += 32) {
      // (all rows of a step on their way before the first is used)
      float k[4][8], q[8];
      auto load = [&](const evconv_heads& h, int t, bool live, float (&v)[8]) __attribute__((always_inline)) {
        load_run<!F32, 8, VEC>(h.data, (token0 + t) * h.token_stride + hk * h.head_stride + c + 8 * g, live && t < count ? a.d_k - c - 8 * g : 0, v);
      };
      load(a.q, row, true, q);
#pragma unroll
      for (int b = 0; b < 4; ++b) load(a.k, b * 16 + m, b <= wave, k[b]);
      __builtin_amdgcn_sched_barrier(0);
      float own[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) own[j] = wave & 2 ? (wave & 1 ? k[3][j] : k[2][j]) : (wave & 1 ? k[1][j] : k[0][j]);
      b16x8 ka[PI], qa[PI], kb[PI];
      split8(own, ka);
      split8(q, qa);
      mfma_parts<2>(qq, qa, qa);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b > wave) break;
        split8(k[b], kb);
        mfma_parts<2>(kk[b], ka, kb);
        mfma_parts<2>(qk[b], qa, kb);
      }
    }
    // norms: the diagonals, which lanes with m / 4 == g hold
    f32x4 own = kk[0];
#pragma unroll
    for (int b = 1; b < 4; ++b)
      if (b == wave) own = kk[b];
    const float u = m & 2 ? (m & 1 ? own[3] : own[2]) : (m & 1 ? own[1] : own[0]);
    const float v = m & 2 ? (m & 1 ? qq[3] : qq[2]) : (m & 1 ? qq[1] : qq[0]);
    if (m >> 2 == g) {
      const bool normalize = a.flags & EVCONV_DELTA_NORMALIZE;
      s_rk[row] = normalize ? 1.0f / norm_of(u) : 1.0f;
      s_rq[row] = normalize ? a.scale / norm_of(v) : a.scale;
    }
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = wave * 16 + 4 * g + i, col = b * 16 + m;
      float x = 0.0f, y = 0.0f;
      if (col <= row) {  // (selected, not multiplied: what is above the diagonal may be anything)
        const float e = expf((float)(s_g[row] - s_g[col])) * s_rk[col];
        if (col < row) x = s_beta[row] * s_rk[row] * e * kk[b][i];
        y = s_rq[row] * e * qk[b][i];
      }
      s_a[row][col] = x;
      qk[b][i] = y;
      if (!(fabsf(x) < INFINITY)) atomicMin(&s_bad, row);
    }
  __syncthreads();
  // Rows from a bad one on are NaN by their beta (below); in T they would reach rows above them through its zeros.
  const int bad = s_bad;
  if (bad < C) {
    for (int i = tid; i < (C - bad) * C; i += 256) s_a[bad + i / C][i % C] = 0.0f;
    __syncthreads();
  }

  // ---- T = (I + A)^-1: the 16 x 16 blocks on the diagonal by substitution, a column to a lane; then blocks of
  // twice the size, whose lower half is -T22 A21 T11 (fp32 matrix instructions; stable where a series in
  // powers of A is not: keys of neighbouring windows are alike)
  if (lane < 16) {
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float sum = i == lane ? 1.0f : 0.0f;
#pragma unroll
      for (int l = 0; l < i; ++l) sum = fmaf(-s_a[wave * 16 + i][wave * 16 + l], l < lane ? 0.0f : x[l], sum);
      x[i] = i < lane ? 0.0f : sum;
      s_t[wave * 16 + i][wave * 16 + lane] = x[i];
    }
  }
  __syncthreads();
  // a 16 x 16 block of X Y, n blocks of 16 deep
  auto product = [&](const float (*x)[C + 1], int xr, int xc, const float (*y)[C + 1], int yr, int yc, int n) {
    f32x4 acc = {0, 0, 0, 0};
    for (int c = 0; c < n * 16; c += 4) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[xr + m][xc + c + g], y[yr + c + g][yc + m], acc, 0, 0, 0);
    return acc;
  };
#pragma unroll
  for (int size = 1; size <= 2; ++size) {  // in blocks of 16
    // block (r, c) of this wave: below the diagonal blocks of `size`
    const bool mine = size == 2 || wave < 2;
    const int r = size == 1 ? 2 * wave + 1 : 2 + (wave >> 1), c = size == 1 ? 2 * wave : wave & 1;
    const int base = size == 1 ? 2 * wave : 0;  // first block of the pair
    f32x4 acc;
    if (mine) acc = product(s_a, r * 16, base * 16, s_t, base * 16, c * 16, size);
    __syncthreads();
    // A21 T11 takes A21's place
    if (mine)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_a[r * 16 + 4 * g + i][c * 16 + m] = acc[i];
    __syncthreads();
    if (mine) {
      acc = product(s_t, r * 16, (base + size) * 16, s_a, (base + size) * 16, c * 16, size);
#pragma unroll
      for (int i = 0; i < 4; ++i) s_t[r * 16 + 4 * g + i][c * 16 + m] = -acc[i];
    }
    __syncthreads();
  }

#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_a[wave * 16 + 4 * g + i][b * 16 + m] = qk[b][i];
  __syncthreads();

  // ---- T and P as left operands, the factors of the rows
  char* const at_t = p.frag_t + (size_t)blockIdx.x * (kTri * kFrag * (3 + PO));
  for (int f = wave; f < 2 * kTri; f += 4) {
    const bool is_p = f >= kTri;
    const int i = is_p ? f - kTri : f, b = i < 2 ? i : 2 + (i - 2) / 2, s = i < 2 ? 0 : (i - 2) % 2;
    const int row = place(b, m), col = 32 * s + 8 * g;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = is_p ? s_a[row][col + j] : col + j <= row ? s_t[row][col + j] : 0.0f;
    b16x8 out[3];
    split8(v, out);
    const int n = is_p ? PO : 3;
    char* q = at_t + (is_p ? kTri * 3 : 0) * kFrag + i * n * kFrag + lane * 16;
#pragma unroll
    for (int part = 0; part < 3; ++part)
      if (part < n) *(b16x8*)(q + part * kFrag) = out[part];
  }
  if (tid < C) {
    float* q = p.scal + (size_t)blockIdx.x * kDeltaScalars;
    const double last = s_g[C - 1];
    q[tid] = tid < bad ? s_beta[tid] : NAN;
    q[C + tid] = s_beta[tid] * s_rk[tid] * expf((float)s_g[tid]);
    q[2 * C + tid] = s_rq[tid] * expf((float)s_g[tid]);
    q[3 * C + tid] = s_rk[tid] * expf((float)(last - s_g[tid]));
    if (tid == 0) q[4 * C] = expf((float)last);
  }
  // ---- K, Q and K' as left operands: once per key head, a part by each of its value heads
  {
    const int first = wave + 4 * (head % p.share), stride = 4 * p.share;
    const int steps = p.dkp / 32;
    const size_t one = (size_t)4 * steps * PI * kFrag;  // of K; the same of Q and K'
    char* const at_k = p.frag_k + ((size_t)slot * a.heads_k + hk) * 3 * one;
    for (int i = first; i < 4 * steps; i += stride) {  // (of K and of Q)
      const int b = i / steps, s = i % steps, row = place(b, m);
      b16x8 out[2][PI];
      load_parts<F32, VEC>(a.k, hk, a.d_k, token0 + row, row < count, 32 * s + 8 * g, out[0]);
      load_parts<F32, VEC>(a.q, hk, a.d_k, token0 + row, row < count, 32 * s + 8 * g, out[1]);
#pragma unroll
      for (int of = 0; of < 2; ++of)
#pragma unroll
        for (int part = 0; part < PI; ++part) *(b16x8*)(at_k + of * one + (size_t)(i * PI + part) * kFrag + lane * 16) = out[of][part];
    }
    for (int f = first; f < 4 * steps; f += stride) {
      const int b = f / 2, s = f % 2, row = place(b, m);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = 32 * s + 8 * g + j;
        v[j] = t < count && row < a.d_k ? load_one<!F32>(a.k.data, (token0 + t) * a.k.token_stride + hk * a.k.head_stride + row) : 0.0f;
      }
      b16x8 out[PI];
      split8(v, out);
#pragma unroll
      for (int part = 0; part < PI; ++part) *(b16x8*)(at_k + 2 * one + (size_t)(f * PI + part) * kFrag + lane * 16) = out[part];
    }
  }
}

// ---- chunks: through a sequence ----------------------------------------------------------------------
// A workgroup: one sequence, one value head, up to eight (four) strips of 16 columns of the state, a wave each, which stay in its
// registers.  The waves share the operands: a chunk's are K, Q, (T, P) and K' in turn, each brought into one of three
// buffers in LDS two stages before it is used (K, Q and K' in halves where they are larger than a buffer).
// Bound by a sequence's longest chain: fp32 operands are three parts, so a product is six matrix instructions, and what comes
// out of one has to be split again for the next; a wave alone on its SIMD reads operands, waits, splits and multiplies in a row.
// 24 sequences of up to 700 tokens, 6 heads of 80 x 112, fp32: 83 us, 7.6 a chunk, beside 28 for delta_prepare.  (Of 18.6 thousand cycles a chunk with v's and o's single values in a row and masks for each, K S
// took 5.2, Q S 2.8, T and P 5.3, K' 4.8: 96 us.)  Before: keys as 128 channels instead of 96 124, every wave with
// operands of its own from L2 222.
template <bool F32, int DKP>
struct ChainShape {
  static constexpr int PI = parts_in(F32), PO = parts_out(F32), STEPS = DKP / 32;
  static constexpr int kRows = 4 * STEPS * PI * kFrag;            // bytes of K; Q and K' alike
  static constexpr int kHalves = kRows > 48 * 1024 ? 2 : 1;
  static constexpr int kTp = kTri * kFrag * (3 + PO);
  static constexpr int kBuffer = kRows / kHalves > kTp ? kRows / kHalves : kTp;
  static constexpr int kStages = 3 * kHalves + 1;                 // of a chunk
  static constexpr int kScalars = kDeltaScalars * 4;
  static constexpr int kBytes = 3 * kBuffer + 2 * kScalars;
  static_assert(kBytes <= 160 * 1024 && kScalars == 2 * kFrag, "LDS");
  // pieces of 1 KB of a stage
  static constexpr int pieces(int stage) { return (stage == 2 * kHalves ? kTp : kRows / kHalves) / kFrag; }
};

// Segments of a sequence side by side, TRANS: as delta_fused (kernels_delta_fused.hip).
template <bool F32, int DKP, bool TRANS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void delta_chain(DeltaParams p) {
  typedef ChainShape<F32, DKP> H;
  constexpr int kSize = F32 ? 4 : 2, PI = H::PI, PO = H::PO, STEPS = H::STEPS, ORD = F32 ? 2 : 1, HALVES = H::kHalves, BLOCKS = 4 / HALVES;
  extern __shared__ __align__(16) char s_mem[];
  const evconv_delta_args& a = p.a;
  const int strips_v = (a.d_v + 15) / 16, strips = strips_v + (TRANS ? (a.d_k + 15) / 16 : 0), groups = (strips + WAVES - 1) / WAVES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int strip = blockIdx.x % groups * WAVES + wave;
  const int segs = TRANS ? p.segs - 1 : p.segs, seg = blockIdx.x / groups % segs;
  const int64_t pair = blockIdx.x / groups / segs;
  const int seq = (int)(pair / a.heads_v), head = (int)(pair % a.heads_v), hk = head / p.share;
  Span span = span_of(p, seq);
  if (span.len <= p.short_len) return;
  const size_t slot0 = (size_t)first_slot(p, span, seq) + (size_t)seg * p.seg_chunks;
  {
    const int64_t skip = (int64_t)seg * p.seg_chunks * C;
    if (span.len <= skip + (TRANS ? p.seg_chunks * C : 0)) return;  // (TRANS: nothing behind it)
    if (TRANS && seg == 0 && (int)(blockIdx.x % groups) * WAVES >= strips_v) return;
    span.first += (int)skip;
    span.len -= (int)skip;
  }
  const bool last = span.len <= p.seg_chunks * C;
  span.len = min(span.len, p.seg_chunks * C);
  const int col = strip * 16 + n;
  const bool unit_columns = TRANS && strip >= strips_v;
  const bool works = strip < strips && !(unit_columns && seg == 0), in = col < a.d_v && !unit_columns;
  const int64_t at = state_at(p, seq, head);
  const int ld = (strips_v + (a.d_k + 15) / 16) * 16;  // floats between the rows of p.trans
  f32x4 S[2 * STEPS];
  {
    const float* from = a.state_in ? a.state_in + at : nullptr;
    int width = a.d_v;
    bool there = at >= 0 && a.state_in && in;
    if (TRANS) there &= seg == 0;
    else if (seg || !last) {
      from = seg ? p.trans + (pair * p.segs + seg - 1) * a.d_k * (int64_t)ld : p.start0 + pair * a.d_k * (int64_t)(strips_v * 16);
      width = seg ? ld : strips_v * 16;
      there = works;
    }
#pragma unroll
    for (int b = 0; b < 2 * STEPS; ++b) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = place(b, 4 * g + i);
        S[b][i] = there && row < a.d_k ? from[row * width + col] : unit_columns && row == col - strips_v * 16 ? 1.0f : 0.0f;
        if (TRANS && seg == 0 && works && row < a.d_k) p.start0[pair * a.d_k * (int64_t)(strips_v * 16) + row * strips_v * 16 + col] = S[b][i];
      }
      asm volatile("" : "+v"(S[b]));  // (waited for here, not in every turn of the loop)
    }
  }
  const int chunks = (span.len + C - 1) / C;
  // a chunk's operands in memory
  auto rows_at = [&](int chunk) { return p.frag_k + ((slot0 + chunk) * a.heads_k + hk) * (size_t)(3 * H::kRows); };
  auto tp_at = [&](int chunk) { return p.frag_t + ((slot0 + chunk) * a.heads_v + head) * (size_t)H::kTp; };
  auto copy = [&](const char* from, char* to) __attribute__((always_inline)) {  // 1 KB, straight into LDS
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + lane * 16), (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  };
  char* const s_scal = s_mem + 3 * H::kBuffer;
  // Stage `stage` of a chunk into buffer `buffer`
  auto request = [&](int chunk, int stage, int buffer) __attribute__((always_inline)) {
    if (chunk >= chunks || (TRANS && stage >= HALVES && stage < 2 * HALVES)) return;
    // stages: K (halves), Q (halves), T and P, K' (halves)
    const bool tp = stage == 2 * HALVES;
    const char* const from = tp ? tp_at(chunk) : rows_at(chunk) + (size_t)(stage < 2 * HALVES ? stage : stage - 1) * (H::kRows / HALVES);
    const int pieces = tp ? H::pieces(2 * HALVES) : H::pieces(0);
    char* const to = s_mem + buffer * H::kBuffer;
#pragma unroll 1
    for (int i = wave; i < pieces; i += WAVES) copy(from + (size_t)i * kFrag, to + i * kFrag);
    if (stage == 0 && wave < 2) copy((const char*)(p.scal + ((slot0 + chunk) * a.heads_v + head) * kDeltaScalars) + wave * kFrag, s_scal + (chunk & 1) * H::kScalars + wave * kFrag);
  };
  int buffer = 0;
  request(0, 0, 0);
  request(0, 1, 1);
  f32x4 R[4], O[4], D[4];
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0f;
  int first_bad = C;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const int64_t token0 = span.first + (int64_t)chunk * C;
    const int count = min(span.len - chunk * C, C);
    const float* const scal = (const float*)(s_scal + (chunk & 1) * H::kScalars);
    auto run = [&](auto number) __attribute__((always_inline)) {
      constexpr int stage = decltype(number)::value;
      // everything that this stage reads has arrived; the stage before it is done with its buffer
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      {
        constexpr int next = stage + 2;
        const int to = buffer >= 1 ? buffer - 1 : 2;  // (two further on, of three)
        if (next < H::kStages) request(chunk, next, to);
        else request(chunk + 1, next - H::kStages, to);
      }
      const char* const q = s_mem + buffer * H::kBuffer + lane * 16;
      buffer = buffer == 2 ? 0 : buffer + 1;
      if (!works) return;
      // What the next wait covers: the values a stage before they are needed, the outputs a stage after they are known.
      // (Whole chunks: a lane's place and distances that are the same for all, without a mask for every token; a few at a time
      // between the matrix instructions, which a row of such requests would hold up.)
      const bool whole = count == C && in;
      const int64_t lane_v = ((token0 + place(0, 4 * g)) * a.v.token_stride + head * a.v.head_stride + col) * kSize;
      const int64_t lane_o = ((token0 + place(0, 4 * g)) * a.o_token_stride + head * a.o_head_stride + col) * kSize;
      auto load_v = [&](int from, int to) __attribute__((always_inline)) {
        if (whole)
#pragma unroll
          for (int t = from; t < to; ++t) v[t] = load_one<!F32>((const char*)a.v.data + lane_v + place(t / 4, t % 4) * a.v.token_stride * kSize, 0);
      };
      auto store_o = [&](int from, int to) __attribute__((always_inline)) {
        if (whole)
#pragma unroll
          for (int t = from; t < to; ++t) store_one<!F32>((char*)a.o + lane_o + place(t / 4, t % 4) * a.o_token_stride * kSize, 0, O[t / 4][t % 4]);
      };
      if constexpr (stage == 0) {
        if (count < C) {
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int t = place(b, 4 * g) + i;
              v[b * 4 + i] = t < count && in ? load_one<!F32>(a.v.data, (token0 + t) * a.v.token_stride + head * a.v.head_stride + col) : 0.0f;
            }
        }
      }
      if constexpr (stage == 2 * HALVES + 1 && !TRANS) {
        if (count < C) {
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int t = place(b, 4 * g) + i;
              if (t < count && in) store_one<!F32>(a.o, (token0 + t) * a.o_token_stride + head * a.o_head_stride + col, O[b][i]);
            }
        }
      }
      auto frag = [&](int i) __attribute__((always_inline)) { return *(const b16x8*)(q + (size_t)i * kFrag); };
      if constexpr (TRANS && stage >= HALVES && stage < 2 * HALVES) {
      } else if constexpr (stage < 2 * HALVES) {  // K S, then Q S
        constexpr bool keys = stage < HALVES;
        constexpr int b0 = stage % HALVES * BLOCKS;
        f32x4 acc[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) acc[b] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          b16x8 k[BLOCKS][PI], Sp[3];
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int part = 0; part < PI; ++part) k[b][part] = frag((b * STEPS + s) * PI + part);
          if constexpr (stage == 0) load_v(16 * s / STEPS, 16 * (s + 1) / STEPS);
          __builtin_amdgcn_sched_barrier(0);
          float x[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = S[2 * s][i];
            x[4 + i] = S[2 * s + 1][i];
          }
          split8(x, Sp);
          if (keys) mfma_parts<2, BLOCKS>(acc, k, Sp);
          else mfma_parts<ORD, BLOCKS>(acc, k, Sp);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          if (keys) R[b0 + b] = acc[b];
          else O[b0 + b] = acc[b];
        }
      } else if constexpr (stage == 2 * HALVES) {
        // R = beta v - beta e^G K S;  e^G Q S;  D = T R;  O += P D
        unsigned bad = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int t0 = place(b, 4 * g);  // this lane's tokens: t0 .. t0 + 3
          const f32x4 beta = *(const f32x4*)(scal + t0), kf = *(const f32x4*)(scal + C + t0), qf = *(const f32x4*)(scal + 2 * C + t0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            R[b][i] = t0 + i < count ? beta[i] * v[b * 4 + i] - kf[i] * R[b][i] : 0.0f;
            if (!TRANS) O[b][i] *= qf[i];
            if (!(fabsf(R[b][i]) < kBf16Overflow)) bad |= 1u << (b * 4 + i);
          }
        }
        first_bad = C;
        if (__ballot(bad != 0)) cut_columns(R, bad, first_bad, g);
        b16x8 Rp[2][3];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = R[2 * s][i];
            x[4 + i] = R[2 * s + 1][i];
          }
          split8(x, Rp[s]);
        }
        bad = 0;
#pragma unroll
        for (int b = 0; b < 4; b += 2) {
          D[b] = D[b + 1] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < 1 + (b >> 1); ++s) {
            b16x8 t[2][3];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int part = 0; part < 3; ++part) t[i][part] = frag(tri(b + i, s) * 3 + part);
            mfma_parts<2, 2>(&D[b], t, Rp[s]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!(fabsf(D[b + i / 4][i % 4]) < kBf16Overflow)) bad |= 1u << (b * 4 + i);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (__ballot(bad != 0 || first_bad < C)) cut_columns(D, bad, first_bad, g);
        if constexpr (!TRANS) {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[i] = D[2 * s][i];
              x[4 + i] = D[2 * s + 1][i];
            }
            b16x8 Dp[PO];
            split8(x, Dp);
#pragma unroll
            for (int b = 2 * s; b < 4; b += 2) {
              b16x8 pp[2][PO];
#pragma unroll
              for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int part = 0; part < PO; ++part) pp[i][part] = frag(kTri * 3 + tri(b + i, s) * PO + part);
              mfma_parts<ORD, 2>(&O[b], pp, Dp);
            }
          }
          if (__ballot(first_bad < C))
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (place(b, 4 * g) + i >= first_bad) O[b][i] = NAN;
        }
        const float decay = scal[4 * C];
#pragma unroll
        for (int b = 0; b < 2 * STEPS; ++b) S[b] *= decay;
#pragma unroll
        for (int b = 0; b < 4; ++b) D[b] *= *(const f32x4*)(scal + 3 * C + place(b, 4 * g));  // w D from here on
      } else {  // S = e^G S + K' (w D)
        constexpr int b0 = (stage - 2 * HALVES - 1) * (2 * STEPS / HALVES), KT = 2 * STEPS / HALVES % 4 ? 2 : 4;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = D[2 * s][i];
            x[4 + i] = D[2 * s + 1][i];
          }
          b16x8 Dw[3];
          split8(x, Dw);
#pragma unroll
          for (int b = 0; b < 2 * STEPS / HALVES; b += KT) {
            b16x8 kt[KT][PI];
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
              for (int part = 0; part < PI; ++part) kt[i][part] = frag(((b + i) * 2 + s) * PI + part);
            if constexpr (stage == 2 * HALVES + 1 && !TRANS) {
              constexpr int kAll = 2 * (2 * STEPS / HALVES / KT);  // turns of these loops
              const int turn = s * (kAll / 2) + b / KT;
              store_o(16 * turn / kAll, 16 * (turn + 1) / kAll);
            }
            __builtin_amdgcn_sched_barrier(0);
            mfma_parts<2, KT>(&S[b0 + b], kt, Dw);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (stage == H::kStages - 1 && first_bad < C)
#pragma unroll
          for (int b = 0; b < 2 * STEPS; ++b) S[b] = f32x4{NAN, NAN, NAN, NAN};
      }
    };
    run(std::integral_constant<int, 0>());
    run(std::integral_constant<int, 1>());
    run(std::integral_constant<int, 2>());
    run(std::integral_constant<int, 3>());
    if constexpr (HALVES == 2) {
      run(std::integral_constant<int, 4>());
      run(std::integral_constant<int, 5>());
      run(std::integral_constant<int, 6>());
    }
  }
  float* const out = TRANS ? p.trans + (pair * p.segs + seg) * a.d_k * (int64_t)ld : at >= 0 && a.state_out && last ? a.state_out + at : nullptr;
  if (out && works && (TRANS || in))
#pragma unroll
    for (int b = 0; b < 2 * STEPS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = place(b, 4 * g + i);
        if (row < a.d_k) out[row * (TRANS ? ld : a.d_v) + col] = S[b][i];
      }
}

template <bool BF16, int ROWS>
void steps_rows(const DeltaParams& p, bool vec, unsigned grid, hipStream_t s) {
  if (p.len == 1) {
    if (vec) delta_step<BF16, ROWS, true, true><<<grid, 256, 0, s>>>(p);
    else delta_step<BF16, ROWS, false, true><<<grid, 256, 0, s>>>(p);
  } else {
    if (vec) delta_step<BF16, ROWS, true, false><<<grid, 256, 0, s>>>(p);
    else delta_step<BF16, ROWS, false, false><<<grid, 256, 0, s>>>(p);
  }
}
template <bool BF16>
void steps_type(const DeltaParams& p, bool vec, unsigned grid, hipStream_t s) {
  if (p.a.d_k <= 32) steps_rows<BF16, 4>(p, vec, grid, s);
  else if (p.a.d_k <= 64) steps_rows<BF16, 8>(p, vec, grid, s);
  else if (p.a.d_k <= 128) steps_rows<BF16, 16>(p, vec, grid, s);
  else steps_rows<BF16, 32>(p, vec, grid, s);
}
template <bool F32, int DKP, bool TRANS, int WAVES>
void chain_pass(const DeltaParams& p, hipStream_t s) {
  const int64_t pairs = (int64_t)p.a.n_seq * p.a.heads_v * (TRANS ? p.segs - 1 : p.segs);
  const int strips = (p.a.d_v + 15) / 16 + (TRANS ? (p.a.d_k + 15) / 16 : 0);
  delta_chain<F32, DKP, TRANS, WAVES><<<(unsigned)(pairs * ((strips + WAVES - 1) / WAVES)), WAVES * 64, ChainShape<F32, DKP>::kBytes, s>>>(p);
}
template <bool F32, int DKP>
void chain(const DeltaParams& p, hipStream_t s) {
  if constexpr (DKP == 256) {
    chain_pass<F32, DKP, false, 4>(p, s);  // (256 rows of a strip do not fit half of a SIMD's registers)
  } else if constexpr (F32) {
    if (p.segs > 1) {
      chain_pass<F32, DKP, true, 8>(p, s);
      launch_delta_join(p, s);
    }
    // Four strips to a workgroup where that gives every compute unit one at most (lengths of their own: two, which are seldom
    // long both): a wave has its SIMD to itself.  us in eight / four: the call above 105 / 96; 8 chunks of 32 heads of
    // 128 x 128 123 / 111, of 64 133 / 122.
    const int64_t halves = (int64_t)p.a.n_seq * p.a.heads_v * ((p.a.d_v + 63) / 64);
    if (p.segs == 1 && p.a.d_v > 64 && halves <= (p.len < 0 ? 512 : 256)) chain_pass<F32, DKP, false, 4>(p, s);
    else chain_pass<F32, DKP, false, 8>(p, s);
  } else {
    chain_pass<F32, DKP, false, 8>(p, s);
  }
}
template <bool F32>
void chunks_type(const DeltaParams& p, hipStream_t s) {
  const unsigned grid = (unsigned)p.slots_total * p.a.heads_v;
  if (p.vec) delta_prepare<F32, true><<<grid, 256, 0, s>>>(p);
  else delta_prepare<F32, false><<<grid, 256, 0, s>>>(p);
  switch (p.dkp) {
    case 32: if constexpr (F32) return chain<F32, 32>(p, s); else return;
    case 64: return chain<F32, 64>(p, s);
    case 96: if constexpr (F32) return chain<F32, 96>(p, s); else return;
    case 128: return chain<F32, 128>(p, s);
    default: return chain<F32, 256>(p, s);
  }
}
}  // namespace

size_t delta_frag_k_bytes(int dtype, int dkp) { return (size_t)3 * 4 * (dkp / 32) * parts_in(dtype == EVCONV_F32) * kFrag; }
size_t delta_frag_t_bytes(int dtype) { return (size_t)kTri * kFrag * (3 + parts_out(dtype == EVCONV_F32)); }

int64_t delta_steps_threads(const DeltaParams& p) { return ((int64_t)p.a.n_seq * p.a.heads_v * ((p.a.d_v + 31) / 32) + 3) / 4 * 256; }
int64_t delta_chunks_threads(const DeltaParams& p) {
  // delta_prepare; delta_chain, of eight strips to a workgroup (the first pass over segments has the keys' strips, too)
  const int strips = (p.a.d_v + 15) / 16 + (p.segs > 1 ? (p.a.d_k + 15) / 16 : 0);
  return std::max((int64_t)p.slots_total * p.a.heads_v * 256, (int64_t)p.a.n_seq * p.a.heads_v * p.segs * ((strips + 7) / 8) * 512);
}

void launch_delta_steps(const DeltaParams& p, hipStream_t s) {
  const bool vec = p.vec && p.a.d_v % 4 == 0 && ((uintptr_t)p.a.state_in | (uintptr_t)p.a.state_out) % 16 == 0;
  const unsigned grid = (unsigned)(delta_steps_threads(p) / 256);
  if (p.a.dtype == EVCONV_BF16) steps_type<true>(p, vec, grid, s);
  else steps_type<false>(p, vec, grid, s);
}

void launch_delta_chunks(const DeltaParams& p, hipStream_t s) {
  if (p.a.dtype == EVCONV_F32) chunks_type<true>(p, s);
  else chunks_type<false>(p, s);
}

}  // namespace evk
