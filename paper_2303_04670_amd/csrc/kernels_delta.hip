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
#include "delta_device.h"

namespace evk {
namespace {

// ---- token by token -------------------------------------------------------------------------------
// A wave: one sequence, one head, 32 columns; 8 lanes x 4 columns across, 8 groups of ROWS rows down.
// o needs S'q after the update, which is e^g (S'q before it) + (k q) d: one pass over the strip gives both
// products, one reduction over the groups sums them.
// Bound by the state's bytes, read once and written once.
template <bool BF16, int ROWS, bool VEC, bool SVEC>
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
  if (s.len > p.short_len) return;
  const int64_t at = state_at(p, seq, head);
  const int row0 = (lane >> 3) * ROWS, col = block * 32 + (lane & 7) * 4;
  f32x4 S[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    S[i] = f32x4{0, 0, 0, 0};
    if (at >= 0 && a.state_in && row0 + i < a.d_k) {
      const float* q = a.state_in + at + (int64_t)(row0 + i) * a.d_v + col;
      if (SVEC) {
        if (col < a.d_v) S[i] = *(const f32x4*)q;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < a.d_v) S[i][j] = q[j];
      }
    }
  }
  const int hk = head / p.share;
  for (int t = 0; t < s.len; ++t) {
    const int64_t token = s.first + t;
    float k[ROWS], q[ROWS], v[4];
    load_run<BF16, ROWS, VEC>(a.k.data, token * a.k.token_stride + hk * a.k.head_stride + row0, a.d_k - row0, k);
    load_run<BF16, ROWS, VEC>(a.q.data, token * a.q.token_stride + hk * a.q.head_stride + row0, a.d_k - row0, q);
    load_run<BF16, 4, false>(a.v.data, token * a.v.token_stride + head * a.v.head_stride + col, a.d_v - col, v);
    const Gates gate = gates_of(p, token, head);
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
      rk = 1.0f / sqrtf(sum[9] + 1e-6f);
      rq = a.scale / sqrtf(sum[10] + 1e-6f);
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
        if (SVEC) {
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
__global__ __launch_bounds__(256) void delta_prepare(DeltaParams p) {
  constexpr int PI = parts_in(F32), PO = parts_out(F32);
  const evconv_delta_args& a = p.a;
  __shared__ float s_a[C][C + 1], s_t[C][C + 1], s_p[C][C + 1];
  __shared__ double s_g[C];
  __shared__ float s_beta[C], s_rk[C], s_rq[C];
  __shared__ int s_bad;  // first token whose row of A is not finite
  const int slot = blockIdx.x / a.heads_v, head = blockIdx.x % a.heads_v, hk = head / p.share;
  // the last sequence whose first slot is not behind this one
  int seq = 0;
  {
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (first_slot(span_of(p, mid), mid) <= slot) lo = mid; else hi = mid - 1;
    }
    seq = lo;
  }
  const Span span = span_of(p, seq);
  const int chunk = slot - first_slot(span, seq);
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
  {
    const int t = tid >> 2, part = tid & 3;  // four threads to a token
    float rk = 1.0f, rq = 1.0f;
    if (a.flags & EVCONV_DELTA_NORMALIZE) {
      float kk = 0.0f, qq = 0.0f;
      if (t < count)
        for (int c = part * 8; c < a.d_k; c += 32) {
          float k[8], q[8];
          load_run<!F32, 8, VEC>(a.k.data, (token0 + t) * a.k.token_stride + hk * a.k.head_stride + c, a.d_k - c, k);
          load_run<!F32, 8, VEC>(a.q.data, (token0 + t) * a.q.token_stride + hk * a.q.head_stride + c, a.d_k - c, q);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            kk = fmaf(k[j], k[j], kk);
            qq = fmaf(q[j], q[j], qq);
          }
        }
      kk += __shfl_xor(kk, 1);
      kk += __shfl_xor(kk, 2);
      qq += __shfl_xor(qq, 1);
      qq += __shfl_xor(qq, 2);
      rk = 1.0f / sqrtf(kk + 1e-6f);
      rq = 1.0f / sqrtf(qq + 1e-6f);
    }
    if (part == 0) {
      s_rk[t] = rk;
      s_rq[t] = rq * a.scale;
    }
  }
  for (int i = tid; i < C * C; i += 256) s_t[i / C][i % C] = 0.0f;
  if (tid == 0) s_bad = C;

  // ---- K K' and Q K', a wave 16 tokens' rows of them
  f32x4 kk[4], qk[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) kk[b] = qk[b] = f32x4{0, 0, 0, 0};
  for (int c = 0; c < p.dkp; c += 32) {
    b16x8 ka[PI], qa[PI], kb[PI];
    const int row = wave * 16 + m;
    load_parts<F32, VEC>(a.k, hk, a.d_k, token0 + row, row < count, c + 8 * g, ka);
    load_parts<F32, VEC>(a.q, hk, a.d_k, token0 + row, row < count, c + 8 * g, qa);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (b > wave) break;
      const int other = b * 16 + m;
      load_parts<F32, VEC>(a.k, hk, a.d_k, token0 + other, other < count, c + 8 * g, kb);
      mfma_parts<2>(kk[b], ka, kb);
      mfma_parts<2>(qk[b], qa, kb);
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
      s_p[row][col] = y;
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

  // ---- T and P as left operands, the factors of the rows
  char* const at_t = p.frag_t + (size_t)blockIdx.x * (kTri * kFrag * (3 + PO));
  for (int f = wave; f < 2 * kTri; f += 4) {
    const bool is_p = f >= kTri;
    const int i = is_p ? f - kTri : f, b = i < 2 ? i : 2 + (i - 2) / 2, s = i < 2 ? 0 : (i - 2) % 2;
    const int row = place(b, m), col = 32 * s + 8 * g;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = is_p ? s_p[row][col + j] : col + j <= row ? s_t[row][col + j] : 0.0f;
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
  // ---- K, Q and K' as left operands, once per key head
  if (head % p.share == 0) {
    const int steps = p.dkp / 32;
    const size_t one = (size_t)4 * steps * PI * kFrag;  // of K; the same of Q and K'
    char* const at_k = p.frag_k + ((size_t)slot * a.heads_k + hk) * 3 * one;
    for (int f = wave; f < 8 * steps; f += 4) {
      const bool is_q = f >= 4 * steps;
      const int i = is_q ? f - 4 * steps : f, b = i / steps, s = i % steps, row = place(b, m);
      b16x8 out[PI];
      load_parts<F32, VEC>(is_q ? a.q : a.k, hk, a.d_k, token0 + row, row < count, 32 * s + 8 * g, out);
#pragma unroll
      for (int part = 0; part < PI; ++part) *(b16x8*)(at_k + is_q * one + (size_t)(i * PI + part) * kFrag + lane * 16) = out[part];
    }
    for (int f = wave; f < 4 * steps; f += 4) {
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
// A wave: one sequence, one value head, 16 columns of the state, which stay in its registers.
template <bool F32, int DKP>
__global__ __launch_bounds__(64) void delta_chain(DeltaParams p) {
  constexpr int PI = parts_in(F32), PO = parts_out(F32), STEPS = DKP / 32, ORD = F32 ? 2 : 1;
  const evconv_delta_args& a = p.a;
  const int strips = (a.d_v + 15) / 16;
  // strips of a head on one XCD (workgroups go round the eight of them): they read the same operands
  const int xcd = blockIdx.x & 7, r = blockIdx.x >> 3;
  const int strip = r % strips;
  const int64_t pair = (int64_t)(r / strips) * 8 + xcd;
  if (pair >= (int64_t)a.n_seq * a.heads_v) return;
  const int seq = (int)(pair / a.heads_v), head = (int)(pair % a.heads_v), hk = head / p.share;
  const Span span = span_of(p, seq);
  if (span.len <= p.short_len) return;
  const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
  const int col = strip * 16 + n;
  const bool in = col < a.d_v;
  const int64_t at = state_at(p, seq, head);
  f32x4 S[2 * STEPS];
#pragma unroll
  for (int b = 0; b < 2 * STEPS; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = place(b, 4 * g + i);
      S[b][i] = at >= 0 && a.state_in && row < a.d_k && in ? a.state_in[at + (int64_t)row * a.d_v + col] : 0.0f;
    }
  const size_t one = (size_t)4 * STEPS * PI * kFrag;
  const int chunks = (span.len + C - 1) / C;
  const int slot0 = first_slot(span, seq);
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const int64_t token0 = span.first + chunk * C;
    const int count = min(span.len - chunk * C, C);
    const size_t slot = slot0 + chunk;
    const char* const at_k = p.frag_k + (slot * a.heads_k + hk) * 3 * one + lane * 16;
    const char* const at_t = p.frag_t + (slot * a.heads_v + head) * (kTri * kFrag * (3 + PO)) + lane * 16;
    const float* const scal = p.scal + (slot * a.heads_v + head) * kDeltaScalars;
    auto frag = [](const char* q, int i) __attribute__((always_inline)) { return *(const b16x8*)(q + (size_t)i * kFrag); };

    // S as right operand
    b16x8 Sp[STEPS][3];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = S[2 * s][i];
        v[4 + i] = S[2 * s + 1][i];
      }
      split8(v, Sp[s]);
    }
    // R = beta v - beta e^G K S, and e^G Q S
    f32x4 R[4], O[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      R[b] = O[b] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        b16x8 k[PI], q[PI];
#pragma unroll
        for (int part = 0; part < PI; ++part) {
          k[part] = frag(at_k, (b * STEPS + s) * PI + part);
          q[part] = frag(at_k + one, (b * STEPS + s) * PI + part);
        }
        mfma_parts<2>(R[b], k, Sp[s]);
        mfma_parts<ORD>(O[b], q, Sp[s]);
      }
    }
    unsigned bad = 0;
    f32x4 w[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int t0 = place(b, 4 * g);  // this lane's tokens: t0 .. t0 + 3
      const f32x4 beta = *(const f32x4*)(scal + t0), kf = *(const f32x4*)(scal + C + t0), qf = *(const f32x4*)(scal + 2 * C + t0);
      w[b] = *(const f32x4*)(scal + 3 * C + t0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool live = t0 + i < count && in;
        const float v = live ? load_one<!F32>(a.v.data, (token0 + t0 + i) * a.v.token_stride + head * a.v.head_stride + col) : 0.0f;
        R[b][i] = t0 + i < count ? beta[i] * v - kf[i] * R[b][i] : 0.0f;
        O[b][i] *= qf[i];
        if (!(fabsf(R[b][i]) < kBf16Overflow)) bad |= 1u << (b * 4 + i);
      }
    }
    int first_bad = C;
    if (__ballot(bad != 0)) cut_columns(R, bad, first_bad, g);
    // D = T R
    b16x8 Rp[2][3];
    f32x4 D[4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = R[2 * s][i];
        v[4 + i] = R[2 * s + 1][i];
      }
      split8(v, Rp[s]);
    }
    bad = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      D[b] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < 1 + (b >> 1); ++s) {
        b16x8 t[3];
#pragma unroll
        for (int part = 0; part < 3; ++part) t[part] = frag(at_t, tri(b, s) * 3 + part);
        mfma_parts<2>(D[b], t, Rp[s]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!(fabsf(D[b][i]) < kBf16Overflow)) bad |= 1u << (b * 4 + i);
    }
    if (__ballot(bad != 0 || first_bad < C)) cut_columns(D, bad, first_bad, g);
    // O += P D;  S = e^G S + K' (w D)
    const float decay = scal[4 * C];
#pragma unroll
    for (int b = 0; b < 2 * STEPS; ++b) S[b] *= decay;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float v[8], vw[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = D[2 * s][i];
        v[4 + i] = D[2 * s + 1][i];
        vw[i] = v[i] * w[2 * s][i];
        vw[4 + i] = v[4 + i] * w[2 * s + 1][i];
      }
      b16x8 Dp[PO], Dw[3];
      split8(v, Dp);
      split8(vw, Dw);
#pragma unroll
      for (int b = 2 * s; b < 4; ++b) {
        b16x8 pp[PO];
#pragma unroll
        for (int part = 0; part < PO; ++part) pp[part] = frag(at_t + kTri * 3 * kFrag, tri(b, s) * PO + part);
        mfma_parts<ORD>(O[b], pp, Dp);
      }
#pragma unroll
      for (int b = 0; b < 2 * STEPS; ++b) {
        b16x8 kt[PI];
#pragma unroll
        for (int part = 0; part < PI; ++part) kt[part] = frag(at_k + 2 * one, (b * 2 + s) * PI + part);
        mfma_parts<2>(S[b], kt, Dw);
      }
    }
    if (first_bad < C)
#pragma unroll
      for (int b = 0; b < 2 * STEPS; ++b) S[b] = f32x4{NAN, NAN, NAN, NAN};
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = place(b, 4 * g) + i;
        if (t < count && in)
          store_one<!F32>(a.o, (token0 + t) * a.o_token_stride + head * a.o_head_stride + col, t < first_bad ? O[b][i] : NAN);
      }
  }
  if (at >= 0 && a.state_out && in)
#pragma unroll
    for (int b = 0; b < 2 * STEPS; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = place(b, 4 * g + i);
        if (row < a.d_k) a.state_out[at + (int64_t)row * a.d_v + col] = S[b][i];
      }
}

template <bool BF16, int ROWS>
void steps_rows(const DeltaParams& p, bool svec, unsigned grid, hipStream_t s) {
  if (p.vec && svec) delta_step<BF16, ROWS, true, true><<<grid, 256, 0, s>>>(p);
  else delta_step<BF16, ROWS, false, false><<<grid, 256, 0, s>>>(p);
}
template <bool BF16>
void steps_type(const DeltaParams& p, bool svec, unsigned grid, hipStream_t s) {
  if (p.a.d_k <= 32) steps_rows<BF16, 4>(p, svec, grid, s);
  else if (p.a.d_k <= 64) steps_rows<BF16, 8>(p, svec, grid, s);
  else if (p.a.d_k <= 128) steps_rows<BF16, 16>(p, svec, grid, s);
  else steps_rows<BF16, 32>(p, svec, grid, s);
}
template <bool F32, int DKP>
void chain(const DeltaParams& p, hipStream_t s) {
  const int64_t pairs = (int64_t)p.a.n_seq * p.a.heads_v, strips = (p.a.d_v + 15) / 16;
  delta_chain<F32, DKP><<<(unsigned)((pairs + 7) / 8 * 8 * strips), 64, 0, s>>>(p);
}
template <bool F32>
void chunks_type(const DeltaParams& p, hipStream_t s) {
  const unsigned grid = (unsigned)p.slots_total * p.a.heads_v;
  if (p.vec) delta_prepare<F32, true><<<grid, 256, 0, s>>>(p);
  else delta_prepare<F32, false><<<grid, 256, 0, s>>>(p);
  switch (p.dkp) {
    case 64: return chain<F32, 64>(p, s);
    case 128: return chain<F32, 128>(p, s);
    default: return chain<F32, 256>(p, s);
  }
}
}  // namespace

size_t delta_frag_k_bytes(int dtype, int dkp) { return (size_t)3 * 4 * (dkp / 32) * parts_in(dtype == EVCONV_F32) * kFrag; }
size_t delta_frag_t_bytes(int dtype) { return (size_t)kTri * kFrag * (3 + parts_out(dtype == EVCONV_F32)); }

void launch_delta_steps(const DeltaParams& p, hipStream_t s) {
  const bool svec = p.a.d_v % 4 == 0 && ((uintptr_t)p.a.state_in | (uintptr_t)p.a.state_out) % 16 == 0;
  const int64_t waves = (int64_t)p.a.n_seq * p.a.heads_v * ((p.a.d_v + 31) / 32);
  const unsigned grid = (unsigned)((waves + 3) / 4);
  if (p.a.dtype == EVCONV_BF16) steps_type<true>(p, svec, grid, s);
  else steps_type<false>(p, svec, grid, s);
}

void launch_delta_chunks(const DeltaParams& p, hipStream_t s) {
  if (p.a.dtype == EVCONV_F32) chunks_type<true>(p, s);
  else chunks_type<false>(p, s);
}

}  // namespace evk
