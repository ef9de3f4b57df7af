// The norms around a block (evconv_block_norm) on gfx950: a row stays in the registers of its threads
// from its one read to its one write, so the kernel is bound by the rows' bytes (few rows: by the
// chain of a launch, a read, one to five reductions and a write).  In fp32 it runs at 4.9 to 5.1 TB/s,
// the rate of a large copy; in bf16 at 4.3 to 4.9: half the bytes to the same exponentials, roundings and
// fp32 weights.  The sums go over a row twice (mean, then squares of differences), so no cancellation.
#include <algorithm>

#include "ops_device.h"
#include "ops_kernels.h"

namespace evk {
namespace {

struct NormParams {
  evconv_norm_args a;
  int lanes;     // threads to a group: a power of two that holds it in vectors of eight
  int64_t row0;  // first row of this launch
};

// Sum over `lanes` neighbouring lanes (a power of two up to 64), the same in all of them.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int d = 1; d < lanes; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Sum (largest bit pattern) over the T threads of a row.
template <int T>
__device__ __forceinline__ float row_sum(float v, float* s_part) {
  v = lanes_sum(v, 64);
  if constexpr (T > 64) {
    __syncthreads();  // (the last reduction's values have been read)
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) v += s_part[i];
  }
  return v;
}
template <int T>
__device__ __forceinline__ unsigned row_max(unsigned v, float* s_part) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = max(v, (unsigned)__shfl_xor((int)v, d));
  if constexpr (T > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = __uint_as_float(v);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T / 64; ++i) v = max(v, __float_as_uint(s_part[i]));
  }
  return v;
}

// Eight fp32 parameters from index i on
template <bool VEC>
__device__ __forceinline__ void load_weights(const float* w, int i, int left, float (&v)[8]) {
  load_run<false, 8, VEC>(w, i, left, v);
}

template <bool BF16, bool VEC>
__device__ __forceinline__ void store_run(void* q, int64_t i, int left, const float (&v)[8]) {
  if constexpr (VEC) {
    if (left <= 0) return;
    if constexpr (BF16) {
      *(uint4*)((uint16_t*)q + i) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
      *(f32x4*)((float*)q + i) = f32x4{v[0], v[1], v[2], v[3]};
      *(f32x4*)((float*)q + i + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) store_one<BF16>(q, i + j, v[j]);
  }
}

// 1 / (1 + exp(-z)).  Of bf16 outputs with the hardware's exponential and reciprocal, whose errors (2^-23, and 2^-24 |z| in the
// exponent, which counts only where the sum is near 1 or the exponential itself is the result) stay far under the outputs' 2^-9.
template <bool BF16>
__device__ __forceinline__ float sigmoid_of(float z) {
  if constexpr (BF16) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
  else return 1.0f / (1.0f + expf(-z));
}

// T threads to a row (64: a wave, several rows to a workgroup), NV vectors of eight values each.
// GROUPED: the branch's norm is over groups (heads) of p.a.group values, each held by p.lanes lanes of one
// wave; otherwise over the row.
template <bool BF16, bool VEC, int T, int NV, bool GROUPED>
__global__ __launch_bounds__(T == 64 ? 256 : T) void block_norm(NormParams p) {
  __shared__ float s_part[T / 64];
  const evconv_norm_args& a = p.a;
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = p.row0 + (T == 64 ? (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6) : blockIdx.x);
  if (row >= a.rows) return;  // (T > 64: never, so every thread of a row meets its barriers)
  const int dim = a.dim, group = GROUPED ? a.group : dim;
  int at[NV], left[NV], in_group[NV];  // first value of a vector, how many are inside, its place in the group
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if (GROUPED) {
      const int which = v * (T / p.lanes) + t / p.lanes, off = t % p.lanes * 8;
      at[v] = which * group + off;
      left[v] = which < dim / group ? min(group - off, 8) : 0;
      in_group[v] = off;
    } else {
      at[v] = (v * T + t) * 8;
      left[v] = min(dim - at[v], 8);
      in_group[v] = at[v];
    }
  }
  // whether value j of vector v is inside (vectors of a multiple of eight are so as a whole)
  auto inside = [&](int v, int j) __attribute__((always_inline)) { return VEC ? left[v] > 0 : j < left[v]; };
  float y[NV][8], x[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if (a.branch) load_run<BF16, 8, VEC>(a.branch, row * a.branch_stride + at[v], left[v], y[v]);
    if (a.x) load_run<BF16, 8, VEC>(a.x, row * a.x_stride + at[v], left[v], x[v]);
  }
  // ---- the branch: norm, gate, scale, sum
  if (a.branch) {
    float z[NV][8];
    if (a.gate)
#pragma unroll
      for (int v = 0; v < NV; ++v) load_run<BF16, 8, VEC>(a.gate, row * a.gate_stride + at[v], left[v], z[v]);
    float scale[NV], mean[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) mean[v] = 0.0f;
    // one sum per group, or one over all vectors
    auto sums = [&](auto&& of, float (&out)[NV]) __attribute__((always_inline)) {
      float all = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (inside(v, j)) s += of(v, j);
        if (GROUPED) out[v] = lanes_sum(s, p.lanes);
        all += s;
      }
      if (!GROUPED) {
        all = row_sum<T>(all, s_part);
#pragma unroll
        for (int v = 0; v < NV; ++v) out[v] = all;
      }
    };
    if (a.norm == EVCONV_NORM_LAYER) {
      sums([&](int v, int j) { return y[v][j]; }, mean);
#pragma unroll
      for (int v = 0; v < NV; ++v) mean[v] /= (float)group;
    }
    sums([&](int v, int j) { const float d = y[v][j] - mean[v]; return d * d; }, scale);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      scale[v] = 1.0f / sqrtf(scale[v] / (float)group + a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[v][j] = (y[v][j] - mean[v]) * scale[v];
      float w[8];
      if (a.post_weight) {
        load_weights<VEC>(a.post_weight, in_group[v], left[v], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] *= w[j];
      }
      if (a.post_bias) {
        load_weights<VEC>(a.post_bias, in_group[v], left[v], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] += w[j];
      }
      if (a.gate)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float s = sigmoid_of<BF16>(z[v][j]);
          y[v][j] *= a.gate_act == EVCONV_GATE_SILU ? z[v][j] * s : s;
        }
      if (a.res_scale) {
        load_weights<VEC>(a.res_scale, at[v], left[v], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] *= w[j];
      }
      if (a.x)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] += x[v][j];
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) y[v][j] = x[v][j];
  }
  if (a.x_out)
#pragma unroll
    for (int v = 0; v < NV; ++v) store_run<BF16, VEC>(a.x_out, row * a.x_out_stride + at[v], left[v], y[v]);
  if (!a.h_out && !a.q) return;
  // ---- the norm before the next block, over the whole row
  if (a.pre_norm) {
    auto sum = [&](float mean, bool square) __attribute__((always_inline)) {
      float s = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (inside(v, j)) s += square ? (y[v][j] - mean) * (y[v][j] - mean) : y[v][j];
      return row_sum<T>(s, s_part);
    };
    const float mean = a.norm == EVCONV_NORM_LAYER ? sum(0.0f, false) / (float)dim : 0.0f;
    const float scale = 1.0f / sqrtf(sum(mean, true) / (float)dim + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[v][j] = (y[v][j] - mean) * scale;
      if (a.pre_weight) {
        load_weights<VEC>(a.pre_weight, at[v], left[v], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] *= w[j];
      }
      if (a.pre_bias) {
        load_weights<VEC>(a.pre_bias, at[v], left[v], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] += w[j];
      }
    }
  }
  if (a.h_out)
#pragma unroll
    for (int v = 0; v < NV; ++v) store_run<BF16, VEC>(a.h_out, row * a.h_out_stride + at[v], left[v], y[v]);
  if (!a.q) return;
  // ---- 8 bits.  The largest magnitude by its bits: those of an infinity or a NaN are above every number's.
  unsigned big = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (inside(v, j)) big = max(big, __float_as_uint(y[v][j]) & 0x7fffffffu);
  big = row_max<T>(big, s_part);
  const float m = __uint_as_float(big);
  const bool finite = big < 0x7f800000u;
  float inverse = finite && big ? 127.0f * (1.0f / m) : 0.0f;
  if (!(inverse < INFINITY)) inverse = 0.0f;
  int8_t* const q = a.q + row * a.q_stride;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = finite ? (int)rintf(y[v][j] * inverse) : 0;
      w[j / 4] |= (unsigned)(i & 255) << (j % 4 * 8);
      if (!VEC && j < left[v]) q[at[v] + j] = (int8_t)i;
    }
    if (VEC && left[v] > 0) *(uint2*)(q + at[v]) = make_uint2(w[0], w[1]);
  }
  for (int c = dim + t; c < a.q_stride; c += T) q[c] = 0;
  if (t == 0) a.q_scale[row] = finite ? m / 127.0f : NAN;
}

template <bool BF16, bool VEC, int T, int NV>
void start(NormParams p, hipStream_t s) {
  // waves of a workgroup: one where there are few rows, so that they spread over the chip
  const int per = T > 64 ? 1 : p.a.rows >= 2048 ? 4 : 1;
  const int threads = T > 64 ? T : 64 * per;
  const int64_t most = kMostThreads / 2 / threads * per;  // rows of a launch
  for (; p.row0 < p.a.rows; p.row0 += most) {
    const unsigned grid = (unsigned)((std::min(most, p.a.rows - p.row0) + per - 1) / per);
    if (p.a.group == p.a.dim) block_norm<BF16, VEC, T, NV, false><<<grid, threads, 0, s>>>(p);
    else block_norm<BF16, VEC, T, NV, true><<<grid, threads, 0, s>>>(p);
  }
}

// How a row is laid over threads, by its vectors.  More values to a thread save barriers and shared reductions; fewer leave
// room for the waves that hide the reads (four vectors: 3 waves per SIMD; one: 8).  us for 32 Mi values of x' and h from x, branch
// and SiLU gate with three weights, rms (336 MB in bf16, 671 MB in fp32: 64 and 128 at the rate of a large copy), bf16 / fp32:
//   dim 1024    64 x 2 69 / 133, 128 x 1 70 / 132          dim 2048   64 x 4 88 / -, 256 x 1 76 / 136
//   dim 4096   256 x 2 75 / 140, 512 x 1 79 / 134          dim 8192  256 x 4 95 / 144, 512 x 2 78 / 139
// and 1024 x 2 at 16384 93 / 169 (one row to a CU at a time).
template <bool BF16, bool VEC>
void start_size(const NormParams& p, hipStream_t s) {
  const int vectors = block_norm_vectors(p.a);
  if (vectors <= 64) start<BF16, VEC, 64, 1>(p, s);
  else if (vectors <= 128) start<BF16, VEC, 64, 2>(p, s);
  else if (vectors <= 256) start<BF16, VEC, 256, 1>(p, s);
  else if (vectors <= 512) start<BF16, VEC, 256, 2>(p, s);
  else if (vectors <= 1024) start<BF16, VEC, 512, 2>(p, s);
  else start<BF16, VEC, 1024, 2>(p, s);
}
}  // namespace

// Threads to a group.
static int group_lanes(const evconv_norm_args& a) {
  int lanes = 1;
  while (lanes * 8 < a.group && lanes < 64) lanes *= 2;
  return lanes;
}
int block_norm_vectors(const evconv_norm_args& a) { return a.group == a.dim ? (a.dim + 7) / 8 : a.dim / a.group * group_lanes(a); }

void launch_block_norm(const evconv_norm_args& a, bool vec, hipStream_t s) {
  const NormParams p{a, group_lanes(a), 0};
  if (a.dtype == EVCONV_BF16) vec ? start_size<true, true>(p, s) : start_size<true, false>(p, s);
  else vec ? start_size<false, true>(p, s) : start_size<false, false>(p, s);
}

}  // namespace evk
