// Product in 8-bit integers with a scale per row and per column (evconv_quant_matmul) on gfx950.
#include "ops_device.h"
#include "ops_kernels.h"

namespace evk {
namespace {

__device__ __forceinline__ float apply_act(float v, int act) {
  if (act == EVCONV_ACT_RELU) return v < 0.0f ? 0.0f : v;  // (a NaN stays one)
  if (act == EVCONV_ACT_SIGMOID) return 1.0f / (1.0f + expf(-v));
  if (act == EVCONV_ACT_TANH) return tanhf(v);
  return v;
}

// A wave: a 16 x 16 block of y, operands straight from memory.
template <bool BF16>
__global__ __launch_bounds__(256) void quant_block(evconv_quant_args a) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int blocks = (a.n + 15) / 16;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t row0 = wave / blocks * 16;
  const int col0 = (int)(wave % blocks) * 16;
  if (row0 >= a.m) return;
  const int8_t* qa = a.a + min(row0 + m, a.m - 1) * a.a_stride + g * 16;
  const int8_t* qb = a.b + (int64_t)min(col0 + m, a.n - 1) * a.b_stride + g * 16;
  i32x4 acc = {0, 0, 0, 0};
  for (int k = 0; k < a.k; k += 64) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i32x4*)(qa + k), *(const i32x4*)(qb + k), acc, 0, 0, 0);
  const int col = col0 + m;
  if (col >= a.n) return;
  const float scale = a.b_scale[col], bias = a.bias ? a.bias[col] : 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = row0 + 4 * g + i;
    if (row < a.m) store_one<BF16>(a.y, row * a.y_stride + col, apply_act((float)acc[i] * a.a_scale[row] * scale + bias, a.act));
  }
}
}  // namespace

QuantPlan plan_quant_matmul(const evconv_quant_args& a) { return QuantPlan{0, 1, 0}; }

void launch_quant_matmul(const evconv_quant_args& a, const QuantPlan& plan, void* workspace, hipStream_t s) {
  const int64_t waves = (a.m + 15) / 16 * ((a.n + 15) / 16);
  const unsigned grid = (unsigned)((waves + 3) / 4);
  if (a.dtype == EVCONV_BF16) quant_block<true><<<grid, 256, 0, s>>>(a);
  else quant_block<false><<<grid, 256, 0, s>>>(a);
}

}  // namespace evk
