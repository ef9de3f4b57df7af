// Product in 8-bit integers with a scale per row and per column (evconv_quant_matmul) on gfx950.
//
// y[m][n] = act(sa[m] sb[n] sum_k a[m][k] b[n][k] + bias[n]).  The sums are those of the 16 x 16 x 64 integer matrix
// instruction: exact, so neither tiles nor splits change a bit of y.  b's rows are the instruction's left operand, so
// that a lane holds values of one row of y: with b's rows taken in the order of weight_row, eight neighbouring ones.
// Few rows: bound by the weights' bytes and the launch; many: by the matrix units (figures at `start`).
#include "ops_device.h"
#include "ops_kernels.h"

namespace evk {
namespace {

constexpr int kSlab = 128;  // bytes of a row that a step of the contraction takes: one cache line

__device__ __forceinline__ float apply_act(float v, int act) {
  if (act == EVCONV_ACT_RELU) return v < 0.0f ? 0.0f : v;  // (a NaN stays one)
  if (act == EVCONV_ACT_SIGMOID) return 1.0f / (1.0f + expf(-v));
  if (act == EVCONV_ACT_TANH) return tanhf(v);
  return v;
}

// Row of b that block `block` holds at its row r: blocks 2 p and 2 p + 1 give a lane (which holds rows 4 g .. 4 g + 3 of
// a result block) the eight rows 32 p + 8 g ...
__device__ __forceinline__ int weight_row(int block, int r) { return 32 * (block >> 1) + 8 * (r >> 2) + 4 * (block & 1) + (r & 3); }

// Factors and biases of eight neighbouring columns
struct Columns {
  float scale[8], bias[8];
  __device__ __forceinline__ Columns(const evconv_quant_args& a, int col) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = min(col + i, a.n - 1);
      scale[i] = a.b_scale[c];
      bias[i] = a.bias ? a.bias[c] : 0.0f;
    }
  }
};
// Eight neighbouring values of a row of y from their sums
template <bool BF16>
__device__ __forceinline__ void put8(const evconv_quant_args& a, int64_t row, int col, float sa, const i32x4& lo, const i32x4& hi, const Columns& k, bool wide) {
  if (row >= a.m || col >= a.n) return;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf((float)(i < 4 ? lo[i] : hi[i - 4]), sa * k.scale[i], k.bias[i]);
  if (a.act != EVCONV_ACT_NONE)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = apply_act(v[i], a.act);
  const int64_t at = row * a.y_stride + col;
  if (wide && col + 8 <= a.n) {
    if constexpr (BF16) {
      *(uint4*)((uint16_t*)a.y + at) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
      *(f32x4*)((float*)a.y + at) = f32x4{v[0], v[1], v[2], v[3]};
      *(f32x4*)((float*)a.y + at + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < a.n) store_one<BF16>(a.y, at + i, v[i]);
  }
}

// ---- tiles through LDS ---------------------------------------------------------------------------------
// Bound by the matrix cores (large), by the weights' bytes and a chain of slabs (few rows).
// A workgroup: BM x BN of y, KG groups of WM x WN waves that take turns at the slabs of the contraction, each with
// two buffers of its own; the loads of a slab go straight into LDS while the one before it is multiplied.
// LDS rows are 128 bytes; the 16-byte pieces of row r stand in the order of key(r), so that the 16 rows a
// load instruction of a wave reads at once lie in different banks.
struct TileParams {
  evconv_quant_args a;
  int tiles_n, tiles, wide;
};
__device__ __forceinline__ int key_a(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int key_b(int row) { return ((row >> 1) & 1) | ((row >> 3) & 3) << 1; }

template <bool BF16, int BM, int BN, int WM, int WN, int KG>
__global__ __launch_bounds__(WM * WN * KG * 64) void quant_tile(TileParams p) {
  constexpr int GT = WM * WN * 64;               // threads of a group
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 blocks of a wave
  constexpr int ROWS = BM + BN, LOADS = ROWS * 8 / GT, STAGE = ROWS * kSlab;
  static_assert(ROWS * 8 % GT == 0 && TN % 2 == 0, "tile");
  extern __shared__ __align__(16) char s_mem[];
  const evconv_quant_args& a = p.a;
  const int group = KG == 1 ? 0 : threadIdx.x / GT, t = KG == 1 ? threadIdx.x : threadIdx.x % GT;
  const int lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), m = lane & 15, g = lane >> 4;
  const int wm = wave / WN, wn = wave % WN;
  // Neighbouring tiles on one XCD (workgroups go round the eight of them), in bands of 8 tiles down
  int tile = blockIdx.x;
  {
    const int per = p.tiles / 8, rest = p.tiles % 8, xcd = tile & 7, i = tile >> 3;
    tile = xcd * per + min(xcd, rest) + i;
  }
  const int tiles_m = p.tiles / p.tiles_n, band = tile / (8 * p.tiles_n), in_band = tile - band * 8 * p.tiles_n;
  const int down = min(8, tiles_m - band * 8);
  const int64_t row0 = (int64_t)(band * 8 + in_band % down) * BM;
  const int col0 = in_band / down * BN;

  char* const mine = s_mem + group * 2 * STAGE;
  const int8_t* from[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int piece = i * GT + t, row = piece >> 3, slot = piece & 7;
    if (row < BM) from[i] = a.a + min(row0 + row, a.m - 1) * a.a_stride + (slot ^ key_a(row)) * 16;
    else from[i] = a.b + (int64_t)min(col0 + row - BM, a.n - 1) * a.b_stride + (slot ^ key_b(row - BM)) * 16;
  }
  const int slabs = (a.k + kSlab - 1) / kSlab, turns = (slabs + KG - 1) / KG;
  auto request = [&](int turn) __attribute__((always_inline)) {
    const int slab = turn * KG + group;
    if (slab >= slabs) return;
    char* const to = mine + (turn & 1) * STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from[i] + (int64_t)slab * kSlab),
                                       (__attribute__((address_space(3))) void*)(to + i * GT * 16), 16, 0, 0);
  };
  i32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  int at_a[TM], at_b[TN], key_m[TM], key_n[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = (wm * TM + i) * 16 + m;
    at_a[i] = row * kSlab;
    key_m[i] = key_a(row);
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int row = weight_row(wn * TN + j, m);
    at_b[j] = (BM + row) * kSlab;
    key_n[j] = key_b(row);
  }
  request(0);
  for (int turn = 0; turn < turns; ++turn) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (turn + 1 < turns) request(turn + 1);
    if (KG > 1 && turn * KG + group >= slabs) continue;
    const char* const q = mine + (turn & 1) * STAGE;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      i32x4 fa[TM], fb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = *(const i32x4*)(q + at_b[j] + ((s * 4 + g) ^ key_n[j]) * 16);
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = *(const i32x4*)(q + at_a[i] + ((s * 4 + g) ^ key_m[i]) * 16);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  }
  if constexpr (KG > 1) {  // the groups' sums meet in LDS
    __syncthreads();
    i32x4* const part = (i32x4*)s_mem;
    if (group > 0)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) part[(((group - 1) * TM + i) * TN + j) * GT + t] = acc[i][j];
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int other = 1; other < KG; ++other)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] += part[(((other - 1) * TM + i) * TN + j) * GT + t];
  }
#pragma unroll
  for (int j = 0; j < TN; j += 2) {
    const int col = col0 + weight_row(wn * TN + j, 4 * g);
    const Columns columns(a, col);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t row = row0 + (wm * TM + i) * 16 + m;
      put8<BF16>(a, row, col, a.a_scale[min(row, a.m - 1)], acc[i][j], acc[i][j + 1], columns, p.wide);
    }
  }
}

template <bool BF16, int BM, int BN, int WM, int WN, int KG>
void start_tile(TileParams p, hipStream_t s) {
  constexpr size_t lds = (size_t)KG * 2 * (BM + BN) * kSlab;
  p.tiles_n = (p.a.n + BN - 1) / BN;
  p.tiles = (int)((p.a.m + BM - 1) / BM) * p.tiles_n;
  quant_tile<BF16, BM, BN, WM, WN, KG><<<p.tiles, WM * WN * KG * 64, lds, s>>>(p);
}
// Small tiles where there are few, and groups of waves that share the contraction, so that enough loads are under
// way; large ones where they fill the chip, so that a byte of LDS feeds more products. us, m x n x k, the
// rows of a rule timed beside their neighbours:
//   16 x 4096 x 4096   16 x 32 by 8 groups 5.1, 32 x 32 by 4 6.2, 64 x 64 10.4  (3.3 TB/s of weights)
//   64 x 4096 x 4096   9.7, 6.9, 10.9;   64 x 1024 x 1024   3.7, 4.0, 5.1
//   1001 x 777 x 1000  64 x 64 5.4, 128 x 128 10.6;   2048 x 2048 x 2048  15.5, 17.5;   4096 x 2048 x 2048  27.9, 23.8
//   3000 x 2048 x 2048  24.2, 22.1;   8000 x 1024 x 4096  54, 39
//   4096 x 4096 x 4096  128 x 128 72, 256 x 256 64.5 (2.1 POP/s);   16384 x 8192 x 2048  323, 308 (1.8 POP/s)
// The largest ones, of which a compute unit holds one at a time, only where more than three quarters of their rounds are full:
//   5000 x 5000 x 3000 (0.78) 101, 94;   6000 x 4096 x 2048 (0.75) 65, 68;   4600 x 4096 x 2048 (0.56) 55, 67
// and both only where not too much of their tiles is outside (inside, of 256 x 256 and of 128 x 128; 64 x 64, 128 x 128, 256 x 256):
//   65536 x 400 x 1024 (0.78, 0.78) 53, 51, 48;   65536 x 200 x 1024 (0.78, 0.78) 31, 29, 27;   65536 x 520 x 1024 (0.68, 0.81) 64, 66, 69
//   65536 x 300 x 1024 (0.59, 0.78) 62, 64, 72;   65536 x 160 x 1024 (0.63, 0.63) 25, 28, 26;   65536 x 257 x 1024 (0.50, 0.67) 54, 56, 67
//   260 x 50000 x 1024 (0.51, 0.68) 31, 34, 43;   65536 x 40 x 1024 (0.16, 0.31) 14, 17, 24
template <bool BF16>
void start(const TileParams& p, hipStream_t s) {
  const evconv_quant_args& a = p.a;
  auto tiles = [&](int bm, int bn) { return ((a.m + bm - 1) / bm) * ((a.n + bn - 1) / bn); };
  auto inside = [&](int side, double share) { return (double)a.m * a.n > share * side * side * tiles(side, side); };
  if (tiles(16, 32) <= 256) start_tile<BF16, 16, 32, 1, 1, 8>(p, s);
  else if (tiles(32, 32) <= 512) start_tile<BF16, 32, 32, 2, 1, 4>(p, s);
  else if (tiles(256, 256) * 4 > (tiles(256, 256) + 255) / 256 * 256 * 3 && inside(256, 0.7)) start_tile<BF16, 256, 256, 2, 4, 1>(p, s);
  else if (tiles(128, 128) >= 384 && inside(128, 0.75)) start_tile<BF16, 128, 128, 2, 2, 1>(p, s);
  else start_tile<BF16, 64, 64, 2, 2, 1>(p, s);
}
}  // namespace

void launch_quant_matmul(const evconv_quant_args& a, hipStream_t s) {
  const bool bf16 = a.dtype == EVCONV_BF16;
  const bool wide = (uintptr_t)a.y % 16 == 0 && a.y_stride * (bf16 ? 2 : 4) % 16 == 0;
  const TileParams p{a, 0, 0, wide};
  if (bf16) start<true>(p, s);
  else start<false>(p, s);
}

}  // namespace evk
