// What the norms over the rows of a matrix share (layer_norm.hip, rms_norm.hip): lanes that share a row, sums over them, and the fold of the workgroups'
// partial sums of a parameter's gradient.
#pragma once

#include "sequence.h"
#include "typed.h"

namespace rslx {

namespace {

constexpr int NORM_THREADS = 256;

// Sum over the TPR lanes of a row; every lane gets it.  `lds`: one float per wavefront and value, double-buffered by the caller.
template <int TPR, int COUNT>
__device__ __forceinline__ void row_sum(float (&v)[COUNT], float* lds) {
  constexpr int IN_WAVE = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = IN_WAVE / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < COUNT; ++i) lds[i * WAVES + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += lds[i * WAVES + w];
      v[i] = s;
    }
  }
}

template <int W, bool WHOLE>
__device__ __forceinline__ bool in_row(int c, int k, int cols) { return WHOLE ? c < cols : c + k < cols; }

// Rows that one workgroup takes at a time.
template <int TPR> constexpr int THREADS_OF = TPR > NORM_THREADS ? TPR : NORM_THREADS;

// dw[c] = sum over the workgroups' partial sums (blockIdx.y = 0), db[c] likewise (1): 16 columns, 64 lanes a column.
constexpr int FOLD_LANES = 64;
__global__ __launch_bounds__(16 * FOLD_LANES) void norm_fold_kernel(const float* partials, int blocks, int cols, float* dweight, float* dbias) {
  __shared__ float lds[FOLD_LANES][17], lds8[8][17];
  float* out = blockIdx.y == 0 ? dweight : dbias;
  if (!out) return;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  const float* p = partials + (int64_t)blockIdx.y * blocks * cols;
  float v[NORM_MAX_BLOCKS / FOLD_LANES], s = 0.f;
#pragma unroll
  for (int i = 0; i < NORM_MAX_BLOCKS / FOLD_LANES; ++i) v[i] = col < cols && r + i * FOLD_LANES < blocks ? p[(int64_t)(r + i * FOLD_LANES) * cols + col] : 0.f;
#pragma unroll
  for (int i = 0; i < NORM_MAX_BLOCKS / FOLD_LANES; ++i) s += v[i];
  lds[r][c] = s;
  __syncthreads();
  if (r < 8) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += lds[r * 8 + k][c];
    lds8[r][c] = s;
  }
  __syncthreads();
  if (r == 0 && col < cols) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += lds8[k][c];
    out[col] = s;
  }
}

// How many lanes share a row and how many loads of 16 bytes each makes.
struct NormShape { int tpr, items; };
inline NormShape norm_shape(int cols, int w) {
  const int n = (cols + w - 1) / w;
  if (n <= 16) return {16, 1};
  if (n <= 32) return {32, 1};
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  if (n <= 256) return {256, 1};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {512, 2};
  if (n <= 2048) return {1024, 2};
  return {1024, 4};
}

inline int norm_rows_per_block(int tpr) { return tpr > NORM_THREADS ? 1 : NORM_THREADS / tpr; }

}  // namespace

}  // namespace rslx
