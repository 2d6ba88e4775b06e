// Layer norm over the rows of a matrix, forward and backward, gfx950.
//
//   m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps),  y = (x - m) r w + b
//   g = dy w,  h = (x - m) r:   dx = r (g - mean g - h mean(g h)),   dw = sum over rows dy h,   db = sum over rows dy
//
// Both are bound by memory: a row is read once into registers (W values a load, ITEMS loads a lane), everything that needs the
// whole row happens there (the variance from the centred values, so that rows far from zero keep their digits; what rounding left of the
// mean shows in the sum of the same values, and is taken off too), and the result is written once.  TPR lanes share a row: part of a wavefront, a wavefront, or a workgroup where one wavefront's registers
// would not hold it.  Sums are fp32: a lane's values in order, then a fixed tree.
#include "sequence.h"
#include "typed.h"

namespace rslx {

namespace {

constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_FORWARD = 1 << 20;     // workgroups of a forward launch; more rows go round

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

template <typename T, int W, int ITEMS, int TPR>
__global__ __launch_bounds__(TPR > NORM_THREADS ? TPR : NORM_THREADS) void layer_norm_kernel(NormArgs a) {
  constexpr int THREADS = TPR > NORM_THREADS ? TPR : NORM_THREADS, ROWS = THREADS / TPR;
  __shared__ float lds[2][2 * (TPR > 64 ? TPR / 64 : 1)];
  const int lane = threadIdx.x % TPR;
  const float n = (float)a.cols;
  // (TPR <= 64: lanes leave the loop in whole rows, and the shuffles stay inside a row; above, the workgroup has one row)
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    Pack<T, W> in[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * TPR + lane) * W;
      if (c < a.cols) in[i] = *reinterpret_cast<const Pack<T, W>*>(x + c);
    }
    float f[ITEMS * W], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        f[i * W + k] = (i * TPR + lane) * W < a.cols ? to_float(in[i].v[k]) : 0.f;
        s[0] += f[i * W + k];
      }
    row_sum<TPR, 1>(s, lds[0]);
    const float near = s[0] / n;
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        f[i * W + k] = (i * TPR + lane) * W < a.cols ? f[i * W + k] - near : 0.f;
        q[0] += f[i * W + k];
        q[1] += f[i * W + k] * f[i * W + k];
      }
    row_sum<TPR, 2>(q, lds[1]);
    const float rest = q[0] / n, mean = near + rest;
    const float variance = q[1] / n - rest * rest;
    const float rstd = 1.f / sqrtf((variance < 0.f ? 0.f : variance) + a.eps);
    T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * TPR + lane) * W;
      if (c < a.cols) {
        Pack<T, W> out;
        Pack<float, W> w, b;
        if (a.weight) w = *reinterpret_cast<const Pack<float, W>*>(a.weight + c);
        if (a.bias) b = *reinterpret_cast<const Pack<float, W>*>(a.bias + c);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          float v = (f[i * W + k] - rest) * rstd;
          if (a.weight) v *= w.v[k];
          if (a.bias) v += b.v[k];
          out.v[k] = from_float<T>(v);
        }
        *reinterpret_cast<Pack<T, W>*>(y + c) = out;
      }
    }
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// The backward pass: a workgroup takes every gridDim.x-th set of rows, so that a lane's columns stay the same and their
// gradients of weight and bias add up in its registers; what the workgroup holds in the end is one row of partial sums, which
// norm_fold_kernel adds up in a fixed order (no atomics: the same inputs give the same bits).
template <typename T, int W, int ITEMS, int TPR>
__global__ __launch_bounds__(TPR > NORM_THREADS ? TPR : NORM_THREADS) void layer_norm_backward_kernel(NormArgs a) {
  constexpr int THREADS = TPR > NORM_THREADS ? TPR : NORM_THREADS, ROWS = THREADS / TPR;
  __shared__ float lds[2][2 * (TPR > 64 ? TPR / 64 : 1)];
  __shared__ float join[ROWS > 1 ? (ROWS - 1) * TPR * ITEMS * W : 1];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv = 1.f / (float)a.cols;
  float dw[ITEMS * W], db[ITEMS * W];
#pragma unroll
  for (int i = 0; i < ITEMS * W; ++i) dw[i] = db[i] = 0.f;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < a.rows; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    Pack<T, W> px[ITEMS], pd[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * TPR + lane) * W;
      if (c < a.cols) {
        px[i] = *reinterpret_cast<const Pack<T, W>*>(x + c);
        pd[i] = *reinterpret_cast<const Pack<T, W>*>(dy + c);
      }
    }
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * TPR + lane) * W;
      if (c < a.cols) {
        Pack<float, W> w;
        if (a.weight) w = *reinterpret_cast<const Pack<float, W>*>(a.weight + c);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          const float d = to_float(pd[i].v[k]), h = (to_float(px[i].v[k]) - mean) * rstd, g = a.weight ? d * w.v[k] : d;
          dw[i * W + k] += d * h;
          db[i * W + k] += d;
          s[0] += g;
          s[1] += g * h;
        }
      }
    }
    if (a.dx) {
      row_sum<TPR, 2>(s, lds[turn]);
      const float mg = s[0] * inv, mgh = s[1] * inv;
      T* dx = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * TPR + lane) * W;
        if (c < a.cols) {
          Pack<T, W> out;
          Pack<float, W> w;
          if (a.weight) w = *reinterpret_cast<const Pack<float, W>*>(a.weight + c);
#pragma unroll
          for (int k = 0; k < W; ++k) {
            const float d = to_float(pd[i].v[k]), h = (to_float(px[i].v[k]) - mean) * rstd, g = a.weight ? d * w.v[k] : d;
            out.v[k] = from_float<T>(rstd * (g - mg - h * mgh));
          }
          *reinterpret_cast<Pack<T, W>*>(dx + c) = out;
        }
      }
    }
  }
  if (!a.partials) return;
  // the workgroup's sets of lanes, first weight, then bias
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    float(&v)[ITEMS * W] = pass == 0 ? dw : db;
    if constexpr (ROWS > 1) {
      __syncthreads();
      if (sub > 0)
#pragma unroll
        for (int i = 0; i < ITEMS * W; ++i) join[((sub - 1) * ITEMS * W + i) * TPR + lane] = v[i];
      __syncthreads();
      if (sub == 0)
        for (int r = 0; r < ROWS - 1; ++r)
#pragma unroll
          for (int i = 0; i < ITEMS * W; ++i) v[i] += join[(r * ITEMS * W + i) * TPR + lane];
    }
    if (sub == 0) {
      float* to = a.partials + ((int64_t)pass * gridDim.x + blockIdx.x) * a.cols;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * TPR + lane) * W;
        if (c < a.cols)
#pragma unroll
          for (int k = 0; k < W; ++k) to[c + k] = v[i * W + k];
      }
    }
  }
}

// dw[c] = sum over the workgroups' partial sums (blockIdx.y = 0), db[c] likewise (1): 16 columns, 16 lanes a column.
__global__ __launch_bounds__(256) void norm_fold_kernel(const float* partials, int blocks, int cols, float* dweight, float* dbias) {
  __shared__ float lds[16][17];
  float* out = blockIdx.y == 0 ? dweight : dbias;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  const float* p = partials + (int64_t)blockIdx.y * blocks * cols;
  float s = 0.f;
  if (col < cols)
    for (int b = r; b < blocks; b += 16) s += p[(int64_t)b * cols + col];
  lds[r][c] = s;
  __syncthreads();
  if (out && r == 0 && col < cols) {
    for (int k = 1; k < 16; ++k) s += lds[k][c];
    out[col] = s;
  }
}

// How many lanes share a row and how many loads each makes.
struct NormShape { int tpr, items; };
NormShape norm_shape(int cols, int w) {
  const int n = (cols + w - 1) / w;
  auto items = [&](int tpr) { int i = 1; while (i * tpr < n) i *= 2; return i; };
  if (n <= 16) return {16, 1};
  if (n <= 32) return {32, 1};
  if (n <= 256) return {64, items(64)};
  if (n <= 256 * (w == 1 ? 8 : 4)) return {256, items(256)};
  return {1024, items(1024)};
}

int norm_rows_per_block(int tpr) { return tpr > NORM_THREADS ? 1 : NORM_THREADS / tpr; }

template <typename T, int W, int ITEMS, int TPR>
void run_norm(const NormArgs& a, bool backward, int blocks, hipStream_t s) {
  constexpr int THREADS = TPR > NORM_THREADS ? TPR : NORM_THREADS;
  if (backward)
    hipLaunchKernelGGL((layer_norm_backward_kernel<T, W, ITEMS, TPR>), dim3(blocks), dim3(THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((layer_norm_kernel<T, W, ITEMS, TPR>), dim3(blocks), dim3(THREADS), 0, s, a);
}

template <typename T, int W>
bool dispatch_norm(const NormArgs& a, bool backward, int blocks, hipStream_t s) {
  const NormShape f = norm_shape(a.cols, W);
  switch (f.tpr * 32 + f.items) {
    case 16 * 32 + 1: run_norm<T, W, 1, 16>(a, backward, blocks, s); return true;
    case 32 * 32 + 1: run_norm<T, W, 1, 32>(a, backward, blocks, s); return true;
    case 64 * 32 + 1: run_norm<T, W, 1, 64>(a, backward, blocks, s); return true;
    case 64 * 32 + 2: run_norm<T, W, 2, 64>(a, backward, blocks, s); return true;
    case 64 * 32 + 4: run_norm<T, W, 4, 64>(a, backward, blocks, s); return true;
    case 256 * 32 + 2: run_norm<T, W, 2, 256>(a, backward, blocks, s); return true;
    case 256 * 32 + 4: run_norm<T, W, 4, 256>(a, backward, blocks, s); return true;
    case 1024 * 32 + 2: run_norm<T, W, 2, 1024>(a, backward, blocks, s); return true;
    case 1024 * 32 + 4: run_norm<T, W, 4, 1024>(a, backward, blocks, s); return true;
    default: break;
  }
  if constexpr (W == 1) {
    switch (f.tpr * 32 + f.items) {
      case 256 * 32 + 8: run_norm<T, W, 8, 256>(a, backward, blocks, s); return true;
      case 1024 * 32 + 8: run_norm<T, W, 8, 1024>(a, backward, blocks, s); return true;
      case 1024 * 32 + 16: run_norm<T, W, 16, 1024>(a, backward, blocks, s); return true;
      default: break;
    }
  }
  return false;
}

// Loads of 16 bytes where every row of every matrix starts at a multiple of them and the columns are whole loads.
bool norm_wide(const NormArgs& a, int size) {
  const int w = 16 / size;
  auto fits = [&](const void* p, int64_t ld) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % w == 0); };
  return a.cols % w == 0 && fits(a.x, a.ldx) && fits(a.y, a.ldy) && fits(a.dy, a.lddy) && fits(a.dx, a.lddx);
}

}  // namespace

int norm_backward_blocks(int64_t rows) {
  const int64_t all = (rows + 15) / 16;
  return (int)(all < 1 ? 1 : all > NORM_MAX_BLOCKS ? NORM_MAX_BLOCKS : all);
}

hipError_t launch_layer_norm(const NormArgs& a, int dtype, bool backward, hipStream_t stream) {
  const int size = dtype == RSLX_F32 ? 4 : 2;
  const bool wide = norm_wide(a, size);
  const NormShape f = norm_shape(a.cols, wide ? 16 / size : 1);
  const int per = norm_rows_per_block(f.tpr);
  const double n = (double)a.rows * a.cols;
  if (a.rows > 0 || backward) {
    TraceScope trace(stream, backward ? "layer_norm_backward" : "layer_norm", (backward ? 12 : 8) * n, (backward ? 3 : 2) * n * size);
    const int64_t sets = (a.rows + per - 1) / per;
    const int blocks = backward ? norm_backward_blocks(a.rows) : (int)(sets < NORM_MAX_FORWARD ? sets : NORM_MAX_FORWARD);
    bool ok;
    if (dtype == RSLX_F32)
      ok = wide ? dispatch_norm<float, 4>(a, backward, blocks, stream) : dispatch_norm<float, 1>(a, backward, blocks, stream);
    else if (dtype == RSLX_BF16)
      ok = wide ? dispatch_norm<bf16_t, 8>(a, backward, blocks, stream) : dispatch_norm<bf16_t, 1>(a, backward, blocks, stream);
    else
      ok = wide ? dispatch_norm<__half, 8>(a, backward, blocks, stream) : dispatch_norm<__half, 1>(a, backward, blocks, stream);
    if (!ok) return hipErrorInvalidValue;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (backward && a.partials) {
    const int blocks = norm_backward_blocks(a.rows);
    TraceScope trace(stream, "layer_norm_fold", 2.0 * blocks * a.cols, 8.0 * blocks * a.cols);
    hipLaunchKernelGGL(norm_fold_kernel, dim3((a.cols + 15) / 16, 2), dim3(256), 0, stream, a.partials, blocks, a.cols, a.dweight, a.dbias);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace rslx
