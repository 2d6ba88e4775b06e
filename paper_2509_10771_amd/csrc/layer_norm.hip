// Layer norm over the rows of a matrix, forward and backward, gfx950.
//
//   m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps),  y = (x - m) r w + b
//   g = dy w,  h = (x - m) r:   dx = r (g - mean g - h mean(g h)),   dw = sum over rows dy h,   db = sum over rows dy
//
// Both are bound by memory: a row is read once into registers (16 bytes a load, ITEMS loads a lane), everything that needs the whole row
// happens there, and the result is written once.  The variance is that of the centred values, so that rows far from zero keep their digits;
// what rounding left of the mean shows in the sum of the same values, and is taken off too.  TPR lanes share a row: part of a wavefront, a
// wavefront, or a workgroup where one wavefront's registers would not hold it.  Sums are fp32: a lane's values in order, then a fixed tree.
//
// What it takes to reach the memory's rate is rows in flight: a workgroup goes round the rows with the next one's loads ahead of this one's
// sums, and keeps the weights in registers.  98304 rows of 512 in bf16: 41.8 us = 4.8 TB/s (a workgroup for every four rows, weights loaded behind the
// sums: 53.6); gradients of 8192 rows of 4096 in bf16: 40.6 us = 5.0 TB/s (66.4) and 6.6 for the fold of the parameters'; of 24576 rows
// of 235 in fp32, which start anywhere: 16.6 us = 4.2 TB/s (value by value 27.6, of 512 workgroups instead of 1024 21.8) and 3.8.
#include "norm_rows.h"

namespace rslx {

namespace {

constexpr int NORM_MAX_FORWARD = 2048;        // workgroups of a forward launch: eight for each CU; more rows go round

// A workgroup takes every gridDim.x-th set of rows; the next row's values are on their way while this one is reduced, and the weights stay in
// registers.
template <typename T, int W, int ITEMS, int TPR, bool WHOLE>
__global__ __launch_bounds__(THREADS_OF<TPR>) void layer_norm_kernel(NormArgs a) {
  constexpr int ROWS = THREADS_OF<TPR> / TPR;
  __shared__ float lds[2][2 * (TPR > 64 ? TPR / 64 : 1)];
  const int lane = threadIdx.x % TPR;
  const float n = (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  Pack<T, W> in[ITEMS];
  auto load = [&](int64_t r) {
    if (r < a.rows)
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) load_piece<T, W, WHOLE>(in[i], static_cast<const T*>(a.x) + r * a.ldx, (i * TPR + lane) * W, a.cols);
  };
  load(row);
  Pack<float, W> w[ITEMS], b[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      w[i].v[k] = 1.f;
      b[i].v[k] = 0.f;
    }
    if (a.weight) load_piece<float, W, WHOLE>(w[i], a.weight, (i * TPR + lane) * W, a.cols);
    if (a.bias) load_piece<float, W, WHOLE>(b[i], a.bias, (i * TPR + lane) * W, a.cols);
  }
  // (TPR <= 64: lanes leave the loop in whole rows, and the shuffles stay inside a row; above, the workgroup has one row)
  for (; row < a.rows; row += stride) {
    float f[ITEMS * W], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        f[i * W + k] = in_row<W, WHOLE>((i * TPR + lane) * W, k, a.cols) ? to_float(in[i].v[k]) : 0.f;
        s[0] += f[i * W + k];
      }
    load(row + stride);
    row_sum<TPR, 1>(s, lds[0]);
    const float near = s[0] / n;
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        f[i * W + k] = in_row<W, WHOLE>((i * TPR + lane) * W, k, a.cols) ? f[i * W + k] - near : 0.f;
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
      Pack<T, W> out;
#pragma unroll
      for (int k = 0; k < W; ++k) out.v[k] = from_float<T>((f[i * W + k] - rest) * rstd * w[i].v[k] + b[i].v[k]);
      store_piece<T, W, WHOLE>(out, y, (i * TPR + lane) * W, a.cols);
    }
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// The backward pass goes round the rows in the same way, so that a lane's columns stay the same and their gradients of weight and bias
// add up in its registers; what the workgroup holds in the end is one row of partial sums, which norm_fold_kernel adds up in a fixed order
// (no atomics: the same inputs give the same bits).
template <typename T, int W, int ITEMS, int TPR, bool WHOLE>
__global__ __launch_bounds__(THREADS_OF<TPR>) void layer_norm_backward_kernel(NormArgs a) {
  constexpr int ROWS = THREADS_OF<TPR> / TPR;
  __shared__ float lds[2][2 * (TPR > 64 ? TPR / 64 : 1)];
  __shared__ float join[ROWS > 1 ? (ROWS - 1) * TPR * ITEMS * W : 1];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + sub;
  Pack<T, W> px[ITEMS], pd[ITEMS];
  float mean = 0.f, rstd = 0.f;
  auto load = [&](int64_t r) {
    if (r < a.rows) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        load_piece<T, W, WHOLE>(px[i], static_cast<const T*>(a.x) + r * a.ldx, (i * TPR + lane) * W, a.cols);
        load_piece<T, W, WHOLE>(pd[i], static_cast<const T*>(a.dy) + r * a.lddy, (i * TPR + lane) * W, a.cols);
      }
      mean = a.mean[r];
      rstd = a.rstd[r];
    }
  };
  load(row);
  Pack<float, W> w[ITEMS];
  // 1024 lanes have 128 registers each: with 16 values a lane the gradients' sums lie in LDS, where nobody else reads or writes a lane's.  With
  // them in registers the compiler kept others on the stack, and stored some inside branches that only some lanes take (2048 rows of 16384
  // in fp32 112 us both launches, in bf16 76; on the stack 155 and 105).
  constexpr bool IN_LDS = TPR == 1024 && ITEMS * W > 8;
  __shared__ __attribute__((aligned(16))) float sums[IN_LDS ? 2 * ITEMS * W * TPR : 4];
  float dw[ITEMS * W], db[ITEMS * W];
  auto sum_at = [&](int pass, int x) -> float4& { return *reinterpret_cast<float4*>(sums + ((pass * ITEMS * W + x) / 4 * TPR + lane) * 4); };
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      w[i].v[k] = 1.f;
      dw[i * W + k] = db[i * W + k] = 0.f;
      if (IN_LDS && k % 4 == 0) sum_at(0, i * W + k) = sum_at(1, i * W + k) = float4{0.f, 0.f, 0.f, 0.f};
    }
    if (a.weight) load_piece<float, W, WHOLE>(w[i], a.weight, (i * TPR + lane) * W, a.cols);
  }
  for (int turn = 0; row < a.rows; row += stride, turn ^= 1) {
    float s[2] = {0.f, 0.f}, h[ITEMS * W], g[ITEMS * W];
    const float scale = rstd;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const int x = i * W + k;
        const bool here = in_row<W, WHOLE>((i * TPR + lane) * W, k, a.cols);
        const float d = here ? to_float(pd[i].v[k]) : 0.f;
        h[x] = here ? (to_float(px[i].v[k]) - mean) * rstd : 0.f;
        g[x] = here ? d * w[i].v[k] : 0.f;
        if constexpr (!IN_LDS) {
          dw[x] += d * h[x];
          db[x] += d;
        } else {
          dw[x % 4] = d * h[x];
          db[x % 4] = d;
          if (x % 4 == 3) {
            float4 &to_w = sum_at(0, x), &to_b = sum_at(1, x);
            to_w = float4{to_w.x + dw[0], to_w.y + dw[1], to_w.z + dw[2], to_w.w + dw[3]};
            to_b = float4{to_b.x + db[0], to_b.y + db[1], to_b.z + db[2], to_b.w + db[3]};
          }
        }
        s[0] += g[x];
        s[1] += g[x] * h[x];
      }
    load(row + stride);
    if (a.dx) {
      row_sum<TPR, 2>(s, lds[turn]);
      const float mg = s[0] * inv, mgh = s[1] * inv;
      T* dx = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Pack<T, W> out;
#pragma unroll
        for (int k = 0; k < W; ++k) out.v[k] = from_float<T>(scale * (g[i * W + k] - mg - h[i * W + k] * mgh));
        store_piece<T, W, WHOLE>(out, dx, (i * TPR + lane) * W, a.cols);
      }
    }
  }
  if (!a.partials) return;
  // the workgroup's sets of lanes, first weight, then bias
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    float(&v)[ITEMS * W] = pass == 0 ? dw : db;
    if constexpr (IN_LDS)
#pragma unroll
      for (int x = 0; x < ITEMS * W; x += 4) {
        const float4 f = sum_at(pass, x);
        v[x] = f.x;
        v[x + 1] = f.y;
        v[x + 2] = f.z;
        v[x + 3] = f.w;
      }
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
        Pack<float, W> out;
#pragma unroll
        for (int k = 0; k < W; ++k) out.v[k] = v[i * W + k];
        store_piece<float, W, WHOLE>(out, to, (i * TPR + lane) * W, a.cols);
      }
    }
  }
}

template <typename T, int W, int ITEMS, int TPR, bool WHOLE>
void run_norm(const NormArgs& a, bool backward, int blocks, hipStream_t s) {
  if (backward)
    hipLaunchKernelGGL((layer_norm_backward_kernel<T, W, ITEMS, TPR, WHOLE>), dim3(blocks), dim3(THREADS_OF<TPR>), 0, s, a);
  else
    hipLaunchKernelGGL((layer_norm_kernel<T, W, ITEMS, TPR, WHOLE>), dim3(blocks), dim3(THREADS_OF<TPR>), 0, s, a);
}

template <typename T, bool WHOLE>
void dispatch_norm(const NormArgs& a, bool backward, int blocks, hipStream_t s) {
  constexpr int W = 16 / (int)sizeof(T);
  const NormShape f = norm_shape(a.cols, W);
  switch (f.tpr * 32 + f.items) {
    case 16 * 32 + 1: run_norm<T, W, 1, 16, WHOLE>(a, backward, blocks, s); break;
    case 32 * 32 + 1: run_norm<T, W, 1, 32, WHOLE>(a, backward, blocks, s); break;
    case 64 * 32 + 1: run_norm<T, W, 1, 64, WHOLE>(a, backward, blocks, s); break;
    case 64 * 32 + 2: run_norm<T, W, 2, 64, WHOLE>(a, backward, blocks, s); break;
    case 256 * 32 + 1: run_norm<T, W, 1, 256, WHOLE>(a, backward, blocks, s); break;
    case 256 * 32 + 2: run_norm<T, W, 2, 256, WHOLE>(a, backward, blocks, s); break;
    case 512 * 32 + 2: run_norm<T, W, 2, 512, WHOLE>(a, backward, blocks, s); break;
    case 1024 * 32 + 2: run_norm<T, W, 2, 1024, WHOLE>(a, backward, blocks, s); break;
    default:
      if constexpr (W == 4) run_norm<T, W, 4, 1024, WHOLE>(a, backward, blocks, s);      // (16384 values are 2048 loads of eight)
      break;
  }
}

// Whether every row of every matrix is a number of whole, aligned loads.
bool norm_whole(const NormArgs& a, int size) {
  const int w = 16 / size;
  auto fits = [&](const void* p, int64_t ld) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % w == 0); };
  return a.cols % w == 0 && fits(a.x, a.ldx) && fits(a.y, a.ldy) && fits(a.dy, a.lddy) && fits(a.dx, a.lddx);
}

}  // namespace

// Workgroups of a backward launch.  Each leaves 2 cols sums behind, which are written and read once more: four sets of rows each where rows are
// many, half as many workgroups where they are long; where rows are few, one set each up to a workgroup per CU (595 rows of 6229 in fp32: 22 us
// both launches, 38 workgroups of 16 rows 41).
int norm_backward_blocks(int64_t rows, int cols) {
  const int64_t per = norm_rows_per_block(norm_shape(cols, 4).tpr), sets = rows / per + (rows % per != 0);
  const int64_t most = cols <= 512 ? NORM_MAX_BLOCKS : NORM_MAX_BLOCKS / 2;
  const int64_t many = sets / 4 < most ? sets / 4 : most, few = sets < 256 ? sets : 256;
  const int64_t blocks = many > few ? many : few;
  return (int)(blocks < 1 ? 1 : blocks);
}

hipError_t launch_layer_norm(const NormArgs& a, int dtype, bool backward, hipStream_t stream) {
  const int size = dtype == RSLX_F32 ? 4 : 2;
  const bool whole = norm_whole(a, size);
  const NormShape f = norm_shape(a.cols, 16 / size);
  const int per = norm_rows_per_block(f.tpr);
  const double n = (double)a.rows * a.cols;
  if (a.rows > 0 || backward) {
    TraceScope trace(stream, backward ? "layer_norm_backward" : "layer_norm", (backward ? 12 : 8) * n, (backward ? 3 : 2) * n * size);
    const int64_t sets = a.rows / per + (a.rows % per != 0);
    const int blocks = backward ? norm_backward_blocks(a.rows, a.cols) : (int)(sets < NORM_MAX_FORWARD ? sets : NORM_MAX_FORWARD);
    if (dtype == RSLX_F32)
      whole ? dispatch_norm<float, true>(a, backward, blocks, stream) : dispatch_norm<float, false>(a, backward, blocks, stream);
    else if (dtype == RSLX_BF16)
      whole ? dispatch_norm<bf16_t, true>(a, backward, blocks, stream) : dispatch_norm<bf16_t, false>(a, backward, blocks, stream);
    else
      whole ? dispatch_norm<__half, true>(a, backward, blocks, stream) : dispatch_norm<__half, false>(a, backward, blocks, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (backward && a.partials) {
    const int blocks = norm_backward_blocks(a.rows, a.cols);
    TraceScope trace(stream, "layer_norm_fold", 2.0 * blocks * a.cols, 8.0 * blocks * a.cols);
    hipLaunchKernelGGL(norm_fold_kernel, dim3((a.cols + 15) / 16, 2), dim3(16 * FOLD_LANES), 0, stream, a.partials, blocks, a.cols, a.dweight, a.dbias);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace rslx
