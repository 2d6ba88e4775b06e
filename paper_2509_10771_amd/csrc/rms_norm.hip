// Root-mean-square norm over the rows of a matrix with the residual's addition, forward (in the inputs' type or in 8 bits) and backward, gfx950.
//
//   z = x + residual,  r = 1 / sqrt(mean z^2 + eps),  y = z r w;      8 bits: s = max |y| / 448,  y8 = y / s
//   h = z r,  k = dy w:   dx = dtotal + r (k - h mean(k h)),   dw = sum over rows dy h
//
// Bound by memory, and built like layer norm: a row is read once into the registers of the TPR lanes that share it, the next one is on its way while
// this one is reduced, results are written once.  Squares and products are summed in fp32: a lane's values in order, then a fixed tree.  98304 rows of 512 in bf16
// into bytes 66 us = 5.3 TB/s; gradients of 24576 rows of 235 in fp32, which start anywhere, 18 us = 5.1 TB/s and 4 for the fold of the weight's.
#include "memory.h"
#include "norm_rows.h"

namespace rslx {

namespace {

constexpr int RMS_MAX_FORWARD = 4096;         // workgroups of a forward launch: sixteen for each CU; more rows go round
constexpr float E4M3_MAX = 448.f;

// The largest of the TPR lanes' values, as the bits of numbers without a sign: a NaN's are above those of every number.
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* lds) {
  constexpr int IN_WAVE = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = IN_WAVE / 2; o > 0; o >>= 1) {
    const uint32_t u = __shfl_xor(v, o, 64);
    v = u > v ? u : v;
  }
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v = lds[w] > v ? lds[w] : v;
  }
  return v;
}

// Four values rounded to e4m3 (nearest even).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true);
}

// A lane's piece i of a row, W values from `at` on, of which those from `first` to `end` are its own.  Rows that start anywhere end with a piece that begins
// earlier, so that it is one load too: 16-bit values that come one by one (IN_PARTS) are each put together in a register, and waited for, with the next row on
// its way (98304 rows of 511 in bf16, to bytes: 80 us, in parts 95; their gradients 92 and 127; of 24576 of 999 in fp32 73 and 135).  The first half of a lane's
// pieces is inside the row (see norm_shape).
template <int W, int ITEMS, int TPR, bool WHOLE, bool IN_PARTS = false>
struct Span {
  int at, first, end;
  __device__ __forceinline__ Span(int i, int cols) : at((i * TPR + (int)threadIdx.x % TPR) * W), first(0), end(W) {
    if (i < ITEMS / 2) return;
    end = cols - at < W ? cols - at : W;
    if (!WHOLE && !IN_PARTS && cols >= W && end < W) {
      const int c = at;
      at = cols - W;
      first = c - at;
      end = W;
    }
  }
  __device__ __forceinline__ bool has(int k) const { return WHOLE ? end > 0 : k >= first && k < end; }
  template <typename T>
  __device__ __forceinline__ void load(Pack<T, W>& p, const T* row, int cols) const {
    if (WHOLE || IN_PARTS || cols < W) load_piece<T, W, WHOLE>(p, row, at, cols);
    else __builtin_memcpy(&p, row + at, sizeof p);
  }
  template <typename T>
  __device__ __forceinline__ void store(const Pack<T, W>& p, T* row, int cols, bool past) const {
    if (WHOLE || IN_PARTS || first == 0) {
      store_piece<T, W, WHOLE>(p, row, at, cols, past);
    } else {
#pragma unroll
      for (int k = 1; k < W; ++k)
        if (k >= first) row[at + k] = p.v[k];
    }
  }
};

template <typename T, int W, int ITEMS, int TPR, bool WHOLE, bool E4M3>
__global__ __launch_bounds__(THREADS_OF<TPR>) void rms_norm_kernel(RmsArgs a) {
  constexpr int ROWS = THREADS_OF<TPR> / TPR;
  typedef Span<W, ITEMS, TPR, WHOLE> Piece;
  __shared__ float lds[2][TPR > 64 ? TPR / 64 : 1];
  __shared__ uint32_t lds_max[TPR > 64 ? TPR / 64 : 1];
  const int lane = threadIdx.x % TPR;
  const float n = (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  Pack<T, W> px[ITEMS], pr[ITEMS];
  auto load = [&](int64_t r) {
    if (r < a.rows)
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Piece(i, a.cols).load(px[i], static_cast<const T*>(a.x) + r * a.ldx, a.cols);
        if (a.residual) Piece(i, a.cols).load(pr[i], static_cast<const T*>(a.residual) + r * a.ldr, a.cols);
      }
  };
  load(row);
  Pack<float, W> w[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int k = 0; k < W; ++k) w[i].v[k] = 1.f;
    if (a.weight) Piece(i, a.cols).load(w[i], a.weight, a.cols);
  }
  // (TPR <= 64: lanes leave the loop in whole rows, and the shuffles stay inside a row; above, the workgroup has one row)
  for (int turn = 0; row < a.rows; row += stride, turn ^= 1) {
    float f[ITEMS * W], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        float z = to_float(px[i].v[k]);
        if (a.residual) z += to_float(pr[i].v[k]);
        f[i * W + k] = Piece(i, a.cols).has(k) ? z : 0.f;
        s[0] += f[i * W + k] * f[i * W + k];
      }
    load(row + stride);
    if (a.total) {
      T* to = static_cast<T*>(a.total) + row * a.ldt;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Pack<T, W> out;
#pragma unroll
        for (int k = 0; k < W; ++k) out.v[k] = from_float<T>(f[i * W + k]);
        Piece(i, a.cols).store(out, to, a.cols, a.past);
      }
    }
    row_sum<TPR, 1>(s, lds[turn]);
    const float rstd = 1.f / sqrtf(s[0] / n + a.eps);
    if constexpr (!E4M3) {
      T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Pack<T, W> out;
#pragma unroll
        for (int k = 0; k < W; ++k) out.v[k] = from_float<T>(f[i * W + k] * rstd * w[i].v[k]);
        Piece(i, a.cols).store(out, y, a.cols, a.past);
      }
    } else {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          f[i * W + k] = Piece(i, a.cols).has(k) ? f[i * W + k] * rstd * w[i].v[k] : 0.f;
          const uint32_t bits = __float_as_uint(f[i * W + k]) & 0x7fffffffu;
          most = bits > most ? bits : most;
        }
      most = row_max<TPR>(most, lds_max);
      float scale = __uint_as_float(most) / E4M3_MAX;
      if (scale < 0x1p-126f) scale = 0x1p-126f;
      const float inv = 1.f / scale;
      uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.ldy;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Pack<uint8_t, W> out;
#pragma unroll
        for (int k = 0; k < W; k += 4) {
          const float* v = f + i * W + k;
          const uint32_t four = pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
          __builtin_memcpy(out.v + k, &four, 4);
        }
        Piece(i, a.cols).store(out, y, a.cols, a.past);
      }
      if (lane == 0) a.scales[row] = scale;
    }
    if (lane == 0 && a.rstd) a.rstd[row] = rstd;
  }
}

// A lane's columns stay the same from row to row, and their gradients of the weight add up in its registers; what the workgroup holds in the end is one
// row of partial sums, which norm_fold_kernel adds up in a fixed order.  1024 lanes have 128 registers each: with 16 values a lane the sums lie in
// LDS, where nobody else reads or writes a lane's, a row is not loaded ahead, and what is made of it is made twice (nothing is left on the stack that way).
template <typename T, int W, int ITEMS, int TPR, bool WHOLE>
__global__ __launch_bounds__(THREADS_OF<TPR>) void rms_norm_backward_kernel(RmsArgs a) {
  constexpr int ROWS = THREADS_OF<TPR> / TPR;
  constexpr bool LONG = TPR == 1024 && ITEMS * W > 8;
  // (LONG: no registers for more; fp32 rows of several pieces a lane: 98304 rows of 511 157 us, as one load 167)
  typedef Span<W, ITEMS, TPR, WHOLE, LONG || (sizeof(T) == 4 && ITEMS > 1)> Piece;
  __shared__ float lds[2][TPR > 64 ? TPR / 64 : 1];
  __shared__ float join[ROWS > 1 ? (ROWS - 1) * TPR * ITEMS * W : 1];
  __shared__ __attribute__((aligned(16))) float sums[LONG ? ITEMS * W * TPR : 4];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv = 1.f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + sub;
  auto sum_at = [&](int x) -> float4& { return *reinterpret_cast<float4*>(sums + (x / 4 * TPR + lane) * 4); };
  Pack<T, W> px[ITEMS], pd[ITEMS], pt[ITEMS];
  float rstd = 0.f;
  auto load = [&](int64_t r) {
    if (r < a.rows) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Piece(i, a.cols).load(px[i], static_cast<const T*>(a.x) + r * a.ldx, a.cols);
        Piece(i, a.cols).load(pd[i], static_cast<const T*>(a.dy) + r * a.lddy, a.cols);
        if (!LONG && a.y && a.residual) Piece(i, a.cols).load(pt[i], static_cast<const T*>(a.residual) + r * a.ldr, a.cols);
      }
      rstd = a.rstd[r];
    }
  };
  if (!LONG) load(row);
  Pack<float, W> w[ITEMS];
  float dw[LONG ? 4 : ITEMS * W];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      w[i].v[k] = 1.f;
      if constexpr (!LONG) dw[i * W + k] = 0.f;
      else if (k % 4 == 0) sum_at(i * W + k) = float4{0.f, 0.f, 0.f, 0.f};
    }
    if (a.weight) Piece(i, a.cols).load(w[i], a.weight, a.cols);
  }
  for (int turn = 0; row < a.rows; row += stride, turn ^= 1) {
    if (LONG) load(row);
    float s[1] = {0.f}, h[LONG ? 1 : ITEMS * W], g[LONG ? 1 : ITEMS * W];
    const float scale = rstd;
    Pack<T, W> t[LONG ? 1 : ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if constexpr (!LONG) t[i] = pt[i];
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const int x = i * W + k;
        const bool here = Piece(i, a.cols).has(k);
        const float d = here ? to_float(pd[i].v[k]) : 0.f, hx = here ? to_float(px[i].v[k]) * scale : 0.f, gx = here ? d * w[i].v[k] : 0.f;
        s[0] += gx * hx;
        if constexpr (!LONG) {
          h[x] = hx;
          g[x] = gx;
          dw[x] += d * hx;
        } else {
          dw[x % 4] = d * hx;
          if (x % 4 == 3) {
            float4& to = sum_at(x);
            to = float4{to.x + dw[0], to.y + dw[1], to.z + dw[2], to.w + dw[3]};
          }
        }
      }
    }
    if (!LONG) load(row + stride);
    if (a.y) {
      row_sum<TPR, 1>(s, lds[turn]);
      const float mean = s[0] * inv;
      T* dx = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        Pack<T, W> out, late;
        if (LONG && a.residual) Piece(i, a.cols).load(late, static_cast<const T*>(a.residual) + row * a.ldr, a.cols);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          float v;
          if constexpr (!LONG) v = scale * (g[i * W + k] - h[i * W + k] * mean);
          else v = scale * (to_float(pd[i].v[k]) * w[i].v[k] - to_float(px[i].v[k]) * scale * mean);
          if (a.residual) v += to_float(LONG ? late.v[k] : t[LONG ? 0 : i].v[k]);
          out.v[k] = from_float<T>(v);
        }
        Piece(i, a.cols).store(out, dx, a.cols, LONG || a.past);      // (LONG: no registers for both)
      }
    }
  }
  if (!a.partials) return;
  if constexpr (ROWS > 1) {
    if (sub > 0)
#pragma unroll
      for (int i = 0; i < ITEMS * W; ++i) join[((sub - 1) * ITEMS * W + i) * TPR + lane] = dw[i];
    __syncthreads();
    if (sub == 0)
      for (int r = 0; r < ROWS - 1; ++r)
#pragma unroll
        for (int i = 0; i < ITEMS * W; ++i) dw[i] += join[(r * ITEMS * W + i) * TPR + lane];
  }
  if (sub == 0) {
    float* to = a.partials + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      Pack<float, W> out;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        if constexpr (LONG) {
          if (k % 4 == 0) {
            const float4 f = sum_at(i * W + k);
            out.v[k] = f.x;
            out.v[k + 1] = f.y;
            out.v[k + 2] = f.z;
            out.v[k + 3] = f.w;
          }
        } else {
          out.v[k] = dw[i * W + k];
        }
      }
      Piece(i, a.cols).store(out, to, a.cols, false);
    }
  }
}

enum RmsKind { RMS_FORWARD, RMS_FORWARD_E4M3, RMS_BACKWARD };

template <typename T, int W, int ITEMS, int TPR, bool WHOLE>
void run_rms(const RmsArgs& a, RmsKind kind, int blocks, hipStream_t s) {
  const dim3 grid(blocks), block(THREADS_OF<TPR>);
  if (kind == RMS_FORWARD) hipLaunchKernelGGL((rms_norm_kernel<T, W, ITEMS, TPR, WHOLE, false>), grid, block, 0, s, a);
  else if (kind == RMS_FORWARD_E4M3) hipLaunchKernelGGL((rms_norm_kernel<T, W, ITEMS, TPR, WHOLE, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rms_norm_backward_kernel<T, W, ITEMS, TPR, WHOLE>), grid, block, 0, s, a);
}

template <typename T, bool WHOLE>
void dispatch_rms(const RmsArgs& a, RmsKind kind, int blocks, hipStream_t s) {
  constexpr int W = 16 / (int)sizeof(T);
  const NormShape f = norm_shape(a.cols, W);
  switch (f.tpr * 32 + f.items) {
    case 16 * 32 + 1: run_rms<T, W, 1, 16, WHOLE>(a, kind, blocks, s); break;
    case 32 * 32 + 1: run_rms<T, W, 1, 32, WHOLE>(a, kind, blocks, s); break;
    case 64 * 32 + 1: run_rms<T, W, 1, 64, WHOLE>(a, kind, blocks, s); break;
    case 64 * 32 + 2: run_rms<T, W, 2, 64, WHOLE>(a, kind, blocks, s); break;
    case 256 * 32 + 1: run_rms<T, W, 1, 256, WHOLE>(a, kind, blocks, s); break;
    case 256 * 32 + 2: run_rms<T, W, 2, 256, WHOLE>(a, kind, blocks, s); break;
    case 512 * 32 + 2: run_rms<T, W, 2, 512, WHOLE>(a, kind, blocks, s); break;
    case 1024 * 32 + 2: run_rms<T, W, 2, 1024, WHOLE>(a, kind, blocks, s); break;
    default:
      if constexpr (W == 4) run_rms<T, W, 4, 1024, WHOLE>(a, kind, blocks, s);      // (16384 values are 2048 loads of eight)
      break;
  }
}

template <typename T>
void run_type(const RmsArgs& a, RmsKind kind, int blocks, hipStream_t s) {
  // whether every row of every matrix is a number of whole, aligned loads
  constexpr int W = 16 / (int)sizeof(T);
  auto fits = [&](const void* p, int64_t ld, int bytes) { return !p || ((reinterpret_cast<uintptr_t>(p) % bytes) == 0 && ld % W == 0); };
  const bool whole = a.cols % W == 0 && fits(a.x, a.ldx, 16) && fits(a.residual, a.ldr, 16) && fits(a.dy, a.lddy, 16) && fits(a.total, a.ldt, 16) &&
                     fits(a.y, a.ldy, kind == RMS_FORWARD_E4M3 ? W : 16);
  whole ? dispatch_rms<T, true>(a, kind, blocks, s) : dispatch_rms<T, false>(a, kind, blocks, s);
}

// Outputs of 16 MB and more, which the dies' L2 could not keep beside the inputs, go past the caches.  Rows of 512 in bf16: 98304 74.6 us, through them 78.4, into bytes
// 68.0 and 70.0, gradients 80.8 and 82.7; 16384 12.1 and 13.0, 11.9 and 12.3, 18.1 and 18.7; 8192 (8 to 17 MB) no difference, nor for gradients of 24576 of 235 in fp32.
constexpr double PAST_BYTES = 16 << 20;

hipError_t run(RmsArgs a, int dtype, RmsKind kind, int blocks, hipStream_t s) {
  const double size = dtype == RSLX_F32 ? 4 : 2, n = (double)a.rows * a.cols;
  a.past = (a.total ? n * size : 0) + (a.y ? n * (kind == RMS_FORWARD_E4M3 ? 1 : size) : 0) >= PAST_BYTES;
  if (dtype == RSLX_F32) run_type<float>(a, kind, blocks, s);
  else if (dtype == RSLX_BF16) run_type<bf16_t>(a, kind, blocks, s);
  else run_type<__half>(a, kind, blocks, s);
  return hipGetLastError();
}

int64_t sets_of(int64_t rows, int cols, int w) {
  const int64_t per = norm_rows_per_block(norm_shape(cols, w).tpr);
  return rows / per + (rows % per != 0);
}

}  // namespace

// Workgroups of a backward launch: as for layer norm.
int rms_backward_blocks(int64_t rows, int cols) {
  const int64_t sets = sets_of(rows, cols, 4);
  const int64_t most = cols <= 512 ? RMS_MAX_BLOCKS : RMS_MAX_BLOCKS / 2;
  const int64_t many = sets / 4 < most ? sets / 4 : most, few = sets < 256 ? sets : 256;
  const int64_t blocks = many > few ? many : few;
  return (int)(blocks < 1 ? 1 : blocks);
}

hipError_t launch_rms_norm(const RmsArgs& a, int dtype, bool e4m3, hipStream_t stream) {
  const double n = (double)a.rows * a.cols, size = dtype == RSLX_F32 ? 4 : 2;
  TraceScope trace(stream, e4m3 ? "rms_norm_e4m3" : "rms_norm", 6 * n, n * (size * (1 + (a.residual != nullptr) + (a.total != nullptr)) + (e4m3 ? 1 : size)));
  const int64_t sets = sets_of(a.rows, a.cols, dtype == RSLX_F32 ? 4 : 8);
  return run(a, dtype, e4m3 ? RMS_FORWARD_E4M3 : RMS_FORWARD, (int)(sets < RMS_MAX_FORWARD ? sets : RMS_MAX_FORWARD), stream);
}

hipError_t launch_rms_norm_backward(const RmsArgs& a, int dtype, hipStream_t stream) {
  const double n = (double)a.rows * a.cols, size = dtype == RSLX_F32 ? 4 : 2;
  const int blocks = rms_backward_blocks(a.rows, a.cols);
  {
    TraceScope trace(stream, "rms_norm_backward", 10 * n, n * size * (2 + (a.residual != nullptr) + (a.y != nullptr)));
    const hipError_t e = run(a, dtype, RMS_BACKWARD, blocks, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.partials) return hipSuccess;
  TraceScope trace(stream, "rms_norm_fold", (double)blocks * a.cols, 4.0 * blocks * a.cols);
  hipLaunchKernelGGL(norm_fold_kernel, dim3((a.cols + 15) / 16, 1), dim3(16 * FOLD_LANES), 0, stream, a.partials, blocks, a.cols, a.dweight, nullptr);
  return hipGetLastError();
}

}  // namespace rslx
