// Gated linear recurrence, gfx950.
//
//   f = sigmoid(g),  h_t = f_t keep_{t-1} h_{t-1} + (1 - f_t) x_t
//   d_t = dh_t + keep_t f_{t+1} d_{t+1},  dx = (1 - f) d,  dg = f (1 - f) d (keep_{t-1} h_{t-1} - x)
#include "memory.h"
#include "typed.h"

namespace rslx {

namespace {

constexpr int REC_THREADS = 256;

// sigmoid(g) and 1 - sigmoid(g), each with its own digits: one is e / (1 + e), the other 1 / (1 + e), of e = exp(-|g|) <= 1.
__device__ __forceinline__ void gate(float g, float& f, float& rest) {
  const float e = expf(-fabsf(g)), high = 1.f / (1.f + e), low = e * high;
  f = g >= 0.f ? high : low;
  rest = g >= 0.f ? low : high;
}

template <typename T> __device__ __forceinline__ T* row_of(const RecMatrix& m, int64_t t, int64_t n) {
  return static_cast<T*>(m.p) + t * m.step + n * m.seq;
}

template <typename T, bool BACKWARD>
__global__ __launch_bounds__(REC_THREADS) void recurrence_kernel(RecArgs a) {
  const int64_t c = (int64_t)blockIdx.x * REC_THREADS + threadIdx.x;
  if (c >= (int64_t)a.N * a.D) return;
  const int n = (int)(c / a.D), d = (int)(c % a.D);
  int len = a.T;
  if (a.lengths) {
    len = a.lengths[n];
    len = len < 0 ? 0 : len > a.T ? a.T : len;
  }
  float h = a.s0 ? a.s0[c] : 0.f;
  for (int64_t t = 0; t < len; ++t) {
    float f, rest;
    gate(to_float(row_of<T>(a.g, t, n)[d]), f, rest);
    if (BACKWARD) a.entered[t * a.N * a.D + c] = h;
    h = f * h + rest * to_float(row_of<T>(a.x, t, n)[d]);
    if (!BACKWARD) row_of<T>(a.h, t, n)[d] = from_float<T>(h);
    if (a.dones && a.dones[t * a.N + n]) h = 0.f;
  }
  if (!BACKWARD) {
    for (int64_t t = len; t < a.T; ++t) row_of<T>(a.h, t, n)[d] = from_float<T>(0.f);
    if (a.s_last) a.s_last[c] = h;
    return;
  }
  for (int64_t t = len; t < a.T; ++t) row_of<T>(a.dx, t, n)[d] = row_of<T>(a.dg, t, n)[d] = from_float<T>(0.f);
  float down = a.ds_last ? a.ds_last[c] : 0.f;
  for (int64_t t = len - 1; t >= 0; --t) {
    float f, rest;
    gate(to_float(row_of<T>(a.g, t, n)[d]), f, rest);
    if (a.dones && a.dones[t * a.N + n]) down = 0.f;
    down += to_float(row_of<T>(a.dh, t, n)[d]);
    row_of<T>(a.dx, t, n)[d] = from_float<T>(rest * down);
    row_of<T>(a.dg, t, n)[d] = from_float<T>(f * rest * down * (a.entered[t * a.N * a.D + c] - to_float(row_of<T>(a.x, t, n)[d])));
    down *= f;
  }
  if (a.ds0) a.ds0[c] = down;
}

template <typename T>
__global__ __launch_bounds__(REC_THREADS) void recurrence_step_kernel(RecArgs a) {
  const int64_t c = (int64_t)blockIdx.x * REC_THREADS + threadIdx.x;
  if (c >= (int64_t)a.N * a.D) return;
  const int n = (int)(c / a.D), d = (int)(c % a.D);
  float f, rest;
  gate(to_float(row_of<T>(a.g, 0, n)[d]), f, rest);
  const float s = a.s0 && !(a.dones && a.dones[n]) ? a.s0[c] : 0.f;
  const float h = f * s + rest * to_float(row_of<T>(a.x, 0, n)[d]);
  a.s_last[c] = h;
  row_of<T>(a.h, 0, n)[d] = from_float<T>(h);
}

}  // namespace

void plan_recurrence(host::Carver& c, RecArgs& a, int, bool backward) {
  if (backward) a.entered = c.take<float>((size_t)a.T * a.N * a.D);
}

hipError_t launch_recurrence(const RecArgs& a, int dtype, bool backward, hipStream_t stream) {
  const double n = (double)a.T * a.N * a.D, size = dtype == RSLX_F32 ? 4 : 2;
  TraceScope trace(stream, backward ? "recurrence_backward" : "recurrence", (backward ? 25 : 10) * n, (backward ? 5 : 3) * n * size);
  const dim3 grid((unsigned)(((int64_t)a.N * a.D + REC_THREADS - 1) / REC_THREADS)), block(REC_THREADS);
#define RUN(T)                                                                                            \
  do {                                                                                                    \
    if (backward) hipLaunchKernelGGL((recurrence_kernel<T, true>), grid, block, 0, stream, a);            \
    else hipLaunchKernelGGL((recurrence_kernel<T, false>), grid, block, 0, stream, a);                    \
  } while (0)
  if (dtype == RSLX_F32) RUN(float);
  else if (dtype == RSLX_BF16) RUN(bf16_t);
  else RUN(__half);
#undef RUN
  return hipGetLastError();
}

hipError_t launch_recurrence_step(const RecArgs& a, int dtype, hipStream_t stream) {
  const double n = (double)a.N * a.D, size = dtype == RSLX_F32 ? 4 : 2;
  TraceScope trace(stream, "recurrence_step", 10 * n, (3 * size + 8) * n);
  const dim3 grid((unsigned)(((int64_t)a.N * a.D + REC_THREADS - 1) / REC_THREADS)), block(REC_THREADS);
  if (dtype == RSLX_F32) hipLaunchKernelGGL((recurrence_step_kernel<float>), grid, block, 0, stream, a);
  else if (dtype == RSLX_BF16) hipLaunchKernelGGL((recurrence_step_kernel<bf16_t>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((recurrence_step_kernel<__half>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace rslx
