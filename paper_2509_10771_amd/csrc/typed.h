// Activations of the sequence operators (linear attention, layer norm) come in three types; arithmetic is fp32, but for the 16-bit walks' products,
// which linear_attention.hip describes.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rslx {

struct bf16_t { uint16_t bits; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16_t x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

// Rounded to nearest, ties to even; a NaN stays one.
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t from_float<bf16_t>(float x) {
  const __bf16 b = (__bf16)x;
  return {__builtin_bit_cast(uint16_t, b)};
}
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half(x); }

// N consecutive values, moved in accesses of up to 16 bytes.
template <typename T, int N> struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack { T v[N]; };

// W values of a row from column c on; WHOLE: rows are whole, aligned loads.  Otherwise rows start anywhere (the load is as wide, global memory
// takes any address) and the last one may be shorter: its values come one by one.
template <typename T, int W, bool WHOLE>
__device__ __forceinline__ void load_piece(Pack<T, W>& p, const T* row, int c, int cols) {
  if constexpr (WHOLE) {
    if (c < cols) p = *reinterpret_cast<const Pack<T, W>*>(row + c);
  } else if (c + W <= cols) {
    __builtin_memcpy(&p, row + c, sizeof p);
  } else {
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
      if (c + k < cols) p.v[k] = row[c + k];
  }
}
template <typename T, int W, bool WHOLE>
__device__ __forceinline__ void store_piece(const Pack<T, W>& p, T* row, int c, int cols) {
  if constexpr (WHOLE) {
    if (c < cols) *reinterpret_cast<Pack<T, W>*>(row + c) = p;
  } else if (c + W <= cols) {
    __builtin_memcpy(row + c, &p, sizeof p);
  } else {
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
      if (c + k < cols) row[c + k] = p.v[k];
  }
}

}  // namespace rslx
