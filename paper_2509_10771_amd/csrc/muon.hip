// Muon step: momentum, the update made orthogonal by quintic Newton-Schulz steps, the weights' step, gfx950.
//
//   m' = beta m + grad,  u = nesterov ? grad + beta m' : m',  X = u / |u|_F  [p, q] with p <= q (a tall matrix is taken transposed)
//   `steps` times:  A = X X^T,  B = a I + b A + c A^2,  X <- B X
//   w' = (1 - lr decay) w - lr scale X
//
// The products run on the fp16 matrix cores in fp32's effect: a value v is held as two fp16 numbers, the rounded 2^12 v and the rounded rest (22
// significant bits), and a product is hi hi + hi lo + lo hi, summed in fp32.  What is left out and what the rest's rounding loses is at most 2^-22
// of a product each; fp32's own rounding is 2^-24 for each of the terms of a sum.  The singular values of X are at most 1.21 in every step (at most 1
// to begin with, and 0 <= a s + b s^3 + c s^5 < 1.203 from 0 to 1.21), those of A at most 1.47 and of B at most a, so no number passes 2^12 * 3.45.  A
// rest below the smallest fp16 number is lost: 2^-37 of a value, where values of X are 2^-8 to 2^-12 of a size.
//
// Every product is of two matrices whose rows hold the contraction index (X X^T; A A as A is symmetric; B and the transposed X), so operands are
// stored as the matrix instruction takes them: blocks of 32 rows x 16 indices, 64 lanes x 8 values of hi, then of lo; block (row / 32, k / 16) row by row.
// A lane's 16 bytes of a block are one load, and a wavefront's are 1024 bytes side by side.  Sides are padded to 32 with zeros.
#include "memory.h"

namespace rslx {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float HOLD = 4096.f, UNHOLD = 0x1p-12f, UNHOLD2 = 0x1p-24f;
constexpr int BLOCK = 1024;               // fp16 values of a block: 512 of hi, 512 of lo

__device__ __forceinline__ int pad32(int n) { return (n + 31) & ~31; }

__device__ __forceinline__ const MuonItem& item_of(const MuonArgs& a, int block) {
  int i = 0;
  while (i + 1 < a.count && a.item[i + 1].first <= block) ++i;
  return a.item[i];
}

// hi and lo of a value that is held times 2^12.
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

// Place of value (row, k) among the blocks of a matrix whose rows have kb blocks; lo lies 512 behind hi.
__device__ __forceinline__ int64_t place(int row, int k, int kb) {
  return ((int64_t)(row >> 5) * kb + (k >> 4)) * BLOCK + ((((k >> 3) & 1) << 5) + (row & 31)) * 8 + (k & 7);
}

constexpr int ELEMENT_THREADS = 256;

__global__ __launch_bounds__(ELEMENT_THREADS) void muon_momentum_kernel(MuonArgs a) {
  const MuonItem& m = item_of(a, blockIdx.x);
  const int first = m.first, blocks = (&m == &a.item[a.count - 1] ? (int)gridDim.x : (&m)[1].first) - first;
  const int64_t n = (int64_t)m.rows * m.cols;
  double sum = 0.0;
  for (int64_t i = (int64_t)(blockIdx.x - first) * ELEMENT_THREADS + threadIdx.x; i < n; i += (int64_t)blocks * ELEMENT_THREADS) {
    const float g = m.grad[i], now = fmaf(a.momentum, m.m_in ? m.m_in[i] : 0.f, g), u = a.nesterov ? fmaf(a.momentum, now, g) : now;
    if (m.m_out) m.m_out[i] = now;
    m.u[i] = u;
    sum += (double)u * u;
  }
  __shared__ double lds[ELEMENT_THREADS / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < ELEMENT_THREADS / 64; ++w) sum += lds[w];
    m.norm[blockIdx.x - first] = sum;
  }
}

int norm_blocks(const MuonItem& m) {
  const int64_t n = ((int64_t)m.rows * m.cols + 4 * ELEMENT_THREADS - 1) / (4 * ELEMENT_THREADS);
  return n < MUON_NORM_BLOCKS ? (int)n : MUON_NORM_BLOCKS;
}

// X and X transposed from u: a wavefront makes 32 x 32 values of X.
__global__ __launch_bounds__(ELEMENT_THREADS) void muon_pack_kernel(MuonArgs a) {
  __shared__ float tile[ELEMENT_THREADS / 64][32][33];
  const MuonItem& m = item_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = ((int64_t)m.rows * m.cols + 4 * ELEMENT_THREADS - 1) / (4 * ELEMENT_THREADS);
  const int parts = n < MUON_NORM_BLOCKS ? (int)n : MUON_NORM_BLOCKS;
  double sum = lane < parts ? m.norm[lane] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  const double inv = sum == 0.0 ? 0.0 : (double)HOLD / sqrt(sum);
  const int P = pad32(m.p) / 32, Q = pad32(m.q) / 32;
  const int at = (blockIdx.x - m.first) * (ELEMENT_THREADS / 64) + wave;
  const bool here = at < P * Q, tall = m.rows > m.cols;
  const int p0 = here ? at / Q * 32 : 0, q0 = here ? at % Q * 32 : 0;
  if (here)
    for (int i = lane; i < 1024; i += 64) {
      const int slow = i >> 5, fast = i & 31;            // of u: rows and columns
      const int row = (tall ? q0 : p0) + slow, col = (tall ? p0 : q0) + fast;
      const float v = row < m.rows && col < m.cols ? (float)(m.u[(int64_t)row * m.cols + col] * inv) : 0.f;
      if (tall) tile[wave][fast][slow] = v;
      else tile[wave][slow][fast] = v;
    }
  __syncthreads();
  if (!here) return;
  const int r = lane & 31, k8 = (lane >> 5) * 8;
  for (int half = 0; half < 2; ++half) {
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(tile[wave][r][half * 16 + k8 + e], h, l);
      hi[e] = h;
      lo[e] = l;
    }
    uint16_t* to = m.x + ((int64_t)(p0 >> 5) * (Q * 2) + (q0 >> 4) + half) * BLOCK + lane * 8;
    *reinterpret_cast<half8*>(to) = hi;
    *reinterpret_cast<half8*>(to + 512) = lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(tile[wave][half * 16 + k8 + e][r], h, l);
      hi[e] = h;
      lo[e] = l;
    }
    to = m.xt[0] + ((int64_t)(q0 >> 5) * (P * 2) + (p0 >> 4) + half) * BLOCK + lane * 8;
    *reinterpret_cast<half8*>(to) = hi;
    *reinterpret_cast<half8*>(to + 512) = lo;
  }
}

enum MuonProduct { MUON_GRAM, MUON_SQUARE, MUON_APPLY, MUON_LAST };

// Tile `t` of the upper triangle, column by column: (0,0), (0,1), (1,1), (0,2), ..
__device__ __forceinline__ void triangle(int t, int& i, int& j) {
  j = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while ((int64_t)j * (j + 1) / 2 > t) --j;
  while ((int64_t)(j + 1) * (j + 2) / 2 <= t) ++j;
  i = t - (int)((int64_t)j * (j + 1) / 2);
}

// One product; a workgroup makes 64 x 64 values, each of its four wavefronts 32 x 32.  A and B are symmetric: of each pair of tiles one is computed and both
// are stored.
template <MuonProduct KIND>
__global__ __launch_bounds__(256) void muon_product_kernel(MuonArgs a, int turn) {
  constexpr bool SYMMETRIC = KIND == MUON_GRAM || KIND == MUON_SQUARE;
  const MuonItem& m = item_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int P = pad32(m.p) / 32, Q = pad32(m.q) / 32;
  int ti, tj;
  if (SYMMETRIC) {
    triangle(blockIdx.x - m.first, ti, tj);
  } else {
    const int tiles = (Q + 1) / 2;
    ti = (blockIdx.x - m.first) / tiles;
    tj = (blockIdx.x - m.first) % tiles;
  }
  const int rb = ti * 2 + (wave >> 1), cb = tj * 2 + (wave & 1), columns = SYMMETRIC ? P : Q;
  if (rb >= P || cb >= columns) return;
  const int kb = KIND == MUON_GRAM ? Q * 2 : P * 2;
  const uint16_t* left = KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : m.b;
  const uint16_t* right = KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : m.xt[turn];
  left += (int64_t)rb * kb * BLOCK + lane * 8;
  right += (int64_t)cb * kb * BLOCK + lane * 8;
  float16v acc = {};
  for (int k = 0; k < kb; ++k, left += BLOCK, right += BLOCK) {
    const half8 lh = *reinterpret_cast<const half8*>(left), ll = *reinterpret_cast<const half8*>(left + 512);
    const half8 rh = *reinterpret_cast<const half8*>(right), rl = *reinterpret_cast<const half8*>(right + 512);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rl, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll, rh, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rh, acc, 0, 0, 0);
  }
  // a lane has one column and four times four rows one after another
  const int col = cb * 32 + (lane & 31);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = rb * 32 + i * 8 + (lane >> 5) * 4;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = acc[i * 4 + e] * UNHOLD;                    // held times 2^12
    if constexpr (KIND == MUON_LAST) {
      const float keep = 1.f - a.lr * a.decay, by = a.lr * m.scale * UNHOLD;
      const bool tall = m.rows > m.cols;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row + e < m.p && col < m.q) {
          const int64_t at = tall ? (int64_t)col * m.cols + row + e : (int64_t)(row + e) * m.cols + col;
          m.w_out[at] = (m.w_in ? keep * m.w_in[at] : 0.f) - by * v[e];
        }
    } else {
      const int64_t at = place(col, row, P * 2);
      if constexpr (KIND == MUON_SQUARE) {
        const half4 h = *reinterpret_cast<const half4*>(m.a + at), l = *reinterpret_cast<const half4*>(m.a + at + 512);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = NS_C * v[e] + NS_B * ((float)h[e] + (float)l[e]) + (row + e == col ? NS_A * HOLD : 0.f);
      }
      half4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        _Float16 h, l;
        split(v[e], h, l);
        hi[e] = h;
        lo[e] = l;
      }
      uint16_t* to = KIND == MUON_GRAM ? m.a : KIND == MUON_SQUARE ? m.b : m.xt[turn ^ 1];
      *reinterpret_cast<half4*>(to + at) = hi;
      *reinterpret_cast<half4*>(to + at + 512) = lo;
      if (!SYMMETRIC || ti != tj) {
        to = KIND == MUON_GRAM ? m.a : KIND == MUON_SQUARE ? m.b : m.x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t mirrored = place(row + e, col, SYMMETRIC ? P * 2 : Q * 2);
          *reinterpret_cast<_Float16*>(to + mirrored) = hi[e];
          *reinterpret_cast<_Float16*>(to + mirrored + 512) = lo[e];
        }
      }
    }
  }
}

template <typename Count>
unsigned place_items(MuonArgs& a, Count count) {
  int64_t n = 0;
  for (int i = 0; i < a.count; ++i) {
    a.item[i].first = (int32_t)n;
    n += count(a.item[i]);
  }
  return (unsigned)n;
}

}  // namespace

hipError_t launch_muon(MuonArgs& a, int steps, hipStream_t stream) {
  double values = 0, gram = 0, square = 0, apply = 0, planes = 0, symmetric = 0;
  for (int i = 0; i < a.count; ++i) {
    const double p = a.item[i].p, q = a.item[i].q;
    values += p * q;
    gram += p * p * q;
    square += p * p * p;
    apply += 2 * p * p * q;
    planes += 4 * p * q;
    symmetric += 4 * p * p;
  }
  const auto blocks32 = [](int n) { return (int64_t)(n + 31) / 32; };
  const auto tiles = [](int n) { return (int64_t)(n + 63) / 64; };
  unsigned grid = place_items(a, [](const MuonItem& m) { return (int64_t)norm_blocks(m); });
  {
    TraceScope trace(stream, "muon_momentum", 6 * values, 16 * values);
    hipLaunchKernelGGL(muon_momentum_kernel, dim3(grid), dim3(ELEMENT_THREADS), 0, stream, a);
  }
  grid = place_items(a, [&](const MuonItem& m) { return (blocks32(m.p) * blocks32(m.q) + 3) / 4; });
  {
    TraceScope trace(stream, "muon_pack", values, 4 * values + 2 * planes);
    hipLaunchKernelGGL(muon_pack_kernel, dim3(grid), dim3(ELEMENT_THREADS), 0, stream, a);
  }
  for (int s = 0; s < steps; ++s) {
    const int turn = s & 1;
    grid = place_items(a, [&](const MuonItem& m) { return tiles(m.p) * (tiles(m.p) + 1) / 2; });
    {
      TraceScope trace(stream, "muon_gram", gram, planes + symmetric);
      hipLaunchKernelGGL((muon_product_kernel<MUON_GRAM>), dim3(grid), dim3(256), 0, stream, a, turn);
    }
    {
      TraceScope trace(stream, "muon_square", square, 2 * symmetric);
      hipLaunchKernelGGL((muon_product_kernel<MUON_SQUARE>), dim3(grid), dim3(256), 0, stream, a, turn);
    }
    grid = place_items(a, [&](const MuonItem& m) { return tiles(m.p) * tiles(m.q); });
    TraceScope trace(stream, "muon_apply", apply, symmetric + 3 * planes);
    if (s + 1 < steps) hipLaunchKernelGGL((muon_product_kernel<MUON_APPLY>), dim3(grid), dim3(256), 0, stream, a, turn);
    else hipLaunchKernelGGL((muon_product_kernel<MUON_LAST>), dim3(grid), dim3(256), 0, stream, a, turn);
  }
  return hipGetLastError();
}

}  // namespace rslx
