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
#include <type_traits>

#include "memory.h"

namespace rslx {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
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

constexpr int ELEMENT_THREADS = 256;

__host__ __device__ inline int norm_blocks(const MuonItem& m) {
  const int64_t n = ((int64_t)m.rows * m.cols + 4 * ELEMENT_THREADS - 1) / (4 * ELEMENT_THREADS);
  return n < MUON_NORM_BLOCKS ? (int)n : MUON_NORM_BLOCKS;
}

// Sum over a workgroup, in a fixed order; the first wavefront has it.
__device__ __forceinline__ double group_sum(double v) {
  __shared__ double lds[ELEMENT_THREADS / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < ELEMENT_THREADS / 64; ++w) v += lds[w];
  return v;
}

// Squares are summed in 64 bits, where no fp32 value's vanishes or overflows.
__global__ __launch_bounds__(ELEMENT_THREADS) void muon_momentum_kernel(MuonArgs a) {
  const MuonItem& m = item_of(a, blockIdx.x);
  const int block = blockIdx.x - m.first;
  const int64_t n = (int64_t)m.rows * m.cols, stride = (int64_t)norm_blocks(m) * ELEMENT_THREADS;
  double sum = 0.0;
  for (int64_t i = (int64_t)block * ELEMENT_THREADS + threadIdx.x; i < n; i += 4 * stride) {
    float g[4], before[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * stride < n) {
        g[k] = m.grad[i + k * stride];
        before[k] = m.m_in ? m.m_in[i + k * stride] : 0.f;
      }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * stride < n) {
        const float now = fmaf(a.momentum, before[k], g[k]), u = a.nesterov ? fmaf(a.momentum, now, g[k]) : now;
        if (m.m_out) m.m_out[i + k * stride] = now;
        m.u[i + k * stride] = u;
        sum += (double)u * u;
      }
  }
  sum = group_sum(sum);
  if (threadIdx.x == 0) m.norm[block] = sum;
}

// X and X transposed from u: a wavefront makes 32 x 32 values of X.
__global__ __launch_bounds__(ELEMENT_THREADS) void muon_pack_kernel(MuonArgs a) {
  __shared__ float tile[ELEMENT_THREADS / 64][32][33];
  const MuonItem& m = item_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double sum = 0.0;
  for (int i = threadIdx.x; i < norm_blocks(m); i += ELEMENT_THREADS) sum += m.norm[i];
  sum = group_sum(sum);
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

// A wavefront's operands for 16 contraction indices: BM blocks of rows of the left matrix, BN of the right one.
template <int BM, int BN>
struct Operands {
  half8 lh[BM], ll[BM], rh[BN], rl[BN];
  __device__ __forceinline__ void load(const uint16_t* const (&left)[BM], const uint16_t* const (&right)[BN], int k) {
#pragma unroll
    for (int i = 0; i < BM; ++i) {
      lh[i] = *reinterpret_cast<const half8*>(left[i] + (int64_t)k * BLOCK);
      ll[i] = *reinterpret_cast<const half8*>(left[i] + (int64_t)k * BLOCK + 512);
    }
#pragma unroll
    for (int j = 0; j < BN; ++j) {
      rh[j] = *reinterpret_cast<const half8*>(right[j] + (int64_t)k * BLOCK);
      rl[j] = *reinterpret_cast<const half8*>(right[j] + (int64_t)k * BLOCK + 512);
    }
  }
  __device__ __forceinline__ void multiply(float16v (&acc)[BM][BN]) const {
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
      for (int j = 0; j < BN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[i], rl[j], acc[i][j], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
      for (int j = 0; j < BN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll[i], rh[j], acc[i][j], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
      for (int j = 0; j < BN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[i], rh[j], acc[i][j], 0, 0, 0);
  }
};

typedef float Tile[32][33];

// What becomes of 32 x 32 values of a product (times 2^24, in the wavefront's tile): block (rb, cb).
template <MuonProduct KIND>
__device__ __forceinline__ void finish(const MuonArgs& a, const MuonItem& m, int turn, int rb, int cb, const Tile& tile) {
  constexpr bool SYMMETRIC = KIND == MUON_GRAM || KIND == MUON_SQUARE;
  const int lane = threadIdx.x & 63, r = lane & 31, k8 = (lane >> 5) * 8;
  const int P = pad32(m.p) / 32, Q = pad32(m.q) / 32;
  if constexpr (KIND == MUON_LAST) {
    const float keep = 1.f - a.lr * a.decay, by = a.lr * m.scale * UNHOLD2;
    const bool tall = m.rows > m.cols;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int slow = i * 2 + (lane >> 5), row = (tall ? cb : rb) * 32 + slow, col = (tall ? rb : cb) * 32 + r;
      if (row < m.rows && col < m.cols) {
        const int64_t at = (int64_t)row * m.cols + col;
        m.w_out[at] = (m.w_in ? keep * m.w_in[at] : 0.f) - by * (tall ? tile[r][slow] : tile[slow][r]);
      }
    }
    return;
  }
#pragma unroll
  for (int way = 0; way < 2; ++way) {                    // as it is, and transposed
    if (SYMMETRIC && way == 1 && rb == cb) break;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int k = half * 16 + k8;
      const int64_t block = way == 0 ? (int64_t)rb * (SYMMETRIC ? P : Q) * 2 + cb * 2 + half : (int64_t)cb * P * 2 + rb * 2 + half;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (way == 0 ? tile[r][k + e] : tile[k + e][r]) * UNHOLD;
      if constexpr (KIND == MUON_SQUARE) {
        const half8 h = *reinterpret_cast<const half8*>(m.a + block * BLOCK + lane * 8), l = *reinterpret_cast<const half8*>(m.a + block * BLOCK + 512 + lane * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = NS_C * v[e] + NS_B * ((float)h[e] + (float)l[e]) + (rb == cb && r == k + e ? NS_A * HOLD : 0.f);
      }
      half8 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        _Float16 h, l;
        split(v[e], h, l);
        hi[e] = h;
        lo[e] = l;
      }
      uint16_t* to = (KIND == MUON_GRAM ? m.a : KIND == MUON_SQUARE ? m.b : way == 0 ? m.x : m.xt[turn ^ 1]) + block * BLOCK + lane * 8;
      *reinterpret_cast<half8*>(to) = hi;
      *reinterpret_cast<half8*>(to + 512) = lo;
    }
  }
}

// One product; a workgroup makes B x B blocks, its four wavefronts a quarter of the contraction each, straight from memory's own layout into registers, DEPTH steps
// of 16 ahead.  A and B are symmetric: of each pair of blocks one is computed and both are stored.
template <MuonProduct KIND, int B, int DEPTH>
__global__ __launch_bounds__(256) void muon_product_kernel(MuonArgs a, int turn) {
  constexpr bool SYMMETRIC = KIND == MUON_GRAM || KIND == MUON_SQUARE;
  __shared__ union {
    float4 part[4][B * B][4][64];                        // wavefront, block, four of its sixteen registers
    Tile tile[4];
  } lds;
  const MuonItem& m = item_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int P = pad32(m.p) / 32, Q = pad32(m.q) / 32, columns = SYMMETRIC ? P : Q;
  int ti, tj;
  if (SYMMETRIC) {
    triangle(blockIdx.x - m.first, ti, tj);
  } else {
    const int tiles = (Q + B - 1) / B;
    ti = (blockIdx.x - m.first) / tiles;
    tj = (blockIdx.x - m.first) % tiles;
  }
  const int kb = KIND == MUON_GRAM ? Q * 2 : P * 2, each = (kb + 3) / 4, k0 = wave * each, k1 = k0 + each < kb ? k0 + each : kb;
  const uint16_t* l0 = (KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : m.b) + lane * 8;
  const uint16_t* r0 = (KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : m.xt[turn]) + lane * 8;
  const uint16_t *left[B], *right[B];
#pragma unroll
  for (int i = 0; i < B; ++i) {                          // (blocks beyond the edge: the last one again, and nothing is stored)
    const int rb = ti * B + i < P ? ti * B + i : P - 1, cb = tj * B + i < columns ? tj * B + i : columns - 1;
    left[i] = l0 + (int64_t)rb * kb * BLOCK;
    right[i] = r0 + (int64_t)cb * kb * BLOCK;
  }
  float16v acc[B][B];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) acc[i][j] = float16v{};
  if (k0 < k1) {
    Operands<B, B> o[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) o[d].load(left, right, k0 + d < k1 ? k0 + d : k1 - 1);
    for (int k = k0; k < k1; k += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (k + d < k1) o[d].multiply(acc);
        o[d].load(left, right, k + d + DEPTH < k1 ? k + d + DEPTH : k1 - 1);
      }
  }
  // the wavefronts' parts, in their order: a wavefront adds up a quarter of the blocks (B = 2), or the first one all of one block
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) lds.part[wave][i * B + j][q][lane] = float4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
  __syncthreads();
  const int rb = ti * B + wave / B, cb = tj * B + wave % B;
  const bool mine = wave < B * B && rb < P && cb < columns && (!SYMMETRIC || rb <= cb);
  float4 sum[4];
  if (mine)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[q] = lds.part[0][wave][q][lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        const float4 p = lds.part[w][wave][q][lane];
        sum[q] = float4{sum[q].x + p.x, sum[q].y + p.y, sum[q].z + p.z, sum[q].w + p.w};
      }
    }
  __syncthreads();
  if (!mine) return;
  // a lane has one column and four times four rows one after another
  Tile& tile = lds.tile[wave];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = q * 8 + (lane >> 5) * 4, col = lane & 31;
    tile[row][col] = sum[q].x;
    tile[row + 1][col] = sum[q].y;
    tile[row + 2][col] = sum[q].z;
    tile[row + 3][col] = sum[q].w;
  }
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  finish<KIND>(a, m, turn, rb, cb, tile);
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
  // blocks of 64 x 64 where they are as many as the GPU has compute units, of 32 x 32 otherwise
  auto product = [&](auto kind, const char* name, double flops, double bytes, int turn) {
    constexpr MuonProduct KIND = decltype(kind)::value;
    auto tiles = [&](int b) {
      return [=](const MuonItem& m) {
        const int64_t rows = (blocks32(m.p) + b - 1) / b, cols = (blocks32(m.q) + b - 1) / b;
        return KIND == MUON_GRAM || KIND == MUON_SQUARE ? rows * (rows + 1) / 2 : rows * cols;
      };
    };
    TraceScope trace(stream, name, flops, bytes);
    const unsigned grid = place_items(a, tiles(2));
    if (grid >= 256) hipLaunchKernelGGL((muon_product_kernel<KIND, 2, 2>), dim3(grid), dim3(256), 0, stream, a, turn);
    else hipLaunchKernelGGL((muon_product_kernel<KIND, 1, 4>), dim3(place_items(a, tiles(1))), dim3(256), 0, stream, a, turn);
  };
  for (int s = 0; s < steps; ++s) {
    product(std::integral_constant<MuonProduct, MUON_GRAM>(), "muon_gram", gram, planes + symmetric, s & 1);
    product(std::integral_constant<MuonProduct, MUON_SQUARE>(), "muon_square", square, 2 * symmetric, s & 1);
    if (s + 1 < steps) product(std::integral_constant<MuonProduct, MUON_APPLY>(), "muon_apply", apply, symmetric + 3 * planes, s & 1);
    else product(std::integral_constant<MuonProduct, MUON_LAST>(), "muon_apply", apply, symmetric + 3 * planes, s & 1);
  }
  return hipGetLastError();
}

}  // namespace rslx
