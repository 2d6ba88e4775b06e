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
//
// Small networks are bound by 17 dependent launches of 4 to 5 us each (actor and critic: 78 us; 2 us of each is the start and the table's load), so a
// launch takes all matrices, and its wavefronts share the contraction.  A large matrix is bound by the matrix cores at the rate that large products reach on the
// card: 2048 x 4096 1.05 to 1.08 ms, its products with X 101 us = 1020 TFLOP/s of fp16 (a library's 8192^3: 1110), the last, with the weights' step, 118.
#include <type_traits>

#include "memory.h"

namespace rslx {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float HOLD = 4096.f, UNHOLD = 0x1p-12f, UNHOLD2 = 0x1p-24f;
constexpr int BLOCK = 1024;               // fp16 values of a block: 512 of hi, 512 of lo

__host__ __device__ inline int pad32(int n) { return (n + 31) & ~31; }

// A matrix as the kernels see it.  p <= q are its sides, X is [p, q] (the transposed update where the matrix is tall), P and Q blocks of 32 rows.
struct Matrix {
  MuonItem m;
  int p, q, P, Q, block, place, index;    // block: the workgroup's among the matrix's, place: among all; index: the matrix's
  bool tall;
  float* u;                               // the update before it is made orthogonal, [rows, cols]
  double* norm;                           // partial sums of its squares
  uint16_t *x, *xt0, *xt1, *a, *b;           // X; X transposed, two in turn; A = X X^T; B = a I + b A + c A^2
};
__host__ __device__ inline size_t values_bytes(int rows, int cols) { return ((size_t)rows * cols * sizeof(float) + 255) / 256 * 256; }

// The matrix that the workgroup belongs to.  Every lane asks for one matrix's entry at once with where they begin, so that the table is read in one go.
__device__ __forceinline__ Matrix matrix_of(const MuonTable& t, MuonGrid grid) {
  constexpr int WORDS = sizeof(MuonItem) / 4;
  static_assert(sizeof(MuonItem) == 64 && RSLX_MUON_MAX_MATRICES <= 64, "an entry is four loads of 16 bytes, a lane has one");
  const int lane = (threadIdx.x & 63) % RSLX_MUON_MAX_MATRICES;
  const int begins = (threadIdx.x & 63) < RSLX_MUON_MAX_MATRICES ? t.first[grid][lane] : INT32_MAX;
  uint32_t entry[WORDS];
  __builtin_memcpy(entry, &t.item[lane], sizeof entry);
  // workgroups go to the eight dies in turn: each die gets a row of neighbours, which share operands in its L2
  const uint32_t each = gridDim.x / 8, more = gridDim.x % 8, die = blockIdx.x % 8;
  const int block = (int)(die * each + (die < more ? die : more) + blockIdx.x / 8);
  const int i = __popcll(__ballot(begins <= block)) - 1;
#pragma unroll
  for (int w = 0; w < WORDS; ++w) entry[w] = __builtin_amdgcn_readlane(entry[w], i);
  Matrix r;
  __builtin_memcpy(&r.m, entry, sizeof entry);
  r.block = block - __builtin_amdgcn_readlane(begins, i);
  r.place = block;
  r.index = i;
  r.tall = r.m.rows > r.m.cols;
  r.p = r.tall ? r.m.cols : r.m.rows;
  r.q = r.tall ? r.m.rows : r.m.cols;
  r.P = pad32(r.p) / 32;
  r.Q = pad32(r.q) / 32;
  char* at = r.m.base;
  r.u = reinterpret_cast<float*>(at);
  at += values_bytes(r.m.rows, r.m.cols);
  r.norm = reinterpret_cast<double*>(at);
  at += MUON_NORM_BLOCKS * sizeof(double);
  r.x = reinterpret_cast<uint16_t*>(at);
  const int64_t plane = (int64_t)r.P * r.Q * 2 * BLOCK, square = (int64_t)r.P * r.P * 2 * BLOCK;
  r.xt0 = r.x + plane;
  r.xt1 = r.xt0 + plane;
  r.a = r.xt1 + plane;
  r.b = r.a + square;
  return r;
}

// Loads and stores of global memory: pointers that come from the table would be accessed as any kind of memory, and those accesses are waited for
// with every access of LDS.
template <typename T> __device__ __forceinline__ T get(const T* p) { return *(const __attribute__((address_space(1))) T*)p; }
template <typename T> __device__ __forceinline__ void set(T* p, T v) { *(__attribute__((address_space(1))) T*)p = v; }
__device__ __forceinline__ half8 get8(const uint16_t* p) { return get(reinterpret_cast<const half8*>(p)); }
__device__ __forceinline__ void set8(uint16_t* p, half8 v) { set(reinterpret_cast<half8*>(p), v); }

// hi and lo of a value that is held times 2^12.
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

constexpr int ELEMENT_THREADS = 256;

__host__ __device__ inline int norm_blocks(int rows, int cols) {
  const int64_t n = ((int64_t)rows * cols + 4 * ELEMENT_THREADS - 1) / (4 * ELEMENT_THREADS);
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
__global__ __launch_bounds__(ELEMENT_THREADS) void muon_momentum_kernel(MuonTable t, MuonTable* in_workspace) {
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < (int)(sizeof t / 4); i += ELEMENT_THREADS) reinterpret_cast<uint32_t*>(in_workspace)[i] = reinterpret_cast<const uint32_t*>(&t)[i];
  const Matrix x = matrix_of(t, MUON_MOMENTUM_GRID);
  const MuonItem& m = x.m;
  const int64_t n = (int64_t)m.rows * m.cols, stride = (int64_t)norm_blocks(m.rows, m.cols) * ELEMENT_THREADS;
  double sum = 0.0;
  for (int64_t i = (int64_t)x.block * ELEMENT_THREADS + threadIdx.x; i < n; i += 4 * stride) {
    float g[4], before[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * stride < n) {
        g[k] = get(m.grad + i + k * stride);
        before[k] = m.m_in ? get(m.m_in + i + k * stride) : 0.f;
      }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * stride < n) {
        const float now = fmaf(t.momentum, before[k], g[k]), u = t.nesterov ? fmaf(t.momentum, now, g[k]) : now;
        if (m.m_out) set(m.m_out + i + k * stride, now);
        set(x.u + i + k * stride, u);
        sum += (double)u * u;
      }
  }
  sum = group_sum(sum);
  if (threadIdx.x == 0) set(x.norm + x.block, sum);
}

// X and X transposed from u: a wavefront makes 32 x 32 values of X.
__global__ __launch_bounds__(ELEMENT_THREADS) void muon_pack_kernel(const MuonTable* t) {
  __shared__ float tile[ELEMENT_THREADS / 64][32][33];
  const Matrix m = matrix_of(*t, MUON_PACK_GRID);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at = m.block * (ELEMENT_THREADS / 64) + wave;
  const bool here = at < m.P * m.Q;
  const int p0 = here ? at / m.Q * 32 : 0, q0 = here ? at % m.Q * 32 : 0;
  float u[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = (m.tall ? q0 : p0) + i * 2 + (lane >> 5), col = (m.tall ? p0 : q0) + (lane & 31);
    u[i] = row < m.m.rows && col < m.m.cols ? get(m.u + (int64_t)row * m.m.cols + col) : 0.f;
  }
  double sum = 0.0;
  for (int i = threadIdx.x; i < norm_blocks(m.m.rows, m.m.cols); i += ELEMENT_THREADS) sum += get(m.norm + i);
  sum = group_sum(sum);
  // 2^12 / |u|_F as a power of two and a factor: neither the values nor the factor leave fp32's range (multiplied in 64 bits the small nets' launch took 9.9 us
  // instead of 5.1)
  int power;
  const float factor = (float)frexp(sum == 0.0 ? 0.0 : (double)HOLD / sqrt(sum), &power);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int slow = i * 2 + (lane >> 5), fast = lane & 31;            // of u: rows and columns
    const float v = ldexpf(u[i], power) * factor;
    if (m.tall) tile[wave][fast][slow] = v;
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
    uint16_t* to = m.x + ((int64_t)(p0 >> 5) * (m.Q * 2) + (q0 >> 4) + half) * BLOCK + lane * 8;
    set8(to, hi);
    set8(to + 512, lo);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(tile[wave][half * 16 + k8 + e][r], h, l);
      hi[e] = h;
      lo[e] = l;
    }
    to = m.xt0 + ((int64_t)(q0 >> 5) * (m.P * 2) + (p0 >> 4) + half) * BLOCK + lane * 8;
    set8(to, hi);
    set8(to + 512, lo);
  }
}

enum MuonProduct { MUON_GRAM, MUON_SQUARE, MUON_APPLY, MUON_LAST };

// Neighbouring workgroups make tiles of the same rows and columns: tiles are numbered in strips of eight rows (of eight columns where only those on
// and above the diagonal count), across the strip first.
constexpr int STRIP = 8;

// Tile `t` of rows x cols.
__device__ __forceinline__ void tile_in_strips(int t, int rows, int cols, int& i, int& j) {
  const int strip = t / (STRIP * cols), in = t % (STRIP * cols), high = rows - strip * STRIP < STRIP ? rows - strip * STRIP : STRIP;
  i = strip * STRIP + in % high;
  j = in / high;
}

// Tile `t` of the upper triangle, column by column: (0,0), (0,1), (1,1), (0,2), ..
__device__ __forceinline__ void triangle(int t, int& i, int& j) {
  j = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while ((int64_t)j * (j + 1) / 2 > t) --j;
  while ((int64_t)(j + 1) * (j + 2) / 2 <= t) ++j;
  i = t - (int)((int64_t)j * (j + 1) / 2);
}

// The same in strips, of n columns: strip g has the 8 g rows above its own triangle.
__device__ __forceinline__ void triangle_in_strips(int t, int n, int& i, int& j) {
  auto before = [](int64_t g) { return STRIP * STRIP * g * (g - 1) / 2 + STRIP * (STRIP + 1) / 2 * g; };
  int g = (int)sqrtf(t * (2.f / (STRIP * STRIP)));
  while (before(g) > t) --g;
  while (before(g + 1) <= t) ++g;
  const int wide = n - g * STRIP < STRIP ? n - g * STRIP : STRIP, in = t - (int)before(g), above = g * STRIP * wide;
  if (in < above) {
    i = in / wide;
    j = g * STRIP + in % wide;
  } else {
    triangle(in - above, i, j);
    i += g * STRIP;
    j += g * STRIP;
  }
}

// Tile `t` of 8 x 4 blocks among those that reach on or above the diagonal, row by row: row i has cols - 2 i.
__device__ __forceinline__ void wide_triangle(int t, int cols, int& i, int& j) {
  auto before = [&](int i) { return i * cols - i * (i - 1); };
  const float b = cols + 1.f, under = b * b - 4.f * t;
  i = (int)((b - sqrtf(under > 0.f ? under : 0.f)) * 0.5f);
  while (i > 0 && before(i) > t) --i;
  while (before(i + 1) <= t) ++i;
  j = 2 * i + t - before(i);
}
__host__ __device__ inline int wide_triangle_tiles(int P) {
  const int rows = (P + 7) / 8, cols = (P + 3) / 4;
  return rows * cols - rows * (rows - 1);
}

// A wavefront's operands for 16 contraction indices: BM blocks of rows of the left matrix, BN of the right one.
template <int BM, int BN>
struct Operands {
  half8 lh[BM], ll[BM], rh[BN], rl[BN];
  __device__ __forceinline__ void load(const uint16_t* const (&left)[BM], const uint16_t* const (&right)[BN], int k) {
#pragma unroll
    for (int i = 0; i < BM; ++i) {
      lh[i] = get8(left[i] + (int64_t)k * BLOCK);
      ll[i] = get8(left[i] + (int64_t)k * BLOCK + 512);
    }
#pragma unroll
    for (int j = 0; j < BN; ++j) {
      rh[j] = get8(right[j] + (int64_t)k * BLOCK);
      rl[j] = get8(right[j] + (int64_t)k * BLOCK + 512);
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

// What becomes of 32 x 32 values of a product (times 2^24, in a tile in LDS): block (rb, cb), in four quarters, which one wavefront makes after another or four
// side by side.  A quarter of a stored result is half of the block's 16-byte units, as it is (0, 1) or transposed (2, 3); of the weights, eight rows.
template <MuonProduct KIND>
struct Quarter {
  static constexpr bool SYMMETRIC = KIND == MUON_GRAM || KIND == MUON_SQUARE;
  bool here;
  int64_t at;                                            // its place in the result (in A where that is read as well), or in the weights
  half8 h, l;                                            // MUON_SQUARE: A there
  float w[4];                                            // MUON_LAST: the weights
  // Where it goes, and what has to be read there.
  __device__ __forceinline__ void ask(const Matrix& m, int quarter, int rb, int cb) {
    const int lane = threadIdx.x & 63;
    if constexpr (KIND == MUON_LAST) {
      const int row = (m.tall ? cb : rb) * 32 + quarter * 8 + (lane >> 5), col = (m.tall ? rb : cb) * 32 + (lane & 31);
      at = (int64_t)row * m.m.cols + col;
      here = col < m.m.cols;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = m.m.w_in && here && row + i * 2 < m.m.rows ? get(m.m.w_in + at + (int64_t)i * 2 * m.m.cols) : 0.f;
    } else {
      const bool turned = quarter >= 2;
      here = !(SYMMETRIC && turned && rb == cb);
      at = ((turned ? (int64_t)cb * m.P * 2 + rb * 2 : (int64_t)rb * (SYMMETRIC ? m.P : m.Q) * 2 + cb * 2) + (quarter & 1)) * BLOCK + lane * 8;
      if constexpr (KIND == MUON_SQUARE)
        if (here) {
          h = get8(m.a + at);
          l = get8(m.a + at + 512);
        }
    }
  }
  __device__ __forceinline__ void make(const MuonTable& t, const Matrix& m, int turn, int quarter, int rb, int cb, const Tile& tile) const {
    const int lane = threadIdx.x & 63, r = lane & 31;
    if (!here) return;
    if constexpr (KIND == MUON_LAST) {
      const float keep = 1.f - t.lr * t.decay, by = t.lr * m.m.scale * UNHOLD2;
      const int slow = quarter * 8 + (lane >> 5), row = (m.tall ? cb : rb) * 32 + slow;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (row + i * 2 < m.m.rows)
          set(m.m.w_out + at + (int64_t)i * 2 * m.m.cols, keep * w[i] - by * (m.tall ? tile[r][slow + i * 2] : tile[slow + i * 2][r]));
    } else {
      const bool turned = quarter >= 2;
      const int k = (quarter & 1) * 16 + (lane >> 5) * 8;
      half8 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = (turned ? tile[k + e][r] : tile[r][k + e]) * UNHOLD;
        if constexpr (KIND == MUON_SQUARE) v = NS_C * v + NS_B * ((float)h[e] + (float)l[e]) + (rb == cb && r == k + e ? NS_A * HOLD : 0.f);
        _Float16 high, low;
        split(v, high, low);
        hi[e] = high;
        lo[e] = low;
      }
      uint16_t *const x = m.x, *const xt0 = m.xt0, *const xt1 = m.xt1;       // (values, not places to choose from: those would lie on the stack)
      uint16_t* const next = turn ? xt0 : xt1;
      uint16_t* const to = (KIND == MUON_GRAM ? m.a : KIND == MUON_SQUARE ? m.b : turned ? next : x) + at;
      set8(to, hi);
      set8(to + 512, lo);
    }
  }
};
template <MuonProduct KIND>
__device__ __forceinline__ void finish(const MuonTable& t, const Matrix& m, int turn, int rb, int cb, const Tile& tile) {
  Quarter<KIND> q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i].ask(m, i, rb, cb);
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i].make(t, m, turn, i, rb, cb, tile);
}

// One product; a workgroup makes B x B blocks, its four wavefronts a quarter of the contraction each, straight from memory's own layout into registers, DEPTH steps
// of 16 ahead.  A and B are symmetric: of each pair of blocks one is computed and both are stored.
template <MuonProduct KIND, int B, int DEPTH>
__global__ __launch_bounds__(256) void muon_product_kernel(const MuonTable* t, int turn) {
  constexpr bool SYMMETRIC = KIND == MUON_GRAM || KIND == MUON_SQUARE;
  // a block's parts (B = 2: those of the wavefronts behind the one that adds them up)
  __shared__ union {
    float4 part[B == 1 ? 4 : B * B][B == 1 ? 4 : 3][B == 1 ? 1 : 4][64];      // block, wavefront, four of its sixteen registers; B = 1: registers, wavefront
    Tile tile[B == 1 ? 1 : 4];
  } lds;
  const Matrix m = matrix_of(*t, SYMMETRIC ? MUON_SYMMETRIC_GRID : MUON_APPLY_GRID);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), columns = SYMMETRIC ? m.P : m.Q;
  int ti, tj;
  if (SYMMETRIC) {
    triangle_in_strips(m.block, (m.P + B - 1) / B, ti, tj);
  } else {
    tile_in_strips(m.block, (m.P + B - 1) / B, (m.Q + B - 1) / B, ti, tj);
  }
  const int kb = (KIND == MUON_GRAM ? m.Q : m.P) * 2, each = (kb + 3) / 4, k0 = wave * each, k1 = k0 + each < kb ? k0 + each : kb;
  const uint16_t* l0 = (KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : m.b) + lane * 8;
  const uint16_t* r0 = (KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : (turn ? m.xt1 : m.xt0)) + lane * 8;
  const uint16_t *left[B], *right[B];
#pragma unroll
  for (int i = 0; i < B; ++i) {                          // (blocks beyond the edge: the last one again, and nothing is stored)
    const int rb = ti * B + i < m.P ? ti * B + i : m.P - 1, cb = tj * B + i < columns ? tj * B + i : columns - 1;
    left[i] = l0 + (int64_t)rb * kb * BLOCK;
    right[i] = r0 + (int64_t)cb * kb * BLOCK;
  }
  Quarter<KIND> quarter;
  if constexpr (B == 1) quarter.ask(m, wave, ti, tj);
  float16v acc[B][B];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) acc[i][j] = float16v{};
  if (k0 < k1) {
    Operands<B, B> o[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (k0 + d < k1) o[d].load(left, right, k0 + d);
    for (int k = k0; k < k1; k += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (k + d < k1) o[d].multiply(acc);
        if (k + d + DEPTH < k1) o[d].load(left, right, k + d + DEPTH);
      }
  }
  if constexpr (B == 1) {
    // every wavefront adds up a quarter of the registers, and makes a quarter of the result
#pragma unroll
    for (int q = 0; q < 4; ++q) lds.part[q][wave][0][lane] = float4{acc[0][0][q * 4], acc[0][0][q * 4 + 1], acc[0][0][q * 4 + 2], acc[0][0][q * 4 + 3]};
    __syncthreads();
    float4 sum = lds.part[wave][0][0][lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const float4 p = lds.part[wave][w][0][lane];
      sum = float4{sum.x + p.x, sum.y + p.y, sum.z + p.z, sum.w + p.w};
    }
    __syncthreads();
    Tile& tile = lds.tile[0];
    const int row = wave * 8 + (lane >> 5) * 4, col = lane & 31;
    tile[row][col] = sum.x;
    tile[row + 1][col] = sum.y;
    tile[row + 2][col] = sum.z;
    tile[row + 3][col] = sum.w;
    __syncthreads();
    quarter.make(*t, m, turn, wave, ti, tj, tile);
    return;
  } else {
  // a block's parts are added up by the wavefront of its number: its own, then those of the ones behind it, around
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int behind = (wave - (i * B + j) + 4) & 3;
      if (behind > 0)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          lds.part[i * B + j][behind - 1][q][lane] = float4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
    }
  __syncthreads();
  const int rb = ti * B + wave / B, cb = tj * B + wave % B;
  const bool mine = wave < B * B && rb < m.P && cb < columns && (!SYMMETRIC || rb <= cb);
  float4 sum[4];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (mine && wave == i * B + j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          sum[q] = float4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
#pragma unroll
          for (int w = 0; w < 3; ++w) {
            const float4 p = lds.part[i * B + j][w][q][lane];
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
  finish<KIND>(*t, m, turn, rb, cb, tile);
  }
}

// The same product with tiles of 8 x 4 blocks, for matrices whose tiles fill the GPU: the kernel above reads 8 KB for every 12 matrix instructions, and is bound
// by what the L2 delivers (16 TB/s, the matrix cores 39 % busy).  Here a wavefront has two rows of blocks to itself, straight from memory, and the four columns
// that all of them need come through LDS, two steps of 16 at a time, the next ones on their way in registers.
// Symmetric products have too few such tiles: they are cut into pieces of the contraction as well, whose sums go to memory and are added up, in their order,
// by muon_fold_kernel.
constexpr int PART = 32 * 1024;                          // sums of a tile's 32 blocks: block, four of its sixteen registers, lane
template <MuonProduct KIND>
__global__ __launch_bounds__(256) void muon_large_kernel(const MuonTable* t, int turn) {
  constexpr bool SYMMETRIC = KIND == MUON_GRAM || KIND == MUON_SQUARE;
  constexpr int RW = 2, CW = 4, UNITS = 256;             // rows and columns of blocks; units of 16 bytes that two steps of a column are
  __shared__ union {
    half8 right[2][CW][2][2][64];                        // turn, column, step, hi and lo
    Tile tile[4];
  } lds;
  const Matrix m = matrix_of(*t, SYMMETRIC ? MUON_PIECES_GRID : MUON_LARGE_GRID);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), columns = SYMMETRIC ? m.P : m.Q;
  const int kb = (KIND == MUON_GRAM ? m.Q : m.P) * 2;
  int ti, tj, first = 0, stages = kb / 2;
  if constexpr (SYMMETRIC) {
    const int tiles = wide_triangle_tiles(m.P), each = (stages + t->pieces - 1) / t->pieces;
    first = m.block / tiles * each;
    stages = stages - first < each ? stages - first : each;      // (may be none)
    wide_triangle(m.block % tiles, (m.P + CW - 1) / CW, ti, tj);
  } else {
    tile_in_strips(m.block, (m.P + 4 * RW - 1) / (4 * RW), (m.Q + CW - 1) / CW, ti, tj);
  }
  const uint16_t* l0 = (KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : m.b) + (int64_t)first * 2 * BLOCK + lane * 8;
  const uint16_t* r0 = (KIND == MUON_GRAM ? m.x : KIND == MUON_SQUARE ? m.a : (turn ? m.xt1 : m.xt0)) + (int64_t)first * 2 * BLOCK + threadIdx.x * 8;
  const uint16_t *left[RW], *right[CW];
  const int row0 = (ti * 4 + wave) * RW, col0 = tj * CW;
#pragma unroll
  for (int i = 0; i < RW; ++i) left[i] = l0 + (int64_t)(row0 + i < m.P ? row0 + i : m.P - 1) * kb * BLOCK;
#pragma unroll
  for (int j = 0; j < CW; ++j) right[j] = r0 + (int64_t)(col0 + j < columns ? col0 + j : columns - 1) * kb * BLOCK;
  float16v acc[RW][CW];
#pragma unroll
  for (int i = 0; i < RW; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) acc[i][j] = float16v{};
  half8 ahead[CW], lh[2][RW], ll[2][RW];
  auto ask = [&](int s) {
#pragma unroll
    for (int j = 0; j < CW; ++j) ahead[j] = get8(right[j] + (int64_t)s * 2 * BLOCK);
  };
  auto put = [&](int s) {
#pragma unroll
    for (int j = 0; j < CW; ++j) (&lds.right[s & 1][j][0][0][0])[threadIdx.x] = ahead[j];
  };
  auto ask_left = [&](int h, int k) {
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      lh[h][i] = get8(left[i] + (int64_t)k * BLOCK);
      ll[h][i] = get8(left[i] + (int64_t)k * BLOCK + 512);
    }
  };
  static_assert(sizeof lds.right[0][0] == UNITS * 16, "a thread has one unit of a column");
  if (stages > 0) ask(0);
  put(0);
  if (stages > 0) ask(stages > 1 ? 1 : 0);               // (in the order of the loop below, which waits for the columns alone that way)
  __builtin_amdgcn_sched_barrier(0);
  if (stages > 0) {
    ask_left(0, 0);
    ask_left(1, 1);
  }
  __syncthreads();
  // Behind the last stage its columns and rows are asked for and put again, and not used: a branch between a load and its use would have the compiler wait for
  // whatever the other way leaves.  The columns of a pair are read while the pair before it is multiplied.
  half8 rh[2][2], rl[2][2];
  auto read = [&](int s, int pair) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      rh[pair & 1][c] = lds.right[s & 1][(pair & 1) * 2 + c][pair >> 1][0][lane];
      rl[pair & 1][c] = lds.right[s & 1][(pair & 1) * 2 + c][pair >> 1][1][lane];
    }
  };
  for (int s = 0; s < stages; ++s) {
    read(s, 0);
    put(s + 1);                                          // (read last in front of the barrier behind stage s - 1)
    ask(s + 2 < stages ? s + 2 : stages - 1);
#pragma unroll
    for (int pair = 0; pair < 4; ++pair) {
      const int h = pair >> 1, j = (pair & 1) * 2, now = pair & 1;
      if (pair < 3) read(s, pair + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[i][j + c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[h][i], rl[now][c], acc[i][j + c], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[i][j + c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll[h][i], rh[now][c], acc[i][j + c], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[i][j + c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[h][i], rh[now][c], acc[i][j + c], 0, 0, 0);
      if (pair & 1) ask_left(h, s + 1 < stages ? s * 2 + 2 + h : s * 2 + h);
    }
    __syncthreads();
  }
  if constexpr (SYMMETRIC) {
    float4v* part = reinterpret_cast<float4v*>(t->parts + (int64_t)m.place * PART) + lane;
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
      for (int j = 0; j < CW; ++j)
        if (row0 + i <= col0 + j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            set(part + (((wave * RW + i) * CW + j) * 4 + q) * 64, float4v{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]});
    return;
  }
  Tile& tile = lds.tile[wave];
#pragma unroll
  for (int i = 0; i < RW; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      const int rb = row0 + i, cb = col0 + j;
      if (rb >= m.P || cb >= m.Q) continue;
#pragma unroll
      for (int q = 0; q < 16; ++q) tile[(q >> 2) * 8 + (lane >> 5) * 4 + (q & 3)][lane & 31] = acc[i][j][q];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      finish<KIND>(*t, m, turn, rb, cb, tile);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

// A wavefront adds up the pieces of a block; eight workgroups have a tile.
template <MuonProduct KIND>
__global__ __launch_bounds__(256) void muon_fold_kernel(const MuonTable* t, int turn) {
  __shared__ Tile tiles[4];
  const Matrix m = matrix_of(*t, MUON_FOLD_GRID);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), block = m.block % 8 * 4 + wave;
  const int count = wide_triangle_tiles(m.P), at = m.block / 8;
  int ti, tj;
  wide_triangle(at, (m.P + 3) / 4, ti, tj);
  const int rb = ti * 8 + block / 4, cb = tj * 4 + block % 4;
  if (rb > cb || cb >= m.P) return;
  const float4v* part = reinterpret_cast<const float4v*>(t->parts + (int64_t)(t->first[MUON_PIECES_GRID][m.index] + at) * PART) + block * 256 + lane;
  float4v sum[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) sum[q] = get(part + q * 64);
  for (int piece = 1; piece < t->pieces; ++piece) {
    part += (int64_t)count * (PART / 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] += get(part + q * 64);
  }
  Tile& tile = tiles[wave];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = q * 8 + (lane >> 5) * 4, col = lane & 31;
    tile[row][col] = sum[q].x;
    tile[row + 1][col] = sum[q].y;
    tile[row + 2][col] = sum[q].z;
    tile[row + 3][col] = sum[q].w;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  finish<KIND>(*t, m, turn, rb, cb, tile);
}

enum MuonShape { SMALL, MEDIUM, LARGE };                 // tiles of 32 x 32, 64 x 64, 256 x 128

// Workgroups of a launch, matrix by matrix.  One that has none begins where the next one does, and matrix_of finds the next.
template <typename Count>
unsigned place_items(MuonTable& t, int count, MuonGrid grid, Count of) {
  int64_t n = 0;
  for (int i = 0; i < RSLX_MUON_MAX_MATRICES; ++i) {
    t.first[grid][i] = i < count ? (int32_t)n : INT32_MAX;
    if (i < count) n += of(t.item[i]);
  }
  return (unsigned)n;
}

// Blocks of the shorter and of the longer side.
int short_blocks(const MuonItem& m) { return pad32(m.rows < m.cols ? m.rows : m.cols) / 32; }
int long_blocks(const MuonItem& m) { return pad32(m.rows < m.cols ? m.cols : m.rows) / 32; }

}  // namespace

size_t muon_item_bytes(int32_t rows, int32_t cols) {
  const size_t P = pad32(rows < cols ? rows : cols), Q = pad32(rows < cols ? cols : rows);
  return values_bytes(rows, cols) + MUON_NORM_BLOCKS * sizeof(double) + sizeof(uint16_t) * 2 * (3 * P * Q + 2 * P * P);
}

// Symmetric products go through the large tiles, in as many pieces as there are compute units for and of 16 stages of 32 contraction indices or more, where
// that takes less time than 64 x 64 tiles.  In stages of a large tile, both products together: the first the longest piece for each round over the compute units,
// and 16 for the sums' way through memory; the second 0.23 of a stage for each of a 64 x 64 tile on every compute unit.  Steps with and without large tiles, us:
// 1930 x 1930 715 and 645, 2048 x 2048 760 and 774, 2048 x 4096 1060 and 1168, 2304 x 2304 1054 and 1025, 2600 x 2600 1283 and 1358, 2700 x 2700 1665 and
// 1444, 3456 x 3456 2975 and 3107, 4096 x 4096 4913 and 4464, two of 1536 x 1536 700 and 662, ten of 1000 x 1024 1011 and 931, thirty-two of 600 x 610
// 1073 and 817.
// It is asked of the matrices from some short side on, of those that save most; the others of the call have launches of their own, which are worth 6 stages (2048 x
// 4096 with 30 x 100 1113, both in 64 x 64 tiles 1188).
size_t plan_muon_parts(MuonTable& t, int count) {
  int P[RSLX_MUON_MAX_MATRICES], Q[RSLX_MUON_MAX_MATRICES], least = 0;
  for (int i = 0; i < count; ++i) P[i] = short_blocks(t.item[i]), Q[i] = long_blocks(t.item[i]);
  int64_t taken = 0;
  double most = 0;
  t.pieces = 0;
  for (int i = 0; i < count; ++i) {
    if (P[i] < 16) continue;
    int64_t tiles = 0, longest = 0;
    double medium = 0;
    bool others = false;
    for (int j = 0; j < count; ++j) {
      if (P[j] < P[i]) {
        others = true;
        continue;
      }
      const int n = (P[j] + 1) / 2;
      tiles += wide_triangle_tiles(P[j]);
      medium += (double)n * (n + 1) / 2 * (P[j] + Q[j]);
    }
    const int64_t fill = tiles < 256 ? 256 / tiles : 1, pieces = fill < P[i] / 16 ? fill : P[i] / 16;
    for (int j = 0; j < count; ++j) {
      const int64_t stages = (P[j] + pieces - 1) / pieces + (Q[j] + pieces - 1) / pieces;
      if (P[j] >= P[i] && stages > longest) longest = stages;
    }
    const double saves = 0.23 * medium / 256 - (double)((tiles * pieces + 255) / 256 * longest + 16 + (others ? 6 : 0));
    if (saves < 0 || (least > 0 && saves <= most)) continue;
    least = P[i];
    most = saves;
    taken = tiles * pieces;
    t.pieces = (int32_t)pieces;
  }
  for (int i = 0; i < count; ++i) t.item[i].in_pieces = least > 0 && P[i] >= least;
  return (size_t)taken * PART;
}

// Tiles of high x wide blocks of a product with X.
static int64_t apply_tiles(const MuonItem& m, int high, int wide) {
  return (int64_t)((short_blocks(m) + high - 1) / high) * ((long_blocks(m) + wide - 1) / wide);
}

// Products with X take 256 x 128 tiles where these take less time than 64 x 64 ones, of the matrices from some short side on, whose take the least.  In stages of
// such a tile: the longest contraction for each round over the compute units; 0.197 of a stage for each of a 64 x 64 tile on every compute unit; 3 for a launch of
// others.  Steps with and without large tiles, us: 2048 x 2048 (128 of them) 830 and 760, 1500 x 3500 (168) 721 and 740, 2048 x 3000 (192) 924 and 970, 2048 x 4096
// (256) 1055 and 1193, 2900 x 2900 (276) 2158 and 1988, 3000 x 3000 (288) 2246 and 2122, 3200 x 3200 (325) 2539 and 2441, 3300 x 3300 (338) 2680 and 2700, 2600 x
// 4096 (352) 1876 and 1922, 3456 x 3456 (378) 2840 and 2983, 4096 x 3000 (384) 2492 and 2674.  2048 x 4096 with 30 x 100 in a launch of its own 1112, with 257 tiles
// 1373.
static void plan_muon_large(MuonTable& t, int count) {
  double most = 0;                                       // all of them in 64 x 64 tiles
  for (int i = 0; i < count; ++i) most += 0.197 / 256 * (double)apply_tiles(t.item[i], 2, 2) * short_blocks(t.item[i]);
  int least = INT32_MAX;
  for (int i = 0; i < count; ++i) {
    const int from = short_blocks(t.item[i]);
    if (from == least || from >= most) continue;         // (a round takes as many stages)
    int64_t tiles = 0;
    int longest = 0;
    double takes = 0;
    for (int j = 0; j < count; ++j) {
      const int P = short_blocks(t.item[j]);
      if (P < from) {
        takes += (takes == 0 ? 3 : 0) + 0.197 / 256 * (double)apply_tiles(t.item[j], 2, 2) * P;
      } else {
        tiles += apply_tiles(t.item[j], 8, 4);
        longest = P > longest ? P : longest;
      }
    }
    takes += (double)((tiles + 255) / 256 * longest);
    if (takes >= most) continue;
    least = from;
    most = takes;
  }
  for (int i = 0; i < count; ++i) t.item[i].large = short_blocks(t.item[i]) >= least;
}

hipError_t launch_muon(MuonTable& t, int count, MuonTable* in_workspace, int steps, hipStream_t stream) {
  plan_muon_large(t, count);
  // operations and bytes of products, of matrices that take large tiles in the second place
  double values = 0, planes = 0, gram[2] = {}, square[2] = {}, apply[2] = {}, gram_bytes[2] = {}, square_bytes[2] = {}, apply_bytes[2] = {};
  for (int i = 0; i < count; ++i) {
    const double rows = t.item[i].rows, cols = t.item[i].cols, p = rows < cols ? rows : cols, q = rows < cols ? cols : rows;
    const int k = t.item[i].in_pieces, l = t.item[i].large;
    values += p * q;
    planes += 4 * p * q;
    gram[k] += p * p * q;
    gram_bytes[k] += 4 * p * q + 4 * p * p;
    square[k] += p * p * p;
    square_bytes[k] += 8 * p * p;
    apply[l] += 2 * p * p * q;
    apply_bytes[l] += 4 * p * p + 12 * p * q;
  }
  // tiles of b x b blocks
  const auto symmetric_tiles = [](int b) {
    return [=](const MuonItem& m) {
      const int64_t n = (short_blocks(m) + b - 1) / b;
      return m.in_pieces ? 0 : n * (n + 1) / 2;
    };
  };
  const auto tiles_with_x = [](int high, int wide, bool large) {
    return [=](const MuonItem& m) { return large == (m.large != 0) ? apply_tiles(m, high, wide) : 0; };
  };
  // of those that are not in pieces or large: 64 x 64 tiles that are as many as the GPU has compute units, 32 x 32 where these are fewer.  Steps with the one and the
  // other, us: 896 x 896 (105 of a symmetric product, 196 with X) 167 and 152, 1024 x 1024 (136 and 256) 179 and 186, 1100 x 1100 (171 and 324) 232 and 216, 1400 x
  // 1400 (253 and 484) 293 and 341
  MuonShape symmetric_shape = MEDIUM, apply_shape = MEDIUM;
  const auto large_tiles = [](const MuonItem& m) { return m.in_pieces ? (int64_t)wide_triangle_tiles(short_blocks(m)) : 0; };
  const unsigned on_pieces = place_items(t, count, MUON_PIECES_GRID, [&](const MuonItem& m) { return large_tiles(m) * t.pieces; });
  const unsigned on_fold = place_items(t, count, MUON_FOLD_GRID, [&](const MuonItem& m) { return large_tiles(m) * 8; });
  unsigned on_symmetric = place_items(t, count, MUON_SYMMETRIC_GRID, symmetric_tiles(2)), on_apply = place_items(t, count, MUON_APPLY_GRID, tiles_with_x(2, 2, false));
  if (on_symmetric < 256) {
    symmetric_shape = SMALL;
    on_symmetric = place_items(t, count, MUON_SYMMETRIC_GRID, symmetric_tiles(1));
  }
  if (on_apply < 256) {
    apply_shape = SMALL;
    on_apply = place_items(t, count, MUON_APPLY_GRID, tiles_with_x(1, 1, false));
  }
  const unsigned on_large = place_items(t, count, MUON_LARGE_GRID, tiles_with_x(8, 4, true));
  const unsigned on_pack = place_items(t, count, MUON_PACK_GRID, [](const MuonItem& m) { return ((int64_t)short_blocks(m) * long_blocks(m) + 3) / 4; });
  const unsigned on_momentum = place_items(t, count, MUON_MOMENTUM_GRID, [](const MuonItem& m) { return (int64_t)norm_blocks(m.rows, m.cols); });
  {
    TraceScope trace(stream, "muon_momentum", 6 * values, 16 * values);
    hipLaunchKernelGGL(muon_momentum_kernel, dim3(on_momentum), dim3(ELEMENT_THREADS), 0, stream, t, in_workspace);
  }
  {
    TraceScope trace(stream, "muon_pack", values, 4 * values + 2 * planes);
    hipLaunchKernelGGL(muon_pack_kernel, dim3(on_pack), dim3(ELEMENT_THREADS), 0, stream, in_workspace);
  }
  auto tiles = [&](auto kind, MuonShape shape, unsigned groups, const char* name, double flops, double bytes, int turn) {
    constexpr MuonProduct KIND = decltype(kind)::value;
    const dim3 grid(groups);
    TraceScope trace(stream, name, flops, bytes);
    if (shape == SMALL) hipLaunchKernelGGL((muon_product_kernel<KIND, 1, 4>), grid, dim3(256), 0, stream, in_workspace, turn);
    else if (shape == MEDIUM) hipLaunchKernelGGL((muon_product_kernel<KIND, 2, 3>), grid, dim3(256), 0, stream, in_workspace, turn);
    else hipLaunchKernelGGL((muon_large_kernel<KIND>), grid, dim3(256), 0, stream, in_workspace, turn);
  };
  auto symmetric_product = [&](auto kind, const char* name, const double (&flops)[2], const double (&bytes)[2], int turn) {
    constexpr MuonProduct KIND = decltype(kind)::value;
    if (on_pieces > 0) {
      tiles(kind, LARGE, on_pieces, name, flops[1], bytes[1], turn);
      TraceScope trace(stream, "muon_fold", 0, 0);
      hipLaunchKernelGGL((muon_fold_kernel<KIND>), dim3(on_fold), dim3(256), 0, stream, in_workspace, turn);
    }
    if (on_symmetric > 0) tiles(kind, symmetric_shape, on_symmetric, name, flops[0], bytes[0], turn);
  };
  auto product_with_x = [&](auto kind, int turn) {
    if (on_large > 0) tiles(kind, LARGE, on_large, "muon_apply", apply[1], apply_bytes[1], turn);
    if (on_apply > 0) tiles(kind, apply_shape, on_apply, "muon_apply", apply[0], apply_bytes[0], turn);
  };
  for (int s = 0; s < steps; ++s) {
    symmetric_product(std::integral_constant<MuonProduct, MUON_GRAM>(), "muon_gram", gram, gram_bytes, s & 1);
    symmetric_product(std::integral_constant<MuonProduct, MUON_SQUARE>(), "muon_square", square, square_bytes, s & 1);
    if (s + 1 < steps) product_with_x(std::integral_constant<MuonProduct, MUON_APPLY>(), s & 1);
    else product_with_x(std::integral_constant<MuonProduct, MUON_LAST>(), s & 1);
  }
  return hipGetLastError();
}

}  // namespace rslx
