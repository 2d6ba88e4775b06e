// Linear attention with a decay for each head, gfx950: walks over sequences in chunks (forward pass and every gradient), the join of
// a long sequence's pieces, and the single step.
//
//   S_i = l S_{i-1} + b_i c_i^T,   o_i = scale S_i^T a_i,   l = exp(log_decay[h])
//
// A chunk of n = 16 positions (in 16-bit types 32: two blocks of 16) is four small products on the matrix cores: the scores P = A B^T, weighted by
// l^(i - j) below the diagonal, O = P C + l^(i + 1) A S, and S <- l^n S + (l^(n - 1 - j) B)^T C.  A wavefront walks one head of one sequence
// (16 DVT columns of it): the state stays in its accumulator registers, and because the order of a contraction's indices is free, nothing has to be
// moved between lanes.  With lane = 16 g + c, the instruction v_mfma_f32_16x16x4_f32 leaves in register r row 4 g + r of column c, and
// reads from an operand row (column) c at index g.  So
//   - the transposed scores B A^T leave P[c][4 g + r]: the left operand of P C if step s takes the contraction index 4 g + s;
//   - rows of state tiles are put to indices so that the state's registers are the right operand of A S as they are when lane (c, g) holds
//     4 DKT values of row c of A, taken 16 bytes at a time (place() below); and the left operand of the state's update is then, for all
//     tiles, DKT consecutive values of a row of B (two times four for fp32 keys of 128);
//   - column tile t is put to e = DVT c + t: C is read, and O written, DVT consecutive values of a row at a time.
// Rows pass through LDS on their way into those layouts, the next chunk's while this one is worked on: loaded into them straight from memory, 16
// rows an access, they take four times the cache accesses, and the caches bound the walk (8192 steps of 16 heads of 128 in bf16: 134 us;
// through LDS 118, with a workgroup's wavefronts sharing the rows of A and B 106, on one card).
//
// What bounds it now: a roll-out of 24 steps in fp32 (4096 environments, four heads of 64) memory, 192 us = 4.9 TB/s; long sequences in 16 bits
// (8192 steps of 16 heads of 128 in bf16: 89 us, three launches) the vector instructions that take the state and the weighted scores apart
// into bf16 values (some 700 a chunk of 32 beside 100 matrix instructions) and the latency of a chunk's loads at two wavefronts a SIMD, which
// their registers allow.  Long sequences of few heads are cut into pieces: one launch for every piece's own contribution to the state, one that
// joins them, one for the outputs.
#include <algorithm>

#include "sequence.h"
#include "split_bf16.h"
#include "typed.h"

namespace rslx {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Positions of a chunk: one block of 16, or two where the 16-bit matrix instructions contract over 32.
template <typename T> constexpr int BLOCKS = sizeof(T) == 2 ? 2 : 1;
constexpr int MOST_CHUNK = 32;
constexpr int WALK_WAVES = 4;           // wavefronts per workgroup
constexpr int64_t WALK_MAX_BLOCKS = 1 << 23;      // workgroups of a launch (2^31 threads); more take further launches

// N consecutive values as they lie in memory; converted where they are used.
template <typename T, int N> struct Frag {
  static constexpr int WORDS = N * (int)sizeof(T) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    const uint32_t x = w[i / 2];
    if constexpr (__is_same(T, bf16_t)) return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
    return __half2float(__ushort_as_half((unsigned short)(i & 1 ? x >> 16 : x)));
  }
};

// Memory is read through buffer descriptors: what lies past a row's end, or in a row that does not exist, is asked for at an offset
// beyond the descriptor's range and comes back as zero, without a branch and without a select; stores there are dropped.
// PIECE: bytes of one access (16; 4 and 2 where widths, strides or addresses are no multiples of 16), 0: rows too far apart for
// 32-bit offsets, value by value through 64-bit addresses.
constexpr uint32_t NOWHERE = 0x80000000u;
constexpr int64_t MAX_OFFSET = 0x7fff0000;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t Descriptor;

__device__ __forceinline__ Descriptor descriptor(const void* base, bool exists = true, int bytes = 0x7fffffff) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, exists ? bytes : 0, 0x00020000);
}

// The rows of a chunk, slot by slot; positions go up or down in memory.
template <int CHUNK> struct Rows {
  const char* low;               // of the row at the lowest address
  int64_t step;                  // bytes from a position to the next one, either sign
  __device__ __forceinline__ void move(int positions) { low += positions * step; }
  __device__ __forceinline__ int order(int slot) const { return step < 0 ? CHUNK - 1 - slot : slot; }
  __device__ __forceinline__ uint32_t at(int slot) const { return (uint32_t)order(slot) * (uint32_t)(step < 0 ? -step : step); }
  __device__ __forceinline__ const char* address(int slot) const { return low + (int64_t)order(slot) * (step < 0 ? -step : step); }
};
template <int CHUNK, typename T>
__device__ __forceinline__ Rows<CHUNK> rows_at(const T* first, int64_t step, int position) {
  const int64_t bytes = step * (int64_t)sizeof(T);
  return {reinterpret_cast<const char*>(first) + (position + (step < 0 ? CHUNK - 1 : 0)) * bytes, bytes};
}

// Where a lane's N values of a row of keys lie: 16 bytes, then 16 more behind those of the other three groups of lanes.  Value y of group g is at place(y) + PE g.
template <typename T> constexpr int PE16 = 16 / (int)sizeof(T);
template <typename T> __device__ __forceinline__ constexpr int place(int y) { return 4 * PE16<T> * (y / PE16<T>) + y % PE16<T>; }

// A value that the compiler does not know: what is made of it is neither kept from elsewhere nor made ahead of time (in registers that the
// products need).
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ float opaque(float x) {
  asm volatile("" : "+v"(x));
  return x;
}

// N values of a row from offset `at` on (or NOWHERE).  `there`: how many values the row has from there on; WHOLE: enough.
template <typename T, int N, int PIECE, bool WHOLE>
__device__ __forceinline__ void load_frag(Frag<T, N>& f, Descriptor d, uint32_t at, int there) {
  constexpr int WORDS = Frag<T, N>::WORDS, PB = PIECE < WORDS * 4 ? PIECE : WORDS * 4, PE = PB / (int)sizeof(T);
#pragma unroll
  for (int k = 0; k < N / PE; ++k) {
    const int o = (int)(WHOLE || k * PE < there ? at + (uint32_t)(k * PB) : NOWHERE);
    if constexpr (PB == 16) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(d, o, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) f.w[4 * k + i] = x[i];
    } else if constexpr (PB == 4) {
      f.w[k] = __builtin_amdgcn_raw_buffer_load_b32(d, o, 0, 0);
    } else {
      const uint32_t x = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(d, o, 0, 0);
      f.w[k / 2] = k % 2 ? f.w[k / 2] | x << 16 : x;
    }
  }
}
// N values of a row from value e0 on, one by one; zero where not `wanted`.  The row exists.
template <typename T, int N>
__device__ __forceinline__ void load_far(Frag<T, N>& f, const char* row, bool wanted, int e0, int width) {
#pragma unroll
  for (int k = 0; k < Frag<T, N>::WORDS; ++k) {
    f.w[k] = 0;
#pragma unroll
    for (int h = 0; h < 4 / (int)sizeof(T); ++h) {
      const int e = e0 + k * (4 / (int)sizeof(T)) + h;
      const bool here = wanted & (e < width);
      const int from = here ? e : 0;
      uint32_t x;
      if constexpr (sizeof(T) == 4) x = reinterpret_cast<const uint32_t*>(row)[from];
      else x = (uint32_t)reinterpret_cast<const uint16_t*>(row)[from] << (16 * h);
      f.w[k] |= here ? x : 0u;
    }
  }
}

// A chunk's rows on their way through LDS.  From memory a wavefront takes them as they lie there, LPR lanes of 16 bytes a row; from LDS,
// where rows are 16 bytes further apart (16 rows then start in 16 different groups of banks), every lane takes what the products want of it.
// WAVES wavefronts take a part of them each.
template <typename T, int LPR, int WAVES> struct Staged {
  static constexpr int CHUNK = 16 * BLOCKS<T>, STEP = 64 / LPR, COUNT = CHUNK / STEP / WAVES, STRIDE = 16 * LPR + 16, BYTES = CHUNK * STRIDE;
  Frag<T, PE16<T>> f[COUNT];
  static __device__ __forceinline__ int slot_of(int i, int lane, int wave) { return lane / LPR + (i * WAVES + wave) * STEP; }
  // The lane's 16 bytes of a row begin at value e0; slots below skip do not exist.
  template <int PIECE, bool WHOLE>
  __device__ __forceinline__ void load(const Rows<CHUNK>& m, int lane, int wave, int skip, bool exists, int e0, int width) {
    const uint32_t from = m.at(slot_of(0, lane, wave)) + e0 * (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const int slot = slot_of(i, lane, wave);
      if constexpr (PIECE != 0)
        load_frag<T, PE16<T>, PIECE, WHOLE>(f[i], descriptor(m.low, exists), slot >= skip ? from + (uint32_t)(i * WAVES * STEP * (int)m.step) : NOWHERE,
                                            width - e0);
      else if (exists) load_far<T, PE16<T>>(f[i], m.address(max(slot, skip)), slot >= skip, e0, width);
    }
  }
  __device__ __forceinline__ void store(char* lds, int lane, int wave) const {
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
      *reinterpret_cast<u32x4*>(lds + slot_of(i, lane, wave) * STRIDE + lane % LPR * 16) = u32x4{f[i].w[0], f[i].w[1], f[i].w[2], f[i].w[3]};
  }
  // Whether any value is infinite or NaN.
  __device__ __forceinline__ bool not_finite() const {
    if constexpr (sizeof(T) == 4) {
      float bad = 0.f;
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) bad = fmaf(f[i].get(k), 0.f, bad);
      return bad != 0.f;
    } else {
      // an exponent of ones carries into the sign's place
      constexpr uint32_t ONE = __is_same(T, __half) ? 0x04000400u : 0x00800080u;
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) bad |= (f[i].w[k] & 0x7fff7fffu) + ONE;
      return (bad & 0x80008000u) != 0;
    }
  }
};
// N values from LDS, in the order of place() where APART.
template <typename T, int N, bool APART>
__device__ __forceinline__ void take(Frag<T, N>& f, const char* p) {
  constexpr int WORDS = Frag<T, N>::WORDS;
  if constexpr (WORDS == 1) f.w[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (WORDS == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    f.w[0] = x[0];
    f.w[1] = x[1];
  } else {
#pragma unroll
    for (int k = 0; k < WORDS / 4; ++k) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + k * (APART ? 64 : 16));
#pragma unroll
      for (int i = 0; i < 4; ++i) f.w[4 * k + i] = x[i];
    }
  }
}
// What a wavefront's lanes wrote to its own LDS is there for all of them (its LDS accesses are carried out in order; the compiler keeps theirs).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <typename T, int N, int PIECE, bool WHOLE>
__device__ __forceinline__ void store_frag(Descriptor d, uint32_t at, int there, const float (&v)[N]) {
  constexpr int PB = PIECE < N * (int)sizeof(T) ? PIECE : N * (int)sizeof(T), PE = PB / (int)sizeof(T);
#pragma unroll
  for (int k = 0; k < N / PE; ++k) {
    const int o = (int)(WHOLE || k * PE < there ? at + (uint32_t)(k * PB) : NOWHERE);
    Pack<T, PE> p;
#pragma unroll
    for (int i = 0; i < PE; ++i) p.v[i] = from_float<T>(v[k * PE + i]);
    if constexpr (PB == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, p), d, o, 0, 0);
    else if constexpr (PB == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, p), d, o, 0, 0);
    else if constexpr (PB == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, p), d, o, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, p), d, o, 0, 0);
  }
}
// N values from value e0 on of one row, whose address all lanes have, in the order of place() where APART; zero past the row's width.
template <typename T, int N, bool APART>
__device__ __forceinline__ void load_row(Frag<T, N>& f, const char* row, int e0, int width) {
  const Descriptor d = descriptor(row, true, width * (int)sizeof(T));
  const int at = e0 * (int)sizeof(T);
#pragma unroll
  for (int y = 0; y < N; ++y) {
    const int o = at + (APART ? place<T>(y) : y) * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) {
      f.w[y] = __builtin_amdgcn_raw_buffer_load_b32(d, o, 0, 0);
    } else {
      const uint32_t x = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(d, o, 0, 0);
      f.w[y / 2] = y % 2 ? f.w[y / 2] | x << 16 : x;
    }
  }
}

// N values of one row, whose address all lanes have, one by one.  Values past the row's width lie beyond the descriptor's range, and so do
// those of a lane that has none `wanted`.
template <typename T, int N>
__device__ __forceinline__ void store_far(const char* row, bool wanted, int e0, int width, const float (&v)[N]) {
  const Descriptor d = descriptor(row, true, width * (int)sizeof(T));
  const uint32_t at = wanted ? (uint32_t)(e0 * (int)sizeof(T)) : NOWHERE;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int o = (int)(at + (uint32_t)(i * (int)sizeof(T)));
    const T x = from_float<T>(v[i]);
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), d, o, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, x), d, o, 0, 0);
  }
}

// N values of a state, BYTES at a time.
template <int N, int BYTES>
__device__ __forceinline__ void load_state(float (&v)[N], Descriptor d, const uint32_t (&at)[N]) {
#pragma unroll
  for (int k = 0; k < N; k += BYTES / 4) {
    if constexpr (BYTES == 16) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(d, (int)at[k], 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k + i] = __uint_as_float(x[i]);
    } else if constexpr (BYTES == 8) {
      const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(d, (int)at[k], 0, 0);
      v[k] = __uint_as_float(x[0]);
      v[k + 1] = __uint_as_float(x[1]);
    } else {
      v[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(d, (int)at[k], 0, 0));
    }
  }
}

// 2^(l2 n), l2 = log2 of the decay: the exponent is formed in 64 bits, so the error is the last bit's however far the position.
__device__ __forceinline__ float decay_pow(double l2, int n) {
  double x = l2 * (double)n;
  x = x < -2000.0 ? -2000.0 : x;
  const double k = rint(x);
  return ldexpf(exp2f((float)(x - k)), (int)k);
}
// A decay of zero (log -inf) stays one: times a distance of zero it must not become NaN.
__device__ __forceinline__ double log2_decay(float log_decay) {
  const double l = log_decay < -10000.f ? -10000.0 : (double)log_decay;
  return l * 1.4426950408889634074;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int sequence_length(const WalkArgs& w, int n) {
  return w.lengths ? min(max(w.lengths[n], 0), w.T) : w.T;
}

// ---- the four products of a chunk ---------------------------------------------------------------------------------
// fp32 operands: fp32 matrix instructions, one block of 16 positions.
//
// 16-bit operands: v_mfma_f32_16x16x32, two blocks.  Its operands hold eight contraction indices a lane, and again any order will do: of
// the widths, the lane's 4 DKT consecutive values as they lie in memory, eight by eight (value DKT r + a is row r of state tile a: pairs
// of tiles fill a register); of the positions, 4 g + s of the first block, then of the second.  What is exact in 16 bits is multiplied as it
// is; what is not (weighted scores, the state, the weighted C) is taken apart into bf16 values: two for results that are rounded to 16
// bits (what is left out is 2^-17 of a term at most, where that rounding is 2^-8 or 2^-11 of the result), three, as many bits as fp32 has, for
// what is added to the state.  fp16 inputs reach products with such parts as two bf16 values of their own, which hold them exactly; the
// product of the two second parts is left out (2^-16 of a term at most).
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> constexpr int PARTS = __is_same(T, __half) ? 2 : 1;      // bf16 values that make an input

__device__ __forceinline__ f32x4 mfma_bf16(const uint32_t* a, const uint32_t* b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, (u32x4){a[0], a[1], a[2], a[3]}),
                                                 __builtin_bit_cast(bf16x8, (u32x4){b[0], b[1], b[2], b[3]}), c, 0, 0, 0);
}
__device__ __forceinline__ float low_half(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_half(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// Two fp32 values as COUNT packed bf16 values each.
template <int COUNT>
__device__ __forceinline__ void parts_of(float x, float y, uint32_t (&p)[COUNT]) {
#pragma unroll
  for (int k = 0; k < COUNT; ++k) {
    p[k] = pack_bf16(x, y);
    if (k + 1 < COUNT) {
      x -= low_half(p[k]);
      y -= high_half(p[k]);
    }
  }
}
// A register of two inputs as bf16 parts.
template <typename T>
__device__ __forceinline__ void input_parts(uint32_t x, uint32_t (&p)[PARTS<T>]) {
  if constexpr (PARTS<T> == 1) p[0] = x;
  else parts_of<2>(__half2float(__ushort_as_half((unsigned short)x)), __half2float(__ushort_as_half((unsigned short)(x >> 16))), p);
}
// The low (HIGH = 0) or high halves of x and y side by side.
template <int HIGH> __device__ __forceinline__ uint32_t halves(uint32_t x, uint32_t y) {
  return __builtin_amdgcn_perm(y, x, HIGH ? 0x07060302u : 0x05040100u);
}
// Values i of four rows of each block, position by position, as an operand of eight.
template <typename T, int N>
__device__ __forceinline__ void column(const Frag<T, N> (&f)[2][4], int i, uint32_t (&x)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t u = f[k / 2][2 * (k % 2)].w[i / 2], v = f[k / 2][2 * (k % 2) + 1].w[i / 2];
    x[k] = i % 2 ? halves<1>(u, v) : halves<0>(u, v);
  }
}

// Transposed scores of a block: P[j][i] at register r of lane (i = c, g), j = 4 g + r.
template <typename T, int DKT>
__device__ __forceinline__ f32x4 scores(const Frag<T, 4 * DKT>& b, const Frag<T, 4 * DKT>& a) {
  f32x4 p = {0.f, 0.f, 0.f, 0.f};
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int x = 0; x < 4 * DKT; ++x) p = __builtin_amdgcn_mfma_f32_16x16x4f32(b.get(x), a.get(x), p, 0, 0, 0);
  } else {
#pragma unroll
    for (int x = 0; x < 2 * DKT; x += 4) {
      const u32x4 u = {b.w[x], b.w[x + 1], b.w[x + 2], b.w[x + 3]}, v = {a.w[x], a.w[x + 1], a.w[x + 2], a.w[x + 3]};
      if constexpr (__is_same(T, bf16_t)) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u), __builtin_bit_cast(bf16x8, v), p, 0, 0, 0);
      else p = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, u), __builtin_bit_cast(f16x8, v), p, 0, 0, 0);
    }
  }
  return p;
}

// o += A S
template <typename T, int DKT, int DVT>
__device__ __forceinline__ void read_state(f32x4 (&o)[BLOCKS<T>][DVT], const Frag<T, 4 * DKT> (&fa)[BLOCKS<T>], const f32x4 (&S)[DKT][DVT]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int a = 0; a < DKT; ++a)
#pragma unroll
        for (int t = 0; t < DVT; ++t) o[0][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[0].get(DKT * s + a), S[a][t][s], o[0][t], 0, 0, 0);
  } else {
#pragma unroll
    for (int k = 0; k < 2 * DKT; k += 4) {
      uint32_t x[2][PARTS<T>][4];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t p[PARTS<T>];
          input_parts<T>(fa[b].w[k + i], p);
#pragma unroll
          for (int j = 0; j < PARTS<T>; ++j) x[b][j][i] = p[j];
        }
#pragma unroll
      for (int t = 0; t < DVT; ++t) {
        uint32_t y[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 2 * (k + i) / DKT, a = 2 * (k + i) % DKT;
          uint32_t p[2];
          parts_of<2>(S[a][t][r], S[a + 1][t][r], p);
          y[0][i] = p[0];
          y[1][i] = p[1];
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < PARTS<T>; ++i)
#pragma unroll
            for (int j = 0; j < 2 - i; ++j) o[b][t] = mfma_bf16(x[b][i], y[j], o[b][t]);
      }
    }
  }
}

// o += P C
template <typename T, int DVT>
__device__ __forceinline__ void add_values(f32x4 (&o)[BLOCKS<T>][DVT], const f32x4 (&P)[BLOCKS<T>][BLOCKS<T>], const Frag<T, DVT> (&fv)[BLOCKS<T>][4]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int t = 0; t < DVT; ++t) o[0][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(P[0][0][s], fv[0][s].get(t), o[0][t], 0, 0, 0);
  } else {
    uint32_t x[2][2][4];                   // [block of i][part]
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t p[2] = {0u, 0u};
        if (k / 2 <= b) parts_of<2>(P[k / 2][b][2 * (k % 2)], P[k / 2][b][2 * (k % 2) + 1], p);
        x[b][0][k] = p[0];
        x[b][1][k] = p[1];
      }
#pragma unroll
    for (int t = 0; t < DVT; ++t) {
      uint32_t v[4], y[PARTS<T>][4];
      column<T, DVT>(fv, t, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t p[PARTS<T>];
        input_parts<T>(v[k], p);
#pragma unroll
        for (int j = 0; j < PARTS<T>; ++j) y[j][k] = p[j];
      }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < PARTS<T> && i + j < 2; ++j) o[b][t] = mfma_bf16(x[b][i], y[j], o[b][t]);
    }
  }
}

// S += (weighted B)^T C; a position whose episode ends inside the chunk leaves nothing.
template <typename T, int DKT, int DVT>
__device__ __forceinline__ void add_state(f32x4 (&S)[DKT][DVT], const Frag<T, DKT> (&fk)[BLOCKS<T>][4], const Frag<T, DVT> (&fv)[BLOCKS<T>][4],
                                          const float (&wk)[BLOCKS<T>][4], uint32_t cut, int g) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const bool stays = (cut >> (4 * g + s)) == 0;
#pragma unroll
      for (int a = 0; a < DKT; ++a) {
        const float k = stays ? fk[0][s].get(a) * wk[0][s] : 0.f;
#pragma unroll
        for (int t = 0; t < DVT; ++t) S[a][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k, fv[0][s].get(t), S[a][t], 0, 0, 0);
      }
    }
  } else {
    uint32_t y[DVT][3][4], mask[4];
#pragma unroll
    for (int t = 0; t < DVT; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int b = k / 2, s = 2 * (k % 2);
        uint32_t p[3];
        parts_of<3>(fv[b][s].get(t) * wk[b][s], fv[b][s + 1].get(t) * wk[b][s + 1], p);
#pragma unroll
        for (int j = 0; j < 3; ++j) y[t][j][k] = p[j];
      }
    if (cut) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = 16 * (k / 2) + 4 * g + 2 * (k % 2);
        mask[k] = ((cut >> i) == 0 ? 0xffffu : 0u) | ((cut >> (i + 1)) == 0 ? 0xffff0000u : 0u);
      }
    }
#pragma unroll
    for (int a = 0; a < DKT; ++a) {
      uint32_t v[4], x[PARTS<T>][4];
      column<T, DKT>(fk, a, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t p[PARTS<T>];
        input_parts<T>(cut ? v[k] & mask[k] : v[k], p);
#pragma unroll
        for (int i = 0; i < PARTS<T>; ++i) x[i][k] = p[i];
      }
#pragma unroll
      for (int t = 0; t < DVT; ++t)
#pragma unroll
        for (int i = 0; i < PARTS<T>; ++i)
#pragma unroll
          for (int j = 0; j < 3 - i; ++j) S[a][t] = mfma_bf16(x[i], y[t][j], S[a][t]);
    }
  }
}

// SHARED: the wavefronts of a workgroup are the tiles of one head's columns and take the rows of A and B together: a fourth of the loads and of the
// registers for them.  LDS then holds two chunks of A and B, so that one barrier a chunk is enough; a wavefront beyond the last column
// helps with the loads.
template <typename T, int DKT, int DVT, int PIECE, bool WHOLE, bool STATES, bool SHARED>
__global__ __launch_bounds__(64 * WALK_WAVES, DKT * DVT > 16 ? 1 : 2) void walk_kernel(WalkArgs w, int tiles, int first_block) {
  constexpr int NB = BLOCKS<T>, CHUNK = 16 * NB;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = uniform((int)(threadIdx.x >> 6));
  const int block = first_block + (int)blockIdx.x;
  int item = SHARED ? block : block * WALK_WAVES + wave;
  const int pieces = STATES ? w.segments - 1 : w.segments;
  const int ji = item % w.jobs; item /= w.jobs;
  const int tile = SHARED ? wave : item % tiles;
  if (!SHARED) item /= tiles;
  const int h = item % w.H; item /= w.H;
  const int n = item % w.N, piece = item / w.N;
  if (piece >= pieces) return;
  const WalkJob& job = w.job[ji];
  const int D = job.D, E = job.E, e_tile = tile * 16 * DVT, e_lane = e_tile + DVT * c;
  const bool idle = e_tile >= E;
  if (!SHARED && idle) return;
  const bool rev = job.reversed != 0;
  const int lead = rev ? 0 : 1;
  const int len = uniform(sequence_length(w, n));
  const int p0 = min(piece * w.seg_len, len), p1 = p0 + min(w.seg_len, len - p0);
  // The first chunk is the one that may be short: it fills the last slots, so that the weights towards the state behind a chunk are
  // the same for every chunk.
  const int chunks = (p1 - p0 + CHUNK - 1) / CHUNK;
  int skip = chunks * CHUNK - (p1 - p0);
  int at = p0 - skip;                     // position of the chunk's slot 0
  const int64_t first = rev ? len - 1 : 0, dir = rev ? -1 : 1;
  auto rows = [&](const WalkMatrix& m) {
    return rows_at<CHUNK>(static_cast<const T*>(m.p) + n * m.seq + h * m.head + first * m.step, dir * m.step, at);
  };
  Rows<CHUNK> A{}, O{}, B = rows(job.b), C = rows(job.c);
  if constexpr (!STATES) {
    A = rows(job.a);
    O = rows(job.o);
  }

  // The rows of a chunk are asked for while the one before it is worked on.
  constexpr int SIZE = (int)sizeof(T), K_LANES = DKT * SIZE, V_LANES = DVT * SIZE;
  using Keys = Staged<T, K_LANES, SHARED ? WALK_WAVES : 1>;
  using Values = Staged<T, V_LANES, 1>;
  constexpr int KEYS = (STATES ? 1 : 2) * Keys::BYTES;      // of B and A
  __shared__ __attribute__((aligned(16))) char lds_keys[(SHARED ? 2 : WALK_WAVES) * KEYS], lds_values[WALK_WAVES * Values::BYTES];
  __shared__ int lds_bad[2][WALK_WAVES];
  const int k_wave = SHARED ? wave : 0;
  char* lds_b = lds_keys + (SHARED ? 0 : wave * KEYS);
  char* const lds_c = lds_values + wave * Values::BYTES;
  Keys sa, sb;
  Values sc;
  uint32_t end = 0;
  // row c = 4 (c / 4) + c % 4 of state tile a is index place(DKT (c % 4) + a) + PE (c / 4): the first of this lane's DKT values for the state
  const int d_col = place<T>(DKT * (c & 3)) + PE16<T> * (c >> 2);
  const uint32_t at_o = O.at(4 * g) + e_lane * SIZE;
  auto load = [&](int first_slot, int at, bool exists) {
    const int k0 = opaque(lane % K_LANES * PE16<T>), v0 = opaque(e_tile + lane % V_LANES * PE16<T>);
    if (w.dones && exists) {
      const int t = rev ? len - 2 - at - lane : at + lane;
      end = w.dones[(int64_t)min(max(t, 0), len - 1) * w.N + n];
    }
    sb.template load<PIECE, WHOLE>(B, lane, k_wave, first_slot, exists, k0, D);
    sc.template load<PIECE, WHOLE>(C, lane, 0, first_slot, exists && !idle, v0, E);
    if constexpr (!STATES) sa.template load<PIECE, WHOLE>(A, lane, k_wave, first_slot, exists, k0, D);
  };
  load(skip, at, chunks > 0);

  f32x4 S[DKT][DVT];
#pragma unroll
  for (int a = 0; a < DKT; ++a)
#pragma unroll
    for (int t = 0; t < DVT; ++t) S[a][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  bool live = false;                      // the state may be other than zero
  if (!STATES && job.s_in != nullptr && !(w.segments == 1 && rev && len > 0 && w.dones && w.dones[(int64_t)(len - 1) * w.N + n])) {
    live = true;
    const int g = opaque(lane >> 4), c = opaque(lane & 15), e_lane = e_tile + DVT * c;
    const Descriptor d = descriptor(job.s_in + (((int64_t)n * w.H + h) * w.segments + piece) * D * E, true, D * E * 4);
    if (job.in_col == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int a = 0; a < DKT; ++a) {
          float v[DVT];
          uint32_t o[DVT];
#pragma unroll
          for (int t = 0; t < DVT; ++t) o[t] = e_lane + t < E ? (uint32_t)((place<T>(DKT * i + a) + PE16<T> * g) * E + e_lane + t) * 4 : NOWHERE;
          if (E % DVT == 0) load_state<DVT, DVT * 4>(v, d, o);
          else load_state<DVT, 4>(v, d, o);
#pragma unroll
          for (int t = 0; t < DVT; ++t) S[a][t][i] = v[t];
        }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < DVT; ++t) {
          float v[DKT];
          uint32_t o[DKT];
#pragma unroll
          for (int a = 0; a < DKT; ++a) {
            const int x = place<T>(DKT * i + a) + PE16<T> * g;
            o[a] = x < D ? (uint32_t)((e_lane + t) * D + x) * 4 : NOWHERE;
          }
          if (D % (DKT < 4 ? DKT : 4) == 0) load_state<DKT, (DKT < 4 ? DKT : 4) * 4>(v, d, o);
          else load_state<DKT, 4>(v, d, o);
#pragma unroll
          for (int a = 0; a < DKT; ++a) S[a][t][i] = v[a];
        }
    }
  }

  // Weights inside a chunk (in a block, and of the second block's positions for the first's), of the state before it, and towards the state
  // behind it.  A lane's four positions of a block are one apart: where no weight ends on the way, one is kept and the others are made of it.
  const double l2 = log2_decay(w.log_decay[h]);
  const float b_scale = rev ? w.scale : 1.f, o_scale = rev ? 1.f : w.scale;
  float step[4], wp[4], wp_next, wq[NB], wk[NB];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    step[r] = __uint_as_float(uniform(__float_as_uint(decay_pow(l2, r))));
    // (No branch that only some lanes take may stand in this kernel: where registers are short the compiler stores some at such a branch's
    // end while lanes are still switched off, and gives those lanes stale values back.  Lanes that have nothing to load or store do it
    // out of range, or all the same; tests/test_kernel_listing.py looks for instructions that switch lanes off.)
    const float x = w.scale * decay_pow(l2, max(c - 4 * g - r, 0));
    wp[r] = c >= 4 * g + r ? x : 0.f;
  }
  wp_next = w.scale * decay_pow(l2, 16 + c - 4 * g - 3);             // (times step[3 - r])
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    wq[b] = o_scale * decay_pow(l2, 16 * b + 4 * g + lead);          // (times step[r])
    wk[b] = b_scale * decay_pow(l2, CHUNK - lead - 16 * b - 4 * g - 3);    // (times step[3 - r])
  }
  // The state is multiplied by l^CHUNK once a chunk.  Rounded to one float, that would err the same way every time (up to 6e-8 a chunk); so it
  // is one of the two floats beside the number, the upper one as often as the number lies towards it: the product of any chunks in a row
  // is off by one step of fp32 at most, however many they are.
  const double chunk_decay = exp2(l2 * CHUNK);
  const float nearest = (float)chunk_decay;
  const bool between = nearest < 1e30f;
  const uint32_t keep_low = uniform(__float_as_uint(nearest) - ((between & ((double)nearest > chunk_decay)) ? 1 : 0));
  // (floats beside each other are 2^(E - 150) apart, E the exponent's bits, at least 1)
  const uint32_t keep_rise = uniform(between ? (uint32_t)ldexp(chunk_decay - (double)__uint_as_float(keep_low), 182 - max((int)(keep_low >> 23), 1)) : 0u);
  uint32_t keep_turn = 0x80000000u;
  float keep = decay_pow(l2, CHUNK - skip);
  // The bf16 matrix instructions cut what they add off downwards (see split_bf16.h), which would add up over the chunks of a long memory (a
  // state of 20 000 steps came out low by 2e-7 of its rms in bf16, 6e-7 in fp16): the state changes its sign with every chunk.
  constexpr bool TURNS = sizeof(T) == 2;
  // (Pieces' own states, which start at zero, end with their own sign.)
  uint32_t sign = TURNS && STATES && chunks % 2 ? 0x80000000u : 0u;      // of the state before the chunk
  if constexpr (TURNS) {
    keep = -keep;
#pragma unroll
    for (int b = 0; b < NB; ++b) wk[b] = -wk[b];
  }
  auto turned = [&](float x) { return TURNS ? __uint_as_float(__float_as_uint(x) ^ sign) : x; };

  const bool wants_state = STATES || (job.s_out != nullptr && piece == w.segments - 1);
  bool any_cut = false;
  int careful = p1;                       // positions from here on are taken one by one
  for (int q = 0; q < chunks; ++q) {
    const bool more = q + 1 < chunks;
    const int skip_now = skip;
    skip = 0;                             // of the next chunk
    // bit i: an episode ends between slots i and i + 1
    uint32_t cut = 0;
    if (w.dones) cut = (uint32_t)__ballot((lane < CHUNK) & (lane >= skip_now) & (end != 0) & !(rev & (at + lane >= len - 1)));
    bool bad = __any(sc.not_finite());
    if constexpr (SHARED) lds_b = lds_keys + (q & 1) * KEYS;
    char* const lds_a = lds_b + Keys::BYTES;
    sb.store(lds_b, lane, k_wave);
    sc.store(lds_c, lane, 0);
    if constexpr (!STATES) sa.store(lds_a, lane, k_wave);
    if constexpr (SHARED) {
      lds_bad[q & 1][wave] = bad ? 1 : 0;
      __syncthreads();
      bad = false;
#pragma unroll
      for (int i = 0; i < WALK_WAVES; ++i) bad |= uniform(lds_bad[q & 1][i]) != 0;
    } else {
      wave_fence();
    }
    // A position's weight for an earlier or later one that it has nothing to do with is zero, but zero times infinity is not: from a chunk
    // on whose C holds anything that is not finite, positions are taken one by one, as the recurrence has them.
    if (bad) {
      careful = at + skip_now;
      break;
    }
    B.move(CHUNK);
    C.move(CHUNK);
    if constexpr (!STATES) A.move(CHUNK);
    load(0, at + CHUNK, more);
    if (SHARED && idle) {
      at += CHUNK;
      continue;
    }
    f32x4 o[NB][DVT];
    f32x4 P[NB][NB];                      // [block of j][block of i]
    if constexpr (!STATES) {
      Frag<T, 4 * DKT> fa[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) take<T, 4 * DKT, true>(fa[b], lds_a + (16 * b + c) * Keys::STRIDE + 16 * g);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        Frag<T, 4 * DKT> fb;
        take<T, 4 * DKT, true>(fb, lds_b + (16 * j + c) * Keys::STRIDE + 16 * g);
#pragma unroll
        for (int i = j; i < NB; ++i) P[j][i] = scores<T, DKT>(fb, fa[i]);
      }
      __builtin_amdgcn_sched_barrier(0);    // (operands are taken from LDS when they are needed: registers are what is short)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < DVT; ++t) o[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (live) {
        read_state<T, DKT, DVT>(o, fa, S);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = q == 0 ? o_scale * decay_pow(l2, max(16 * b + 4 * g + r - skip_now, 0) + lead) : opaque(wq[b]) * turned(step[r]);
#pragma unroll
            for (int t = 0; t < DVT; ++t) o[b][t][r] *= x;
          }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j <= i; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) P[j][i][r] = j < i ? P[j][i][r] * (opaque(wp_next) * step[3 - r]) : c >= 4 * g + r ? P[j][i][r] * wp[r] : 0.f;
    }
    if constexpr (!STATES) {
      if (cut) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = 16 * b + 4 * g + r;
#pragma unroll
            for (int t = 0; t < DVT; ++t) o[b][t][r] = (cut & ((1u << i) - 1u)) == 0 ? o[b][t][r] : 0.f;
            // here i is the earlier position
#pragma unroll
            for (int x = b; x < NB; ++x) P[b][x][r] = ((cut >> i) & ((1u << ((16 * x + c - i) & 31)) - 1u)) == 0 ? P[b][x][r] : 0.f;
          }
      }
    }

    Frag<T, DVT> fv[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) take<T, DVT, false>(fv[b][i], lds_c + (16 * b + 4 * g + i) * Values::STRIDE + DVT * c * SIZE);
    if constexpr (!STATES) {
      add_values<T, DVT>(o, P, fv);
      const uint32_t from_o = opaque((int)at_o);
      const int there_o = opaque(E - e_lane);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int slot = 16 * b + 4 * g + r;
          float v[DVT];
#pragma unroll
          for (int t = 0; t < DVT; ++t) v[t] = o[b][t][r];
          if constexpr (PIECE != 0)
            store_frag<T, DVT, PIECE, WHOLE>(descriptor(O.low), slot >= skip_now ? from_o + (uint32_t)((16 * b + r) * (int)O.step) : NOWHERE, there_o, v);
          else
#pragma unroll
            for (int x = 0; x < 4; ++x) store_far<T, DVT>(O.address(16 * b + 4 * x + r), (g == x) & (slot >= skip_now), e_lane, E, v);
        }
      O.move(CHUNK);
    }
    if (!more && !wants_state) break;       // nobody reads the state behind the last chunk
    if (live) {
      if (cut) {                           // (a state that is not finite ends with its episode too)
#pragma unroll
        for (int a = 0; a < DKT; ++a)
#pragma unroll
          for (int t = 0; t < DVT; ++t) S[a][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      } else {
#pragma unroll
        for (int a = 0; a < DKT; ++a)
#pragma unroll
          for (int t = 0; t < DVT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[a][t][r] *= keep;
      }
    }
    Frag<T, DKT> fk[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) take<T, DKT, true>(fk[b][i], lds_b + (16 * b + 4 * g + i) * Keys::STRIDE + d_col * SIZE);
    float weight[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) weight[b][r] = opaque(wk[b]) * turned(step[3 - r]);
    add_state<T, DKT, DVT>(S, fk, fv, weight, cut, g);
    live = true;
    wave_fence();
    at += CHUNK;
    if constexpr (STATES) any_cut |= cut != 0;
    keep_turn += keep_rise;               // (a carry out of 32 bits: the upper one)
    keep = __uint_as_float(keep_low + (keep_turn < keep_rise ? 1u : 0u));
    if constexpr (TURNS) {
      keep = -keep;
      sign ^= 0x80000000u;
    }
  }
  if (sign && (wants_state || careful < p1)) {
#pragma unroll
    for (int a = 0; a < DKT; ++a)
#pragma unroll
      for (int t = 0; t < DVT; ++t) S[a][t] = -S[a][t];
  }

  if (careful < p1) {
    const int g = opaque(lane >> 4), c = opaque(lane & 15), e_lane = e_tile + DVT * c;
    const float l1 = decay_pow(l2, 1);
    at = STATES ? uniform(careful) : careful;      // (without outputs the compiler does not see that it is the same for all lanes)
    Rows<CHUNK> a{}, b = rows(job.b), z = rows(job.c), out{};
    if constexpr (!STATES) {
      a = rows(job.a);
      out = rows(job.o);
    }
    for (; at < p1; ++at) {
      const int t = rev ? len - 2 - at : at;
      const bool cut = w.dones && t >= 0 && w.dones[(int64_t)t * w.N + n] != 0;
      Frag<T, 4 * DKT> xa, xb;
      Frag<T, DVT> xc;
      load_row<T, 4 * DKT, true>(xb, b.address(0), PE16<T> * g, D);
      load_row<T, DVT, false>(xc, z.address(0), e_lane, E);
      if constexpr (!STATES) load_row<T, 4 * DKT, true>(xa, a.address(0), PE16<T> * g, D);
      float sum[DVT] = {};
#pragma unroll
      for (int x = 0; x < DKT; ++x)
#pragma unroll
        for (int t = 0; t < DVT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float v = fmaf(xb.get(DKT * r + x) * b_scale, xc.get(t), rev ? S[x][t][r] : S[x][t][r] * l1);
            if constexpr (!STATES) sum[t] = fmaf(xa.get(DKT * r + x), v, sum[t]);
            if (rev) v *= l1;
            S[x][t][r] = cut ? 0.f : v;
          }
      if constexpr (!STATES) {
#pragma unroll
        for (int t = 0; t < DVT; ++t) {
          sum[t] += __shfl_xor(sum[t], 16, 64);
          sum[t] = (sum[t] + __shfl_xor(sum[t], 32, 64)) * o_scale;
        }
        store_far<T, DVT>(out.address(0), lane < 16, e_lane, E, sum);
        a.move(1);
        out.move(1);
      }
      b.move(1);
      z.move(1);
      if constexpr (STATES) any_cut |= cut;
    }
  }

  if (wants_state) {
    const int g = opaque(lane >> 4), c = opaque(lane & 15), e_lane = e_tile + DVT * c;
    const Descriptor d = descriptor(job.s_out + (((int64_t)n * w.H + h) * (STATES ? w.segments : 1) + (STATES ? piece + 1 : 0)) * D * E, true, D * E * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int a = 0; a < DKT; ++a) {
        float v[DVT];
#pragma unroll
        for (int t = 0; t < DVT; ++t) v[t] = S[a][t][i];
        const uint32_t o = (uint32_t)((place<T>(DKT * i + a) + PE16<T> * g) * E + e_lane) * 4;
        if (E % DVT == 0) store_frag<float, DVT, 16, false>(d, o, E - e_lane, v);
        else store_frag<float, DVT, 4, false>(d, o, E - e_lane, v);
      }
  }
  if constexpr (STATES) {
    if (w.cuts && h == 0 && tile == 0) w.cuts[((int64_t)ji * w.N + n) * w.segments + piece] = any_cut ? 1 : 0;
  } else {
    if (SHARED && idle) return;
    // steps that do not exist: zero
    const float zero[DVT] = {};
    const int t0 = max(len, piece * w.seg_len), t1 = piece == w.segments - 1 ? w.T : min((piece + 1) * w.seg_len, w.T);
    Rows<CHUNK> Z = rows_at<CHUNK>(static_cast<const T*>(job.o.p) + n * job.o.seq + h * job.o.head, job.o.step, t0);
    for (int t = t0; t < t1; t += 16, Z.move(16))
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool exists = 4 * g + r < t1 - t;
        if constexpr (PIECE != 0) store_frag<T, DVT, PIECE, WHOLE>(descriptor(Z.low), exists ? Z.at(4 * g + r) + e_lane * SIZE : NOWHERE, E - e_lane, zero);
        else
#pragma unroll
          for (int x = 0; x < 4; ++x) store_far<T, DVT>(Z.address(4 * x + r), (g == x) & exists, e_lane, E, zero);
      }
  }
}

// One thread per element of a head's state: slot 0 takes the start, then every slot what it adds to the decayed one before it.  A piece's decay
// is two floats, so that its rounding does not add up over hundreds of pieces (a state that is not finite needs no second one).
constexpr int JOIN_MAX = 512;
struct JoinStarts { const float* start[WALK_MAX_JOBS]; };
__global__ __launch_bounds__(256) void walk_join_kernel(WalkArgs w, JoinStarts starts) {
  __shared__ float f[JOIN_MAX], f_rest[JOIN_MAX];
  __shared__ int cut[JOIN_MAX];
  const int ji = blockIdx.z, n = blockIdx.x / w.H, h = blockIdx.x % w.H;
  const WalkJob& job = w.job[ji];
  const int len = sequence_length(w, n);
  const double l2 = log2_decay(w.log_decay[h]);
  // The first slots are on their way while the decays are made.
  const int size = job.D * job.E, e = min((int)(blockIdx.y * 256 + threadIdx.x), size - 1);
  const bool here = (int)(blockIdx.y * 256 + threadIdx.x) < size;
  const int64_t head = (int64_t)n * w.H + h;
  float* slot = job.s_out + head * w.segments * size + e;
  constexpr int AHEAD = 8;
  float x[AHEAD];
  auto load = [&](int m0) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) x[k] = slot[(int64_t)(min(m0 + k, w.segments - 2) + 1) * size];
  };
  load(0);
  float run = starts.start[ji] ? starts.start[ji][head * size + e] : 0.f;
  if (job.reversed && len > 0 && w.dones && w.dones[(int64_t)(len - 1) * w.N + n]) run = 0.f;
  for (int m = threadIdx.x; m < w.segments - 1; m += 256) {
    const double decay = exp2(l2 * (double)min(max(len - m * w.seg_len, 0), w.seg_len));
    f[m] = (float)decay;
    f_rest[m] = f[m] < 1e30f ? (float)(decay - (double)f[m]) : 0.f;
    cut[m] = w.cuts[((int64_t)ji * w.N + n) * w.segments + m];
  }
  __syncthreads();
  if (!here) return;
  slot[0] = run;
  for (int m0 = 0; m0 < w.segments - 1; m0 += AHEAD) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (m0 + k >= w.segments - 1) break;
      const float finite = fabsf(run) < 3.4e38f ? run : 0.f;
      run = cut[m0 + k] ? x[k] : fmaf(run, f[m0 + k], fmaf(finite, f_rest[m0 + k], x[k]));
      slot[(int64_t)(m0 + k + 1) * size] = run;
    }
    if (m0 + AHEAD < w.segments - 1) load(m0 + AHEAD);
  }
}

// ---- one step -----------------------------------------------------------------------------------------------------
// S <- l S + k v^T, o = scale S^T q: the state is read and written once, four columns a lane, and that is all that costs time.  LR lanes
// cover a row of the state; the other groups of lanes take other rows, and their parts of o are added up at the end.  A wavefront has one
// head of one environment; SPLIT: the four of a workgroup take its rows in turn (heads are few, and a state is read in a quarter of the trips).
// 4096 environments of four heads of 64 x 64: 104 us = 5.2 TB/s.
template <typename T, bool WHOLE, bool SPLIT>
__global__ __launch_bounds__(256) void attention_step_kernel(StepArgs a, int LR) {
  constexpr int W = 4, HEADS = SPLIT ? 1 : 4;
  __shared__ float sq[HEADS][RSLX_ATTN_MAX_DIM], sk[HEADS][RSLX_ATTN_MAX_DIM], so[SPLIT ? 4 : 1][RSLX_ATTN_MAX_DIM];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, own = SPLIT ? 0 : wave;
  const int64_t head = SPLIT ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave, heads = (int64_t)a.N * a.H;
  const bool here = head < heads;
  const int n = here ? (int)(head / a.H) : 0, h = here ? (int)(head % a.H) : 0;
  if (here) {
    const T* q = static_cast<const T*>(a.q.p) + n * a.q.seq + h * a.q.head;
    const T* k = static_cast<const T*>(a.k.p) + n * a.k.seq + h * a.k.head;
    for (int d = SPLIT ? (int)threadIdx.x : lane; d < a.Dk; d += SPLIT ? 256 : 64) {
      sq[own][d] = a.scale * to_float(q[d]);
      sk[own][d] = to_float(k[d]);
    }
  }
  __syncthreads();
  if (!SPLIT && !here) return;
  const T* v = static_cast<const T*>(a.v.p) + n * a.v.seq + h * a.v.head;
  T* o = static_cast<T*>(const_cast<void*>(a.o.p)) + n * a.o.seq + h * a.o.head;
  const float decay = decay_pow(log2_decay(a.log_decay[h]), 1);
  const bool reset = a.reset && a.reset[n] != 0;
  const float* in = a.s_in && !reset ? a.s_in + head * a.Dk * a.Dv : nullptr;
  float* out = a.s_out + head * a.Dk * a.Dv;
  const int groups = (SPLIT ? 256 : 64) / LR, group = (SPLIT ? (int)threadIdx.x : lane) / LR;
  constexpr int AHEAD = 8;
  const int e = (lane % LR) * W;
  float vv[W], acc[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    vv[i] = e + i < a.Dv ? to_float(v[e + i]) : 0.f;
    acc[i] = 0.f;
  }
  for (int d0 = group; d0 < a.Dk; d0 += groups * AHEAD) {
    Pack<float, W> s[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
#pragma unroll
      for (int i = 0; i < W; ++i) s[k].v[i] = 0.f;
      if (in) load_piece<float, W, WHOLE>(s[k], in + (int64_t)min(d0 + k * groups, a.Dk - 1) * a.Dv, e, a.Dv);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int d = d0 + k * groups;
      if (d < a.Dk) {
        const float kk = sk[own][d], qq = sq[own][d];
#pragma unroll
        for (int i = 0; i < W; ++i) {
          s[k].v[i] = fmaf(kk, vv[i], in ? s[k].v[i] * decay : 0.f);
          acc[i] = fmaf(qq, s[k].v[i], acc[i]);
        }
        store_piece<float, W, WHOLE>(s[k], out + (int64_t)d * a.Dv, e, a.Dv);
      }
    }
  }
  for (int x = 32; x >= LR; x >>= 1)
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] += __shfl_xor(acc[i], x, 64);
  if constexpr (SPLIT) {
    if (lane < LR)
#pragma unroll
      for (int i = 0; i < W; ++i) so[wave][e + i] = acc[i];
    __syncthreads();
    for (int x = threadIdx.x; x < a.Dv; x += 256) o[x] = from_float<T>((so[0][x] + so[1][x]) + (so[2][x] + so[3][x]));
  } else if (lane < LR) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (e + i < a.Dv) o[e + i] = from_float<T>(acc[i]);
  }
}

template <typename T>
void run_step(const StepArgs& a, bool whole, bool split, unsigned blocks, int LR, hipStream_t s) {
  const dim3 grid(blocks), threads(256);
  if (whole && split) hipLaunchKernelGGL((attention_step_kernel<T, true, true>), grid, threads, 0, s, a, LR);
  else if (whole) hipLaunchKernelGGL((attention_step_kernel<T, true, false>), grid, threads, 0, s, a, LR);
  else if (split) hipLaunchKernelGGL((attention_step_kernel<T, false, true>), grid, threads, 0, s, a, LR);
  else hipLaunchKernelGGL((attention_step_kernel<T, false, false>), grid, threads, 0, s, a, LR);
}

struct WalkClass { int dkt, dvt; };
WalkClass walk_class(int D, int E, int size) { return {D <= 32 ? 2 : D <= 64 ? 4 : 8, E <= 32 || (D > 64 && size == 2) ? 2 : 4}; }

template <typename T, int DKT, int DVT, int PIECE, bool WHOLE, bool SHARED = false>
void run_walk(const WalkArgs& w, int tiles, int64_t items, hipStream_t s) {
  const int64_t blocks = SHARED ? items : (items * tiles + WALK_WAVES - 1) / WALK_WAVES;
  for (int64_t first = 0; first < blocks; first += WALK_MAX_BLOCKS) {
    const dim3 grid((unsigned)std::min(blocks - first, WALK_MAX_BLOCKS)), threads(64 * WALK_WAVES);
    if (w.states_only)
      hipLaunchKernelGGL((walk_kernel<T, DKT, DVT, PIECE, WHOLE, true, SHARED>), grid, threads, 0, s, w, tiles, (int)first);
    else
      hipLaunchKernelGGL((walk_kernel<T, DKT, DVT, PIECE, WHOLE, false, SHARED>), grid, threads, 0, s, w, tiles, (int)first);
  }
}

template <typename T, int PIECE, bool WHOLE>
void dispatch_walk(const WalkArgs& w, WalkClass k, int tiles, int64_t items, hipStream_t s) {
  switch (k.dkt * 8 + k.dvt) {
    case 2 * 8 + 2: run_walk<T, 2, 2, PIECE, WHOLE>(w, tiles, items, s); break;
    case 2 * 8 + 4: run_walk<T, 2, 4, PIECE, WHOLE>(w, tiles, items, s); break;
    case 4 * 8 + 2: run_walk<T, 4, 2, PIECE, WHOLE>(w, tiles, items, s); break;
    case 4 * 8 + 4: run_walk<T, 4, 4, PIECE, WHOLE>(w, tiles, items, s); break;
    case 8 * 8 + 2:
      if constexpr (sizeof(T) == 2)
        if (tiles > 2) {
          run_walk<T, 8, 2, PIECE, WHOLE, true>(w, tiles, items, s);
          break;
        }
      run_walk<T, 8, 2, PIECE, WHOLE>(w, tiles, items, s);
      break;
    default:
      if constexpr (sizeof(T) == 4) run_walk<T, 8, 4, PIECE, WHOLE>(w, tiles, items, s);      // (16-bit types have no such class)
      break;
  }
}

// The largest access that every row of every matrix allows.  16 / 4 / 2 bytes, rows of the same width further apart: 8192 steps of 16 heads of 128 in bf16
// 88 / 104 / 135 us, gradients 179 / 229 / 343; a roll-out of 24 steps of 4096, four heads of 64, in bf16 148 / 187 / 291, in fp32 206 / 249.  Rows too far
// apart for 32-bit offsets: 24 steps of 1024 in fp32 139 us, 53 where they are not.
int walk_piece(const WalkArgs& w, int size) {
  uintptr_t bits = 0;
  bool near = true;
  auto add = [&](const WalkMatrix& m, int width) {
    if (!m.p) return;
    bits |= reinterpret_cast<uintptr_t>(m.p) | (uintptr_t)m.step * size | (uintptr_t)m.seq * size | (uintptr_t)m.head * size | (uintptr_t)width * size;
    constexpr int64_t MOST = MAX_OFFSET / MOST_CHUNK;
    near = near && m.step < MOST / size && m.step > -(MOST / size);
  };
  for (int j = 0; j < w.jobs; ++j) {
    add(w.job[j].a, w.job[j].D);
    add(w.job[j].b, w.job[j].D);
    add(w.job[j].c, w.job[j].E);
    add(w.job[j].o, w.job[j].E);
  }
  return !near ? 0 : bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

// Whether every width fills its tiles: 32, 64 or 128, the everyday ones.
bool walk_whole(const WalkArgs& w, WalkClass k) {
  for (int j = 0; j < w.jobs; ++j)
    if (w.job[j].D != 16 * k.dkt || w.job[j].E % (16 * k.dvt) != 0) return false;
  return true;
}

template <typename T>
void launch_pieces(const WalkArgs& w, WalkClass k, int piece, int tiles, int64_t items, hipStream_t s) {
  if (piece == 16 && walk_whole(w, k)) dispatch_walk<T, 16, true>(w, k, tiles, items, s);
  else if (piece == 16) dispatch_walk<T, 16, false>(w, k, tiles, items, s);
  else if (piece == 4) dispatch_walk<T, 4, false>(w, k, tiles, items, s);
  else if (piece == 0) run_walk<T, 8, 4, 0, false>(w, tiles, items, s);       // one class for all widths: rows gigabytes apart are no everyday case
  else if constexpr (sizeof(T) == 2) dispatch_walk<T, 2, false>(w, k, tiles, items, s);
}

}  // namespace

int walk_waves_per_head(int D, int E, int size) {
  const WalkClass k = walk_class(D, E, size);
  return (E + 16 * k.dvt - 1) / (16 * k.dvt);
}

// Pieces of a long sequence (of RSLX_ATTN_MAX_STEPS at most: what is rounded up to whole chunks has 32 bits) where the sequences' heads are too few to fill the chip.
int walk_segments(int64_t waves, int32_t T, int32_t* seg_len) {
  constexpr int64_t TARGET = 2048;        // two wavefronts for each of the 1024 SIMDs
  // Shorter pieces are more of them side by side, and more states to move: of at least 32 / 64 / 128 positions, 512 steps of 16 heads of 64 in
  // fp32 27 / 35 / 54 us, 2048 of 8 of 128 in bf16 46 / 38 / 42, 100 of 4 of 32 in fp32 22 / 15 / 15 (in one piece).
  constexpr int LEAST = 64;
  int64_t m = waves > 0 ? TARGET / waves : 1;
  m = m < T / LEAST ? m : T / LEAST;
  m = m < JOIN_MAX ? m : JOIN_MAX;
  if (m <= 1) {
    *seg_len = T < 1 ? MOST_CHUNK : (T - 1) / MOST_CHUNK * MOST_CHUNK + MOST_CHUNK;
    return 1;
  }
  const int64_t len = ((T + m - 1) / m + MOST_CHUNK - 1) / MOST_CHUNK * MOST_CHUNK;      // (m has 64 bits)
  *seg_len = (int32_t)len;
  return (int)((T + len - 1) / len);
}

hipError_t launch_walk(const WalkArgs& all, int dtype, hipStream_t stream) {
  bool done[WALK_MAX_JOBS] = {};
  const int size = dtype == RSLX_F32 ? 4 : 2;
  for (int j = 0; j < all.jobs; ++j) {
    if (done[j]) continue;
    // jobs of the same tile class share a launch: they read the same matrices
    const WalkClass k = walk_class(all.job[j].D, all.job[j].E, size);
    WalkArgs w = all;
    w.jobs = 0;
    int tiles = 0;
    double flops = 0, bytes = 0;
    for (int i = j; i < all.jobs; ++i) {
      const WalkClass q = walk_class(all.job[i].D, all.job[i].E, size);
      if (done[i] || q.dkt != k.dkt || q.dvt != k.dvt) continue;
      done[i] = true;
      w.job[w.jobs++] = all.job[i];
      const WalkJob& x = all.job[i];
      tiles = max(tiles, walk_waves_per_head(x.D, x.E, size));
      const double tokens = (double)all.T * all.N * all.H;
      flops += tokens * x.D * x.E * (all.states_only ? 2 : 4);
      bytes += tokens * size * (all.states_only ? x.D + x.E : 2 * x.D + 2 * x.E);
    }
    const int piece = walk_piece(w, size);
    if (piece == 0)
      for (int i = 0; i < w.jobs; ++i) tiles = max(tiles, (w.job[i].E + 63) / 64);
    const int64_t items = (int64_t)(w.states_only ? w.segments - 1 : w.segments) * w.N * w.H * w.jobs;
    TraceScope trace(stream, w.states_only ? "linear_attention_states" : "linear_attention_walk", flops, bytes);
    if (dtype == RSLX_F32)
      launch_pieces<float>(w, k, piece, tiles, items, stream);
    else if (dtype == RSLX_BF16)
      launch_pieces<bf16_t>(w, k, piece, tiles, items, stream);
    else
      launch_pieces<__half>(w, k, piece, tiles, items, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_walk_join(const WalkArgs& w, const float* const* starts, hipStream_t stream) {
  JoinStarts s{};
  int size = 0;
  for (int j = 0; j < w.jobs; ++j) {
    s.start[j] = starts[j];
    size = max(size, w.job[j].D * w.job[j].E);
  }
  TraceScope trace(stream, "linear_attention_join", 2.0 * size * w.segments * w.N * w.H * w.jobs, 8.0 * size * w.segments * w.N * w.H * w.jobs);
  hipLaunchKernelGGL(walk_join_kernel, dim3((unsigned)(w.N * w.H), (unsigned)((size + 255) / 256), (unsigned)w.jobs), dim3(256), 0, stream, w, s);
  return hipGetLastError();
}

hipError_t launch_attention_step(const StepArgs& a, int dtype, hipStream_t stream) {
  const int64_t heads = (int64_t)a.N * a.H;
  // A wavefront per head fills the chip from some heads for each CU on; before that a head's rows are split.  560 heads of 128 x 126 16.7 us split,
  // 2000 of 128 x 64 27.0 (one wavefront each 30.1); 1800 of 64 x 64 12.6 split, 11.6 not.
  const bool split = heads < (a.Dk > 64 ? 2048 : 1024);
  const int64_t blocks = split ? heads : (heads + 3) / 4;
  int LR = 1;
  while (LR * 4 < a.Dv) LR *= 2;
  const double n = (double)heads * a.Dk * a.Dv;
  TraceScope trace(stream, "linear_attention_step", 5 * n, 8 * n);
  const bool whole = a.Dv % 4 == 0;
  if (dtype == RSLX_F32) run_step<float>(a, whole, split, (unsigned)blocks, LR, stream);
  else if (dtype == RSLX_BF16) run_step<bf16_t>(a, whole, split, (unsigned)blocks, LR, stream);
  else run_step<__half>(a, whole, split, (unsigned)blocks, LR, stream);
  return hipGetLastError();
}

}  // namespace rslx
