// Gated linear recurrence, gfx950.
//
//   f = sigmoid(g),  h_t = f_t keep_{t-1} h_{t-1} + (1 - f_t) x_t
//   q_t = f_t (dh_t + keep_t q_{t+1}),  d_t = dh_t + keep_t q_{t+1},  dx = (1 - f) d,  dg = f (1 - f) d (keep_{t-1} h_{t-1} - x)
//
// Both directions are scans of maps s -> A s + B, whose compositions are such maps again; an episode's end is the map that forgets s, held as a flag of its
// own, so that no 0 times infinity arises.  A lane takes LANE_STEPS steps of four channels into registers and composes their maps; 16 lanes side by side
// read 64 channels, 128 to 256 bytes of a row; the wavefront's four sets of lanes and the workgroup's wavefronts compose theirs through shuffles and
// LDS; then every lane walks its steps again from the state that enters them.  Every value is read once and every result written once, as long as a
// workgroup's steps hold the sequence, or channels are many enough for workgroups to go along whole sequences (forward).  Otherwise sequences
// are cut into pieces: one launch leaves every piece's map, a second the states between the pieces, a third makes the results.
//
// Bound by memory where values are read once: a roll-out of 24 steps of 4096 environments of 256 in fp32 61 us = 5.1 TB/s, the gradients of a quarter of
// it 27 us = 4.9 TB/s.  In pieces inputs are read twice, the second time from the last-level cache where they fit: 8192 steps of 4 environments of 1024 in
// bf16 72 us (maps 31 us, 4.4 TB/s; join 5; results 35), gradients of 4096 steps 56 us.  Gates cost 16-bit walks as much as memory does, so that what stands
// beside them counts: addresses are common to a wavefront where offsets fit 32 bits, steps are not asked one by one where all exist and none ends an episode
// (40 -> 17 vector instructions a value; 90 -> 76 us and 92 -> 63 for these two).
#include "memory.h"
#include "overlap.h"
#include "typed.h"

namespace rslx {

namespace {

constexpr int REC_THREADS = 256;
constexpr int W = 4;                      // channels of a lane
constexpr int ROW = 16;                   // lanes side by side
constexpr int TILE = W * ROW;             // channels of a workgroup
constexpr int SETS = 64 / ROW;            // sets of lanes of a wavefront, one after another in time

// f = sigmoid(g) = 1 / (1 + E) and 1 - f = E f, of E = exp(-g): each keeps its own digits.  Below -87, where f leaves fp32's normal numbers, g counts as -87.
// For fp32 the exponential is that of the product g log2(e) in two parts, the rounded one for the instruction and what rounding left as a factor.  Gates of 16
// bits do without the second: E is off by up to |g| 2^-24 more then, where the type's own half step is |g| 2^-9 or 2^-12 (8192 steps of
// 4 environments, 1024 channels, in bf16: 71 us, with the factor 76).
template <typename T>
__device__ __forceinline__ void gate(float g, float& f, float& rest) {
  constexpr float LOG2E = 1.44269504f, LOG2E_REST = 1.92596299e-8f, LN2 = 0.693147181f;
  const float low = g < -87.f ? -87.f : g;
  float e;
  if constexpr (sizeof(T) == 4) {
    const float m = low > 128.f ? 128.f : low, p = -m * LOG2E, left = fmaf(-m, LOG2E, -p) - m * LOG2E_REST;      // (exp(-128) is zero in fp32)
    e = __builtin_amdgcn_exp2f(p);
    e = fmaf(e, left * LN2, e);
  } else {
    e = __builtin_amdgcn_exp2f(low * -LOG2E);
  }
  f = __builtin_amdgcn_rcpf(1.f + e);
  rest = e * f;
}

template <typename T> __device__ __forceinline__ T* row_of(const RecMatrix& m, int64_t t, int64_t n) {
  return static_cast<T*>(m.p) + t * m.step + n * m.seq;
}

struct Four { float v[W]; };
__device__ __forceinline__ Four all(float x) { return {{x, x, x, x}}; }

// s -> A s + B, or s -> B where an episode ends inside.
struct Map {
  Four a, b;
  int cut;
  __device__ __forceinline__ Four operator()(const Four& s) const {
    Four r;
#pragma unroll
    for (int k = 0; k < W; ++k) r.v[k] = cut ? b.v[k] : fmaf(a.v[k], s.v[k], b.v[k]);
    return r;
  }
  // this one behind `first`
  __device__ __forceinline__ void after(const Map& first) {
    b = (*this)(first.b);
#pragma unroll
    for (int k = 0; k < W; ++k) a.v[k] *= first.a.v[k];
    cut |= first.cut;
  }
};
__device__ __forceinline__ Map same() { return {all(1.f), all(0.f), 0}; }

// The map of another lane.
template <bool UP>
__device__ __forceinline__ Map from_lane(const Map& m, int distance) {
  Map r;
#pragma unroll
  for (int k = 0; k < W; ++k) {
    r.a.v[k] = UP ? __shfl_up(m.a.v[k], distance, 64) : __shfl_down(m.a.v[k], distance, 64);
    r.b.v[k] = UP ? __shfl_up(m.b.v[k], distance, 64) : __shfl_down(m.b.v[k], distance, 64);
  }
  r.cut = UP ? __shfl_up(m.cut, distance, 64) : __shfl_down(m.cut, distance, 64);
  return r;
}

// Maps of a workgroup's wavefronts.
template <int WAVES>
struct WaveMaps {
  float4 a[WAVES][ROW], b[WAVES][ROW];
  int cut[WAVES];
  __device__ __forceinline__ void put(int wave, int lane, const Map& m) {
    a[wave][lane] = *reinterpret_cast<const float4*>(&m.a);
    b[wave][lane] = *reinterpret_cast<const float4*>(&m.b);
    if (lane == 0) cut[wave] = m.cut;
  }
  __device__ __forceinline__ Map get(int wave, int lane) const {
    Map m;
    *reinterpret_cast<float4*>(&m.a) = a[wave][lane];
    *reinterpret_cast<float4*>(&m.b) = b[wave][lane];
    m.cut = cut[wave];
    return m;
  }
};

// Every set of lanes has the map of its steps; `s` is the state in front of the first (FORWARD) or behind the last one of the workgroup's steps.  Returns the
// state in front of (behind) the lane's own, and leaves the one at the other end in s.  `maps` is free again after the next such call with other maps.
template <int WAVES, bool FORWARD>
__device__ __forceinline__ Four enter(Map m, Four& s, WaveMaps<WAVES>& maps) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & (ROW - 1);
#pragma unroll
  for (int o = ROW; o < 64; o *= 2) {
    const Map other = from_lane<FORWARD>(m, o);
    if (FORWARD ? lane >= o : lane + o < 64) m.after(other);
  }
  const Map before = from_lane<FORWARD>(m, ROW);
  const bool first = FORWARD ? lane < ROW : lane >= 64 - ROW, last = FORWARD ? lane >= 64 - ROW : lane < ROW;
  Four mine = s;
  if constexpr (WAVES > 1) {
    if (last) maps.put(wave, col, m);
    __syncthreads();
#pragma unroll 2
    for (int i = 0; i < WAVES; ++i) {
      const int w = FORWARD ? i : WAVES - 1 - i;
      if (w == wave) mine = s;
      s = maps.get(w, col)(s);
    }
  } else {
    const Four end = m(s);
#pragma unroll
    for (int k = 0; k < W; ++k) s.v[k] = __shfl(end.v[k], (FORWARD ? 64 - ROW : 0) + col, 64);
  }
  return first ? mine : before(mine);
}

// The map of all of the workgroup's steps, from those of its sets of lanes.
template <int WAVES, bool FORWARD>
__device__ __forceinline__ Map whole(Map m, WaveMaps<WAVES>& maps) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & (ROW - 1);
#pragma unroll
  for (int o = ROW; o < 64; o *= 2) {
    const Map other = from_lane<FORWARD>(m, o);
    if (FORWARD ? lane >= o : lane + o < 64) m.after(other);
  }
  if (FORWARD ? lane >= 64 - ROW : lane < ROW) maps.put(wave, col, m);
  __syncthreads();
  m = maps.get(FORWARD ? 0 : WAVES - 1, col);
#pragma unroll 1
  for (int i = 1; i < WAVES; ++i) {
    Map next = maps.get(FORWARD ? i : WAVES - 1 - i, col);
    next.after(m);
    m = next;
  }
  return m;
}

// A workgroup's place: a tile of channels of a sequence, a piece of the steps.
struct Place {
  int64_t n;
  int d, len, piece;
  bool full;                                // every lane has four channels: the same for the whole workgroup
  int from, shift;                          // the last four channels that a lane may read from, and how far behind them its own are (D >= W)
};
// `last_first`: in the other order on each die, for a launch that reads what the one before it read: what that read last lies in the caches still (gradients of
// 2048 steps of 32 sequences, 1024 channels in bf16: 227 us, in the same order 250; 777 steps of 37 of 200 in fp32 46 and 48).  Forward pieces run all at once, and
// nothing is gained.
__device__ __forceinline__ Place place_of(const RecArgs& a, bool last_first = false) {
  const int tiles = (a.D + TILE - 1) / TILE;
  // workgroups go to the eight dies in turn.  Where neighbours share lines of memory, each die gets a row of them, so that its L2 joins what they read and
  // write (500 steps of 300 sequences, 203 channels in bf16: 77 us, in turn 86); where they do not, in turn is better (8192 steps of 4, 1024 channels: 73 and 81)
  const uint32_t each = gridDim.x / 8, more = gridDim.x % 8, die = blockIdx.x % 8;
  uint32_t turn = blockIdx.x / 8;
  if (last_first) turn = each + (die < more ? 1 : 0) - 1 - turn;
  const uint32_t block = a.shared_lines ? die * each + (die < more ? die : more) + turn : turn * 8 + die;
  const int64_t all_tiles = (int64_t)a.N * tiles, at = block % all_tiles;
  Place p;
  p.piece = (int)(block / all_tiles);
  p.n = at / tiles;
  p.d = (int)(at % tiles) * TILE + (threadIdx.x & (ROW - 1)) * W;
  p.full = (int)(at % tiles) * TILE + TILE <= a.D;
  p.from = p.d <= a.D - W ? p.d : a.D - W;
  p.shift = (p.d - p.from) & (W - 1);
  p.len = a.T;
  if (a.lengths) {
    const int len = a.lengths[p.n];
    p.len = len < 0 ? 0 : len > a.T ? a.T : len;
  }
  return p;
}

template <bool WHOLE>
__device__ __forceinline__ Four load_state(const float* s, const RecArgs& a, const Place& p) {
  Pack<float, W> v;
#pragma unroll
  for (int k = 0; k < W; ++k) v.v[k] = 0.f;
  if (s) load_piece<float, W, WHOLE>(v, s + p.n * a.D, p.d, a.D);
  return *reinterpret_cast<const Four*>(&v);
}
template <bool WHOLE>
__device__ __forceinline__ void store_state(float* s, const RecArgs& a, const Place& p, const Four& f) {
  if (s) store_piece<float, W, WHOLE>(*reinterpret_cast<const Pack<float, W>*>(&f), s + p.n * a.D, p.d, a.D);
}
// A piece's entry of a workspace array [pieces, N, D rounded up to four].
__device__ __forceinline__ float4* piece_at(float* base, const RecArgs& a, const Place& p) {
  return reinterpret_cast<float4*>(base + ((int64_t)p.piece * a.N + p.n) * ((a.D + W - 1) / W * W) + p.d);
}

// A matrix as a lane sees it: its row of step i behind the wavefront's first.  WHOLE: rows are whole, aligned loads, and what differs between lanes fits 32 bits:
// the address is a common one and an offset that stays, for any i; lanes beyond the last channel read the first one's.
// STREAM: how large matrices go past the caches, which keep other things then: 1, what is written; 2, what is read as well (see stream_of).
template <typename T, bool WHOLE, int STREAM>
struct Rows {
  typedef uint32_t Bits __attribute__((ext_vector_type(sizeof(T) * W / 4)));
  static constexpr bool EDGE = !WHOLE && sizeof(T) == 2;
  char* base;
  uint32_t offset;
  T* mine;
  int64_t step;
  __device__ __forceinline__ Rows(const RecMatrix& m, const RecArgs& a, const Place& p, int64_t t, int ahead) : step(m.step) {
    if constexpr (WHOLE) {
      base = reinterpret_cast<char*>(static_cast<T*>(m.p) + t * m.step + p.n * m.seq);
      offset = ((uint32_t)ahead * (uint32_t)m.step + (uint32_t)(p.d < a.D ? p.d : 0)) * (uint32_t)sizeof(T);
    } else {
      mine = static_cast<T*>(m.p) + (t + ahead) * m.step + p.n * m.seq;
    }
  }
  __device__ __forceinline__ void load(Pack<T, W>& v, int i, const RecArgs& a, const Place& p) const {
    if constexpr (WHOLE && STREAM == 2) {
      const Bits bits = __builtin_nontemporal_load(reinterpret_cast<const Bits*>(base + i * step * (int64_t)sizeof(T) + offset));
      __builtin_memcpy(&v, &bits, sizeof v);
    } else if constexpr (WHOLE) v = *reinterpret_cast<const Pack<T, W>*>(base + i * step * (int64_t)sizeof(T) + offset);
    else load_piece<T, W, false>(v, mine + i * step, p.d, a.D);
  }
  // EDGE: 16-bit values of rows that start anywhere.  Those of a row's last channels, which four need not be, come in one load as well, and rows are loaded without
  // asking which steps exist: what is loaded in parts, or under a condition, is put together in a register, and waited for there and then (500 steps of 300 sequences,
  // 203 channels in bf16: 78 us, in parts 130; their gradients 158 and 244).  Values of 32 bits have registers of their own: in fp32 106 in parts, 135 in this way.
  __device__ __forceinline__ void load_edge(Pack<T, W>& v, int i, const Place& p) const {
    uint64_t bits;
    __builtin_memcpy(&bits, mine + i * step + p.from, sizeof bits);
    bits >>= p.shift * 16;
    __builtin_memcpy(&v, &bits, sizeof bits);
  }
  // all of the lane's steps; EDGE: the step `last` in place of those behind it
  template <int L>
  __device__ __forceinline__ void load(Pack<T, W> (&v)[L], const RecArgs& a, const Place& p, int64_t last = L) const {
    if (!WHOLE && p.full) {
#pragma unroll
      for (int i = 0; i < L; ++i) __builtin_memcpy(&v[i], mine + (!EDGE || i < last ? i : last) * step + p.d, sizeof v[i]);
    } else if (!EDGE || a.D < W) {
#pragma unroll
      for (int i = 0; i < L; ++i) load(v[i], !EDGE || i < last ? i : (int)last, a, p);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) load_edge(v[i], i < last ? i : (int)last, p);
    }
  }
  template <int L>
  __device__ __forceinline__ void store(const Pack<T, W> (&v)[L], const RecArgs& a, const Place& p) const {
    if (WHOLE || !p.full) {
#pragma unroll
      for (int i = 0; i < L; ++i) store(v[i], i, a, p);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) __builtin_memcpy(mine + i * step + p.d, &v[i], sizeof v[i]);
    }
  }
  __device__ __forceinline__ void store(const Pack<T, W>& v, int i, const RecArgs& a, const Place& p) const {
    if constexpr (WHOLE) {
      if (p.d >= a.D) return;
      Bits bits;
      __builtin_memcpy(&bits, &v, sizeof v);
      Bits* to = reinterpret_cast<Bits*>(base + i * step * (int64_t)sizeof(T) + offset);
      if constexpr (STREAM > 0) __builtin_nontemporal_store(bits, to);
      else *to = bits;
    } else {
      store_piece<T, W, false>(v, mine + i * step, p.d, a.D);
    }
  }
};

// Zeros behind the last step that exists.
template <int L, typename T, bool WHOLE, int STREAM>
__device__ __forceinline__ void store_nothing(const Rows<T, WHOLE, STREAM>& r, int64_t t0, const RecArgs& a, const Place& p) {
  Pack<T, W> zero;
#pragma unroll
  for (int k = 0; k < W; ++k) zero.v[k] = from_float<T>(0.f);
#pragma unroll
  for (int i = 0; i < L; ++i)
    if (t0 + i < a.T) r.store(zero, i, a, p);
}

// Which of the lane's steps from t0 on end an episode.
template <int L>
__device__ __forceinline__ uint32_t ends_of(const RecArgs& a, const Place& p, int64_t t0) {
  uint32_t ends = 0;
  if (a.dones)
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (t0 + i < p.len && a.dones[(t0 + i) * a.N + p.n]) ends |= 1u << i;
  return ends;
}

// Forward: a workgroup goes along its piece, WAVES * SETS * L steps at a time.  MAPS: no results, the piece's map alone.  Where every step of a wavefront exists and
// none ends an episode (`plain`), nothing is asked step by step.
template <typename T, int L, int WAVES, bool WHOLE, int STREAM, bool MAPS>
__global__ __launch_bounds__(WAVES * 64) void recurrence_kernel(RecArgs a) {
  constexpr bool EDGE = Rows<T, WHOLE, STREAM>::EDGE;
  __shared__ WaveMaps<WAVES> maps[2];
  const Place p = place_of(a);
  const int ahead = threadIdx.x / ROW * L;
  const int64_t begin = (int64_t)p.piece * a.piece_steps, end = begin + a.piece_steps < a.T ? begin + a.piece_steps : a.T;
  Four s = all(0.f);
  Map piece = same();
  if (!MAPS) {
    if (a.pieces > 1 && p.d < a.D) *reinterpret_cast<float4*>(&s) = *piece_at(a.into, a, p);
    else if (a.pieces == 1) s = load_state<WHOLE>(a.s0, a, p);
  }
  int turn = 0;
  for (int64_t t = begin; t < end; t += WAVES * SETS * L, turn ^= 1) {
    const int64_t t0 = t + ahead;
    const Rows<T, WHOLE, STREAM> rx(a.x, a, p, t, ahead), rg(a.g, a, p, t, ahead);
    Pack<T, W> px[L], pg[L];
    const uint32_t ends = ends_of<L>(a, p, t0);
    const bool plain = __all(ends == 0 && t0 + L <= p.len), none = __all(t0 >= p.len);
    float f[L][W], v[L][W];
    Map m = same();
    auto gates = [&]() {
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          float rest;
          gate<T>(to_float(pg[i].v[k]), f[i][k], rest);
          v[i][k] = rest * to_float(px[i].v[k]);
        }
    };
    if (none) {
      // (the map that hands the state on)
    } else if (plain) {
      rg.load(pg, a, p);
      rx.load(px, a, p);
      gates();
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          m.b.v[k] = i == 0 ? v[0][k] : fmaf(f[i][k], m.b.v[k], v[i][k]);
          m.a.v[k] = i == 0 ? f[0][k] : m.a.v[k] * f[i][k];
        }
    } else {
      if (EDGE) {
        rg.load(pg, a, p, p.len - 1 - t0);
        rx.load(px, a, p, p.len - 1 - t0);
      } else {
#pragma unroll
        for (int i = 0; i < L; ++i)
          if (t0 + i < p.len) {
            rg.load(pg[i], i, a, p);
            rx.load(px[i], i, a, p);
          }
      }
      gates();
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          // steps that do not exist hand the state on
          if (t0 + i >= p.len) f[i][k] = 1.f, v[i][k] = 0.f;
          m.b.v[k] = ends >> i & 1 ? 0.f : fmaf(f[i][k], m.b.v[k], v[i][k]);
          m.a.v[k] *= f[i][k];
        }
      m.cut = ends != 0;
    }
    if constexpr (MAPS) {
      Map next = whole<WAVES, true>(m, maps[turn]);
      next.after(piece);
      piece = next;
      continue;
    }
    Four h = enter<WAVES, true>(m, s, maps[turn]);
    const Rows<T, WHOLE, STREAM> rh(a.h, a, p, t, ahead);
    if (plain) {
      Pack<T, W> out[L];
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          h.v[k] = fmaf(f[i][k], h.v[k], v[i][k]);
          out[i].v[k] = from_float<T>(h.v[k]);
        }
      rh.store(out, a, p);
    } else if (none) {
      store_nothing<L>(rh, t0, a, p);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        Pack<T, W> out;
#pragma unroll
        for (int k = 0; k < W; ++k) {
          h.v[k] = fmaf(f[i][k], h.v[k], v[i][k]);
          out.v[k] = from_float<T>(t0 + i < p.len ? h.v[k] : 0.f);
          if (ends >> i & 1) h.v[k] = 0.f;
        }
        if (t0 + i < a.T) rh.store(out, i, a, p);
      }
    }
  }
  if (threadIdx.x >= ROW || p.d >= a.D) return;
  if constexpr (MAPS) {
    *piece_at(a.gates, a, p) = *reinterpret_cast<const float4*>(&piece.a);
    *piece_at(a.into, a, p) = *reinterpret_cast<const float4*>(&piece.b);
    if (p.d == 0) a.cuts[(int64_t)p.piece * a.N + p.n] = piece.cut;
  } else if (p.piece == a.pieces - 1) {
    store_state<WHOLE>(a.s_last, a, p, s);
  }
}

// Backward: a piece is the steps that a workgroup holds at once.  MAPS: the piece's maps of both directions (whose gates' product is the same).
template <typename T, int L, int WAVES, bool WHOLE, int STREAM, bool MAPS>
__global__ __launch_bounds__(WAVES * 64) void recurrence_backward_kernel(RecArgs a) {
  constexpr bool EDGE = Rows<T, WHOLE, STREAM>::EDGE;
  __shared__ WaveMaps<WAVES> maps[2];
  const Place p = place_of(a, !MAPS && a.pieces > 1);
  const int ahead = threadIdx.x / ROW * L;
  const int64_t t = (int64_t)p.piece * (WAVES * SETS * L), t0 = t + ahead;
  const Rows<T, WHOLE, STREAM> rx(a.x, a, p, t, ahead), rg(a.g, a, p, t, ahead), rd(a.dh, a, p, t, ahead);
  Pack<T, W> px[L], pg[L], pd[L];
  const uint32_t ends = ends_of<L>(a, p, t0);
  const bool plain = __all(ends == 0 && t0 + L <= p.len), none = __all(t0 >= p.len);
  float f[L][W], rest[L][W];
  Map m = same(), up = same();
  auto gates = [&]() {
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) gate<T>(to_float(pg[i].v[k]), f[i][k], rest[i][k]);
  };
  if (none) {
    // (the maps that hand the states on)
  } else if (plain) {
    rg.load(pg, a, p);
    rx.load(px, a, p);
    rd.load(pd, a, p);
    gates();
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float v = rest[i][k] * to_float(px[i].v[k]);
        m.b.v[k] = i == 0 ? v : fmaf(f[i][k], m.b.v[k], v);
        m.a.v[k] = i == 0 ? f[0][k] : m.a.v[k] * f[i][k];
      }
#pragma unroll
    for (int i = L - 1; i >= 0; --i)
#pragma unroll
      for (int k = 0; k < W; ++k) up.b.v[k] = f[i][k] * (i == L - 1 ? to_float(pd[i].v[k]) : up.b.v[k] + to_float(pd[i].v[k]));
  } else {
    if (EDGE) {
      rg.load(pg, a, p, p.len - 1 - t0);
      rx.load(px, a, p, p.len - 1 - t0);
      rd.load(pd, a, p, p.len - 1 - t0);
    }
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (t0 + i < p.len) {
        if (!EDGE) {
          rg.load(pg[i], i, a, p);
          rx.load(px[i], i, a, p);
          rd.load(pd[i], i, a, p);
        }
      } else {
        // steps that do not exist hand both states on
#pragma unroll
        for (int k = 0; k < W; ++k) px[i].v[k] = pd[i].v[k] = pg[i].v[k] = from_float<T>(0.f);
      }
    gates();
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) {
        if (t0 + i >= p.len) f[i][k] = 1.f, rest[i][k] = 0.f;
        m.b.v[k] = ends >> i & 1 ? 0.f : fmaf(f[i][k], m.b.v[k], rest[i][k] * to_float(px[i].v[k]));
        m.a.v[k] *= f[i][k];
      }
#pragma unroll
    for (int i = L - 1; i >= 0; --i)
#pragma unroll
      for (int k = 0; k < W; ++k) up.b.v[k] = f[i][k] * ((ends >> i & 1 ? 0.f : up.b.v[k]) + to_float(pd[i].v[k]));
    m.cut = up.cut = ends != 0;
  }
  up.a = m.a;
  if constexpr (MAPS) {
    m = whole<WAVES, true>(m, maps[0]);
    up = whole<WAVES, false>(up, maps[1]);
    if (threadIdx.x >= ROW || p.d >= a.D) return;
    *piece_at(a.gates, a, p) = *reinterpret_cast<const float4*>(&m.a);
    *piece_at(a.into, a, p) = *reinterpret_cast<const float4*>(&m.b);
    *piece_at(a.back, a, p) = *reinterpret_cast<const float4*>(&up.b);
    if (p.d == 0) a.cuts[(int64_t)p.piece * a.N + p.n] = m.cut;
    return;
  }
  Four s = all(0.f), q = all(0.f);
  if (a.pieces > 1) {
    if (p.d < a.D) {
      *reinterpret_cast<float4*>(&s) = *piece_at(a.into, a, p);
      *reinterpret_cast<float4*>(&q) = *piece_at(a.back, a, p);
    }
  } else {
    s = load_state<WHOLE>(a.s0, a, p);
    q = load_state<WHOLE>(a.ds_last, a, p);
  }
  Four h = enter<WAVES, true>(m, s, maps[0]), down = enter<WAVES, false>(up, q, maps[1]);
  if (p.piece == 0 && threadIdx.x < ROW) store_state<WHOLE>(a.ds0, a, p, q);
  const Rows<T, WHOLE, STREAM> rdx(a.dx, a, p, t, ahead), rdg(a.dg, a, p, t, ahead);
  if (none) {
    store_nothing<L>(rdx, t0, a, p);
    store_nothing<L>(rdg, t0, a, p);
    return;
  }
  float in[L][W];                           // f (1 - f) (h - x), of the states h that the steps start from
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float x = to_float(px[i].v[k]);
      in[i][k] = f[i][k] * (h.v[k] - x);
      h.v[k] = fmaf(f[i][k], h.v[k], rest[i][k] * x);
      if (!plain && (ends >> i & 1)) h.v[k] = 0.f;
    }
#pragma unroll
  for (int i = L - 1; i >= 0; --i) {
    Pack<T, W> dx, dg;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if (!plain && (ends >> i & 1)) down.v[k] = 0.f;
      const float d = down.v[k] + to_float(pd[i].v[k]), by = rest[i][k] * d;
      const bool here = plain || t0 + i < p.len;
      dx.v[k] = from_float<T>(here ? by : 0.f);
      dg.v[k] = from_float<T>(here ? by * in[i][k] : 0.f);
      down.v[k] = f[i][k] * d;
    }
    if (plain || t0 + i < a.T) {
      rdx.store(dx, i, a, p);
      rdg.store(dg, i, a, p);
    }
  }
}

// The states between the pieces, in place of the pieces' maps: the one in front of each (into), and behind each on the way back (back, blockIdx.y = 1).  A lane has a
// channel, each of the sixteen wavefronts a sixteenth of the pieces, whose map it makes before it walks them (8192 steps of 2 sequences of 64 channels, 128
// pieces: 4 us; one after another 13).
constexpr int JOIN_WAVES = 16, JOIN_AHEAD = 8;
__global__ __launch_bounds__(JOIN_WAVES * 64) void recurrence_join_kernel(RecArgs a) {
  __shared__ float map_a[JOIN_WAVES][64], map_b[JOIN_WAVES][64];
  __shared__ int map_cut[JOIN_WAVES][64];
  const int width = (a.D + W - 1) / W * W, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t channels = (int64_t)a.N * width, c = (int64_t)blockIdx.x * 64 + lane;
  const bool here = c < channels;
  const int64_t n = here ? c / width : 0;
  const int d = here ? (int)(c % width) : 0, each = (a.pieces + JOIN_WAVES - 1) / JOIN_WAVES;
  const int64_t begin = (int64_t)wave * each, end = here ? (begin + each < a.pieces ? begin + each : a.pieces) : 0;
  const bool back = blockIdx.y != 0;
  float* at = back ? a.back : a.into;
  float scale[JOIN_AHEAD], add[JOIN_AHEAD];
  int cut[JOIN_AHEAD];
  auto ask = [&](int64_t first) {
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i)
      if (first + i < end) {
        const int64_t piece = back ? a.pieces - 1 - first - i : first + i;
        scale[i] = a.gates[piece * channels + c];
        add[i] = at[piece * channels + c];
        cut[i] = a.cuts[piece * a.N + n];
      }
  };
  float all_a = 1.f, all_b = 0.f;
  int any = 0;
  for (int64_t first = begin; first < end; first += JOIN_AHEAD) {
    ask(first);
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i)
      if (first + i < end) {
        all_b = cut[i] ? add[i] : fmaf(scale[i], all_b, add[i]);
        all_a *= scale[i];
        any |= cut[i];
      }
  }
  map_a[wave][lane] = all_a;
  map_b[wave][lane] = all_b;
  map_cut[wave][lane] = any;
  __syncthreads();
  const float* start = back ? a.ds_last : a.s0;
  float s = start && here && d < a.D ? start[n * a.D + d] : 0.f;
  for (int w = 0; w < wave; ++w) s = map_cut[w][lane] ? map_b[w][lane] : fmaf(map_a[w][lane], s, map_b[w][lane]);
  for (int64_t first = begin; first < end; first += JOIN_AHEAD) {
    if (each > JOIN_AHEAD) ask(first);                   // (fewer are in the registers still)
#pragma unroll
    for (int i = 0; i < JOIN_AHEAD; ++i)
      if (first + i < end) {
        at[(back ? a.pieces - 1 - first - i : first + i) * channels + c] = s;
        s = cut[i] ? add[i] : fmaf(scale[i], s, add[i]);
      }
  }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(REC_THREADS) void recurrence_step_kernel(RecArgs a) {
  const int per = (a.D + W - 1) / W;
  const int64_t c = (int64_t)blockIdx.x * REC_THREADS + threadIdx.x;
  if (c >= (int64_t)a.N * per) return;
  Place p;
  p.n = c / per;
  p.d = (int)(c % per) * W;
  Pack<T, W> px, pg, out;
  load_piece<T, W, WHOLE>(pg, row_of<T>(a.g, 0, p.n), p.d, a.D);
  load_piece<T, W, WHOLE>(px, row_of<T>(a.x, 0, p.n), p.d, a.D);
  Four s = load_state<WHOLE>(a.dones && a.dones[p.n] ? nullptr : a.s0, a, p);
#pragma unroll
  for (int k = 0; k < W; ++k) {
    float f, rest;
    gate<T>(to_float(pg.v[k]), f, rest);
    s.v[k] = fmaf(f, s.v[k], rest * to_float(px.v[k]));
    out.v[k] = from_float<T>(s.v[k]);
  }
  store_state<WHOLE>(a.s_last, a, p, s);
  store_piece<T, W, WHOLE>(out, row_of<T>(a.h, 0, p.n), p.d, a.D);
}

// How the steps are shared out: wavefronts of a workgroup, steps of a lane; see plan_recurrence.
enum RecShape { FORWARD_1 = 0, FORWARD_4, BACKWARD_1, BACKWARD_4, BACKWARD_4_SHORT, BACKWARD_2_SHORT };
constexpr int LANE_STEPS[] = {4, 4, 8, 8, 4, 4}, SHAPE_WAVES[] = {1, 4, 1, 4, 4, 2};
int steps_of(int shape) { return LANE_STEPS[shape] * SHAPE_WAVES[shape] * SETS; }

template <typename T, bool WHOLE, int STREAM, bool MAPS>
void run_shape(const RecArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)a.N * ((a.D + TILE - 1) / TILE) * a.pieces);
#define RUN(shape, kernel) \
  case shape: hipLaunchKernelGGL((kernel<T, LANE_STEPS[shape], SHAPE_WAVES[shape], WHOLE, STREAM, MAPS>), dim3(grid), dim3(SHAPE_WAVES[shape] * 64), 0, s, a); break
  switch (a.shape) {
    RUN(FORWARD_4, recurrence_kernel);
    RUN(BACKWARD_4, recurrence_backward_kernel);
    RUN(BACKWARD_4_SHORT, recurrence_backward_kernel);
    RUN(BACKWARD_2_SHORT, recurrence_backward_kernel);
    default:
      if constexpr (!MAPS) switch (a.shape) {
        RUN(FORWARD_1, recurrence_kernel);
        RUN(BACKWARD_1, recurrence_backward_kernel);
      }
  }
#undef RUN
}

// Whether every row of every matrix is a number of whole, aligned loads, and the rows of the `held` steps that a workgroup has at once lie within 2^31 bytes,
// upwards.  The distance of steps has no part in it where there is one: so for each shape of its own, and of the steps that there are (24 steps of 8192
// environments of 256 channels in fp32: forward 123 us, as rows that start anywhere 150; gradients 205 and 242; of 16384 in bf16 162 and 180, 258 and 291).
bool rec_whole(const RecArgs& a, int size, int held) {
  if (held > a.T) held = a.T;
  auto fits = [&](const RecMatrix& m) {
    return !m.p || (reinterpret_cast<uintptr_t>(m.p) % (W * size) == 0 && m.seq % W == 0 &&
                    (held <= 1 || (m.step % W == 0 && m.step >= 0 && m.step < ((int64_t)1 << 31) / held / size - a.D)));
  };
  return a.D % W == 0 && fits(a.x) && fits(a.g) && fits(a.h) && fits(a.dh) && fits(a.dx) && fits(a.dg);
}

// Outputs of 16 MB and more, which the dies' L2 could not keep beside the inputs, are written past the caches; inputs are read past them where the call moves more than
// the last-level cache's 256 MB and reads them once.  24 steps of fp32 roll-outs of 256 channels, us through the caches, outputs past them, inputs as well: forward
// 341 environments (8 MB of outputs) 12.5, 11.9, 12.2; 683 (17 MB) 14.0, 14.0, 15.3; 2048 37.6, 29.4, 33.8; 3000 (221 MB moved) 53.3, 46.6, 48.1; 3600 (265 MB) 65, 63.6,
// 61.9; 4096 74.8, 71.9, 62.1; gradients of 1024 31.2, 28.3, 31.6; of 4096 130, 127, 107.  In bf16 forward 4096 50.5, 38.4, 44.8; 8192 95.8, 94.2, 84.0.
int stream_of(const RecArgs& a, int size) {
  const double matrix = (double)a.T * a.N * a.D * size;
  const int outputs = a.h.p ? 1 : 2, inputs = a.h.p ? 2 : 3;
  if (outputs * matrix < (double)(16 << 20)) return 0;
  return a.pieces == 1 && (outputs + inputs) * matrix > 256e6 ? 2 : 1;
}

// Whether tiles of a row meet inside a line of memory.
bool shared_lines(const RecArgs& a, int size) {
  auto apart = [&](const RecMatrix& m) { return !m.p || (reinterpret_cast<uintptr_t>(m.p) | (uint64_t)m.step * size | (uint64_t)m.seq * size) % 128 == 0; };
  return (int64_t)a.D * size % 128 != 0 || !(apart(a.x) && apart(a.g) && apart(a.h) && apart(a.dh) && apart(a.dx) && apart(a.dg));
}

template <typename T>
void run_type(const RecArgs& a, bool maps, hipStream_t s) {
  const bool whole = rec_whole(a, (int)sizeof(T), steps_of(a.shape));
  const int stream = stream_of(a, (int)sizeof(T));
  if (maps) whole ? run_shape<T, true, 0, true>(a, s) : run_shape<T, false, 0, true>(a, s);
  else if (!whole) run_shape<T, false, 0, false>(a, s);
  else if (stream == 0) run_shape<T, true, 0, false>(a, s);
  else if (stream == 1) run_shape<T, true, 1, false>(a, s);
  else run_shape<T, true, 2, false>(a, s);
}

void run(const RecArgs& a, int dtype, bool maps, hipStream_t s) {
  if (dtype == RSLX_F32) run_type<float>(a, maps, s);
  else if (dtype == RSLX_BF16) run_type<bf16_t>(a, maps, s);
  else run_type<__half>(a, maps, s);
}

}  // namespace

// Forward, a wavefront along each sequence and 64 channels where these fill the GPU with eight wavefronts for each compute unit, or where 16 steps are all;
// otherwise four, 64 steps at a time, in about 1024 pieces where these are few (100 steps of 300 sequences of 256 channels in bf16: 14.1 us, with one
// 16.7; 777 steps of 37 of 200 in fp32: 32, in 512 pieces 37, in 2048 31; 8192 steps of 4 of 1024 in bf16: 72, in 512 pieces 81).
// Backward, the smallest workgroup that holds the sequence: 32, 64 or 128 steps.  Longer ones are cut into pieces: of 32 up to 2048 steps (777 steps of 37 of 203 in
// fp16, ragged: 37.5 us, pieces of 64 41.5, in fp32 57 and 59.5; 200 steps of 500 of 203 in bf16 112 and 123, in fp32 203 and 223; 2000 steps of 16 of 512 in bf16 53.6
// and 54.3, in fp32 95.9 and 97.5; 1024 steps of 300 of 256 in bf16 270 and 270, in fp32 504 and 497), where the join has few; beyond, of 128 where these
// are many and rows aligned (4096 steps of 4 of 1024 in bf16: 58 us, pieces of 64 61), of 64 otherwise (8192 steps of 4 of 256 in fp32: 53 us, pieces of 128
// 55, of 32 58).
void plan_recurrence(host::Carver& c, RecArgs& a, int dtype, bool backward) {
  const int64_t tiles = (int64_t)a.N * (((int64_t)a.D + TILE - 1) / TILE);
  a.pieces = 1;
  a.piece_steps = a.T;
  if (backward) {
    const auto pieces = [&](int shape) { return tiles * (((int64_t)a.T + steps_of(shape) - 1) / steps_of(shape)); };
    if (a.T <= steps_of(BACKWARD_1)) a.shape = BACKWARD_1;
    else if (a.T <= steps_of(BACKWARD_4_SHORT)) a.shape = BACKWARD_4_SHORT;
    else if (a.T <= steps_of(BACKWARD_4)) a.shape = BACKWARD_4;
    else if (a.T <= 2048 && pieces(BACKWARD_2_SHORT) < (int64_t)1 << 24) a.shape = BACKWARD_2_SHORT;      // (as many as a launch has)
    else if (a.T > 2048 && a.x.p && rec_whole(a, host::type_size(dtype), steps_of(BACKWARD_4)) && pieces(BACKWARD_4) >= 1536) a.shape = BACKWARD_4;
    else a.shape = BACKWARD_4_SHORT;
    a.piece_steps = steps_of(a.shape);
  } else {
    a.shape = a.T <= steps_of(FORWARD_1) || tiles >= 2048 ? FORWARD_1 : FORWARD_4;
    if (a.shape == FORWARD_4 && tiles > 0) {
      const int64_t blocks = ((int64_t)a.T + steps_of(FORWARD_4) - 1) / steps_of(FORWARD_4), want = (1023 + tiles) / tiles;
      const int64_t each = tiles >= 256 || want < 2 ? blocks : (blocks + want - 1) / want;
      a.piece_steps = each * steps_of(FORWARD_4);
    }
  }
  if (a.piece_steps > 0 && a.piece_steps < a.T) a.pieces = (int32_t)((a.T + a.piece_steps - 1) / a.piece_steps);
  if (a.pieces > 1) {
    const size_t states = (size_t)a.pieces * a.N * ((a.D + W - 1) / W * W);
    a.gates = c.take<float>(states);
    a.into = c.take<float>(states);
    if (backward) a.back = c.take<float>(states);
    a.cuts = c.take<int32_t>((size_t)a.pieces * a.N);
  }
}

hipError_t launch_recurrence(RecArgs& a, int dtype, bool backward, hipStream_t stream) {
  a.shared_lines = shared_lines(a, host::type_size(dtype));
  const double n = (double)a.T * a.N * a.D, size = dtype == RSLX_F32 ? 4 : 2;
  if (a.pieces > 1) {
    {
      TraceScope trace(stream, backward ? "recurrence_backward_maps" : "recurrence_maps", (backward ? 20 : 16) * n, (backward ? 3 : 2) * n * size);
      run(a, dtype, true, stream);
    }
    const double states = (double)a.pieces * a.N * a.D;
    TraceScope trace(stream, "recurrence_join", 2 * states, (backward ? 16 : 12) * states);
    const int64_t channels = (int64_t)a.N * ((a.D + W - 1) / W * W);
    hipLaunchKernelGGL(recurrence_join_kernel, dim3((unsigned)((channels + 63) / 64), backward ? 2 : 1), dim3(JOIN_WAVES * 64), 0, stream, a);
  }
  TraceScope trace(stream, backward ? "recurrence_backward" : "recurrence", (backward ? 25 : 10) * n, (backward ? 5 : 3) * n * size);
  run(a, dtype, false, stream);
  return hipGetLastError();
}

hipError_t launch_recurrence_step(const RecArgs& a, int dtype, hipStream_t stream) {
  const double n = (double)a.N * a.D, size = dtype == RSLX_F32 ? 4 : 2;
  TraceScope trace(stream, "recurrence_step", 10 * n, (3 * size + 8) * n);
  const dim3 grid((unsigned)(((int64_t)a.N * ((a.D + W - 1) / W) + REC_THREADS - 1) / REC_THREADS)), block(REC_THREADS);
  const bool whole = rec_whole(a, (int)size, 1);
#define RUN(T)                                                                                          \
  do {                                                                                                  \
    if (whole) hipLaunchKernelGGL((recurrence_step_kernel<T, true>), grid, block, 0, stream, a);        \
    else hipLaunchKernelGGL((recurrence_step_kernel<T, false>), grid, block, 0, stream, a);             \
  } while (0)
  if (dtype == RSLX_F32) RUN(float);
  else if (dtype == RSLX_BF16) RUN(bf16_t);
  else RUN(__half);
#undef RUN
  return hipGetLastError();
}

}  // namespace rslx
