// Linear attention with a decay for each head, gfx950: walks over sequences in chunks (forward pass and every gradient), the join of
// a long sequence's pieces, and the single step.
//
//   S_i = l S_{i-1} + b_i c_i^T,   o_i = scale S_i^T a_i,   l = exp(log_decay[h])
//
// A chunk of 16 positions is four small products on the fp32 matrix cores: the scores P = A B^T, weighted by l^(i - j) below the diagonal,
// O = P C + l^(i + 1) A S, and S <- l^16 S + (l^(15 - j) B)^T C.  A wavefront walks one head of one sequence (16 DVT columns of it) by
// itself: the state stays in its accumulator registers, and because the order of a contraction's indices is free, nothing has to be
// moved between lanes.  With lane = 16 g + c, the instruction v_mfma_f32_16x16x4_f32 leaves in register r row 4 g + r of column c, and
// reads from an operand row (column) c at index g.  So
//   - the transposed scores B A^T leave P[c][4 g + r]: the left operand of P C if step s takes the contraction index 4 g + s;
//   - row r of state tile a is put to index d = DKT (4 g + r) + a: then the state's registers are the right operand of A S as they
//     are, if lane (c, g) holds A[c][4 DKT g ...], 4 DKT consecutive values; and the left operand of the state's update, tile a, is
//     B[4 g + s][DKT c + a]: DKT consecutive values of a row;
//   - column tile t is put to e = DVT c + t: C is read, and O written, DVT consecutive values of a row at a time.
// Every operand comes straight from memory in the layout in which it is used: no LDS, no barriers, no shuffles.
#include "sequence.h"
#include "typed.h"

namespace rslx {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int CHUNK = 16;
constexpr int WALK_WAVES = 4;           // wavefronts per workgroup; they share nothing but the caches

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

template <int N> struct alignas(N * 4) Words { uint32_t v[N]; };

// Values e0 .. e0 + N - 1 of a row of `width`; zero past the row's end and where the row does not exist (`row` then points at one that does).
// whole: all of them exist.
template <typename T, int N, bool VEC>
__device__ __forceinline__ void load_frag(Frag<T, N>& f, const T* row, int e0, int width, bool exists, bool whole) {
  constexpr int WORDS = Frag<T, N>::WORDS;
  if constexpr (VEC) {
    constexpr int PW = WORDS < 4 ? WORDS : 4, PE = PW * 4 / (int)sizeof(T);
#pragma unroll
    for (int k = 0; k < WORDS / PW; ++k) {
      const int e = e0 + k * PE;
      Words<PW> x;
      if (whole) {
        x = *reinterpret_cast<const Words<PW>*>(row + e);
      } else {
        const bool in = exists && e < width;
        x = *reinterpret_cast<const Words<PW>*>(row + (in ? e : 0));
#pragma unroll
        for (int i = 0; i < PW; ++i) x.v[i] = in ? x.v[i] : 0u;
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) f.w[k * PW + i] = x.v[i];
    }
  } else {
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {
      if constexpr (sizeof(T) == 4) {
        const bool in = exists && e0 + k < width;
        const uint32_t x = reinterpret_cast<const uint32_t*>(row)[in ? e0 + k : 0];
        f.w[k] = in ? x : 0u;
      } else {
        const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
        const int e = e0 + 2 * k;
        const bool in0 = exists && e < width, in1 = exists && e + 1 < width;
        const uint32_t x0 = r[in0 ? e : 0], x1 = r[in1 ? e + 1 : 0];
        f.w[k] = (in0 ? x0 : 0u) | (in1 ? x1 << 16 : 0u);
      }
    }
  }
}

template <typename T, int N, bool VEC>
__device__ __forceinline__ void store_row(T* row, int e0, int width, const float (&v)[N]) {
  if constexpr (VEC) {
    if (e0 >= width) return;
    Pack<T, N> p;
#pragma unroll
    for (int i = 0; i < N; ++i) p.v[i] = from_float<T>(v[i]);
    *reinterpret_cast<Pack<T, N>*>(row + e0) = p;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e0 + i < width) row[e0 + i] = from_float<T>(v[i]);
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

// Whether an episode ends between position p and the next one.
__device__ __forceinline__ bool cut_behind(const WalkArgs& w, bool reversed, int n, int len, int p) {
  const int t = reversed ? len - 2 - p : p;
  return t >= 0 && p < len && w.dones[(int64_t)t * w.N + n] != 0;
}

template <typename T, int DKT, int DVT, bool VEC, bool STATES>
__global__ __launch_bounds__(64 * WALK_WAVES, DKT * DVT > 16 ? 1 : 2) void walk_kernel(WalkArgs w, int tiles) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  int item = uniform((int)blockIdx.x * WALK_WAVES + (int)(threadIdx.x >> 6));
  const int pieces = STATES ? w.segments - 1 : w.segments;
  const int ji = item % w.jobs; item /= w.jobs;
  const int tile = item % tiles; item /= tiles;
  const int h = item % w.H; item /= w.H;
  const int n = item % w.N, piece = item / w.N;
  if (piece >= pieces) return;
  const WalkJob& job = w.job[ji];
  const int D = job.D, E = job.E, e_tile = tile * 16 * DVT, e_lane = e_tile + DVT * c;
  if (e_tile >= E) return;
  const bool rev = job.reversed != 0;
  const int lead = rev ? 0 : 1;
  const int len = uniform(sequence_length(w, n));
  const int p0 = min(piece * w.seg_len, len), p1 = min(p0 + w.seg_len, len);
  const int64_t first = rev ? len - 1 : 0, dir = rev ? -1 : 1;
  auto base = [&](const WalkMatrix& m) { return static_cast<const T*>(m.p) + n * m.seq + h * m.head + first * m.step; };
  const T* A = STATES ? nullptr : base(job.a);
  const T* B = base(job.b);
  const T* C = base(job.c);
  T* O = STATES ? nullptr : const_cast<T*>(base(job.o));
  const int64_t sa = dir * job.a.step, sb = dir * job.b.step, sc = dir * job.c.step, so = dir * job.o.step;
  const bool whole_d = D == 16 * DKT, whole_e = e_tile + 16 * DVT <= E;

  // weights that every whole chunk shares
  const double l2 = log2_decay(w.log_decay[h]);
  float wp[4], wq[4], wk[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = 4 * g + r;
    wp[r] = c >= i ? w.scale * decay_pow(l2, c - i) : 0.f;
    wq[r] = (rev ? 1.f : w.scale) * decay_pow(l2, i + lead);
    wk[r] = (rev ? w.scale : 1.f) * decay_pow(l2, CHUNK - lead - i);
  }
  // The state is multiplied by the same number once a chunk: its rounding would add up over a long sequence (3e-8 a chunk), so it
  // is kept in two parts.
  const double chunk_decay = exp2(l2 * CHUNK);
  const float f_hi = (float)chunk_decay, f_lo = f_hi < 1e30f ? (float)(chunk_decay - (double)f_hi) : 0.f;

  f32x4 S[DKT][DVT];
#pragma unroll
  for (int a = 0; a < DKT; ++a)
#pragma unroll
    for (int t = 0; t < DVT; ++t) S[a][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  bool live = false;                      // the state may be other than zero
  if (!STATES && job.s_in != nullptr && !(w.segments == 1 && rev && len > 0 && w.dones && w.dones[(int64_t)(len - 1) * w.N + n])) {
    live = true;
    const float* s = job.s_in + (((int64_t)n * w.H + h) * w.segments + piece) * D * E;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d0 = DKT * (4 * g + i);
      if (job.in_col == 1 && E % DVT == 0) {
#pragma unroll
        for (int a = 0; a < DKT; ++a)
          if (d0 + a < D && e_lane < E) {
            const Pack<float, DVT> x = *reinterpret_cast<const Pack<float, DVT>*>(s + (int64_t)(d0 + a) * job.in_row + e_lane);
#pragma unroll
            for (int t = 0; t < DVT; ++t) S[a][t][i] = x.v[t];
          }
      } else if (job.in_row == 1 && D % DKT == 0) {
#pragma unroll
        for (int t = 0; t < DVT; ++t)
          if (d0 < D && e_lane + t < E) {
            const Pack<float, DKT> x = *reinterpret_cast<const Pack<float, DKT>*>(s + (int64_t)(e_lane + t) * job.in_col + d0);
#pragma unroll
            for (int a = 0; a < DKT; ++a) S[a][t][i] = x.v[a];
          }
      } else {
#pragma unroll
        for (int a = 0; a < DKT; ++a)
#pragma unroll
          for (int t = 0; t < DVT; ++t)
            if (d0 + a < D && e_lane + t < E) S[a][t][i] = s[(int64_t)(d0 + a) * job.in_row + (int64_t)(e_lane + t) * job.in_col];
      }
    }
  }

  const bool wants_state = STATES || (job.s_out != nullptr && piece == w.segments - 1);
  bool any_cut = false;
  int careful = p0;                       // positions before this one are taken one at a time
  for (int p = p0; p < p1;) {
    const int m = p < careful ? 1 : min(CHUNK, p1 - p);
    const bool whole_m = m == CHUNK;
    Frag<T, 4 * DKT> fa, fb;
    Frag<T, DKT> fk[4];
    Frag<T, DVT> fv[4];
    const int row_c = min(c, m - 1);
    if constexpr (!STATES) {
      load_frag<T, 4 * DKT, VEC>(fb, B + (p + row_c) * sb, 4 * DKT * g, D, c < m, whole_m && whole_d);
      load_frag<T, 4 * DKT, VEC>(fa, A + (p + row_c) * sa, 4 * DKT * g, D, c < m, whole_m && whole_d);
    }
    const bool update = wants_state || p + m < p1;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int j = 4 * g + s, row = min(j, m - 1);
      load_frag<T, DVT, VEC>(fv[s], C + (p + row) * sc, e_lane, E, j < m, whole_m && whole_e);
      load_frag<T, DKT, VEC>(fk[s], B + (p + row) * sb, DKT * c, D, j < m, whole_m && whole_d);
    }
    // bit i: an episode ends between positions p + i and p + i + 1
    uint32_t cut = 0;
    if (w.dones) cut = (uint32_t)__ballot(lane < m && cut_behind(w, rev, n, len, p + lane)) & 0xffffu;

    // A position's weight for an earlier or later one that it has nothing to do with is zero, but zero times infinity is not: where a
    // chunk's C holds anything that is not finite its positions go one at a time, as the recurrence does.
    if (m > 1) {
      float bad = 0.f;
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int t = 0; t < DVT; ++t) bad = fmaf(fv[s].get(t), 0.f, bad);
      if (__any(bad != 0.f)) {
        careful = p + m;
        continue;
      }
    }

    if constexpr (!STATES) {
      f32x4 P = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4 * DKT; ++x) P = __builtin_amdgcn_mfma_f32_16x16x4f32(fb.get(x), fa.get(x), P, 0, 0, 0);
      f32x4 o[DVT];
#pragma unroll
      for (int t = 0; t < DVT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (live) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int a = 0; a < DKT; ++a)
#pragma unroll
            for (int t = 0; t < DVT; ++t) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa.get(DKT * s + a), S[a][t][s], o[t], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool reached = (cut & ((1u << (4 * g + r)) - 1u)) == 0;
#pragma unroll
          for (int t = 0; t < DVT; ++t) o[t][r] = reached ? o[t][r] * wq[r] : 0.f;
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 4 * g + r;
        const bool same = c >= j && ((cut >> j) & ((1u << ((c - j) & 31)) - 1u)) == 0;
        P[r] = same ? P[r] * wp[r] : 0.f;
      }
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int t = 0; t < DVT; ++t) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(P[s], fv[s].get(t), o[t], 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 4 * g + r;
        float v[DVT];
#pragma unroll
        for (int t = 0; t < DVT; ++t) v[t] = o[t][r];
        if (i < m) store_row<T, DVT, VEC>(O + (p + i) * so, e_lane, E, v);
      }
    }

    if (update) {
      float hi = f_hi, lo = f_lo, wj[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) wj[s] = wk[s];
      if (!whole_m) {
        hi = decay_pow(l2, m);
        lo = 0.f;
#pragma unroll
        for (int s = 0; s < 4; ++s) wj[s] = 4 * g + s < m ? (rev ? w.scale : 1.f) * decay_pow(l2, m - lead - 4 * g - s) : 0.f;
      }
      if (live) {
#pragma unroll
        for (int a = 0; a < DKT; ++a)
#pragma unroll
          for (int t = 0; t < DVT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[a][t][r] = cut ? 0.f : fmaf(S[a][t][r], lo, S[a][t][r] * hi);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bool stays = (cut >> (4 * g + s)) == 0;
#pragma unroll
        for (int a = 0; a < DKT; ++a) {
          const float k = stays ? fk[s].get(a) * wj[s] : 0.f;
#pragma unroll
          for (int t = 0; t < DVT; ++t) S[a][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k, fv[s].get(t), S[a][t], 0, 0, 0);
        }
      }
      live = true;
    }
    if constexpr (STATES) any_cut |= cut != 0;
    p += m;
  }

  if (wants_state) {
    float* s = job.s_out + (((int64_t)n * w.H + h) * (STATES ? w.segments : 1) + (STATES ? piece + 1 : 0)) * D * E;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int a = 0; a < DKT; ++a) {
        const int d = DKT * (4 * g + i) + a;
        float v[DVT];
#pragma unroll
        for (int t = 0; t < DVT; ++t) v[t] = S[a][t][i];
        if (d >= D) continue;
        if (E % DVT == 0)
          store_row<float, DVT, true>(s + (int64_t)d * E, e_lane, E, v);
        else
          store_row<float, DVT, false>(s + (int64_t)d * E, e_lane, E, v);
      }
  }
  if constexpr (STATES) {
    if (w.cuts && h == 0 && tile == 0 && lane == 0) w.cuts[((int64_t)ji * w.N + n) * w.segments + piece] = any_cut ? 1 : 0;
  } else {
    // steps that do not exist: zero
    T* Z = static_cast<T*>(const_cast<void*>(job.o.p)) + n * job.o.seq + h * job.o.head;
    const float zero[DVT] = {};
    const int t1 = piece == w.segments - 1 ? w.T : min((piece + 1) * w.seg_len, w.T);
    for (int t = max(len, piece * w.seg_len) + g; t < t1; t += 4) store_row<T, DVT, VEC>(Z + (int64_t)t * job.o.step, e_lane, E, zero);
  }
}

// One thread per element of a head's state: slot 0 takes the start, then every slot what it adds to the decayed one before it.
constexpr int JOIN_MAX = 512;
struct JoinStarts { const float* start[WALK_MAX_JOBS]; };
__global__ __launch_bounds__(256) void walk_join_kernel(WalkArgs w, JoinStarts starts) {
  __shared__ float f[JOIN_MAX];
  __shared__ int cut[JOIN_MAX];
  const int ji = blockIdx.z, n = blockIdx.x / w.H, h = blockIdx.x % w.H;
  const WalkJob& job = w.job[ji];
  const int len = sequence_length(w, n);
  const double l2 = log2_decay(w.log_decay[h]);
  for (int m = threadIdx.x; m < w.segments - 1; m += 256) {
    f[m] = decay_pow(l2, min(max(len - m * w.seg_len, 0), w.seg_len));
    cut[m] = w.cuts[((int64_t)ji * w.N + n) * w.segments + m];
  }
  __syncthreads();
  const int e = blockIdx.y * 256 + threadIdx.x, size = job.D * job.E;
  if (e >= size) return;
  const int64_t head = (int64_t)n * w.H + h;
  float* slot = job.s_out + head * w.segments * size + e;
  float run = starts.start[ji] ? starts.start[ji][head * size + e] : 0.f;
  if (job.reversed && len > 0 && w.dones && w.dones[(int64_t)(len - 1) * w.N + n]) run = 0.f;
  slot[0] = run;
  constexpr int AHEAD = 8;
  for (int m0 = 0; m0 < w.segments - 1; m0 += AHEAD) {
    float x[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) x[k] = slot[(int64_t)(min(m0 + k, w.segments - 2) + 1) * size];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (m0 + k >= w.segments - 1) break;
      run = cut[m0 + k] ? x[k] : fmaf(run, f[m0 + k], x[k]);
      slot[(int64_t)(m0 + k + 1) * size] = run;
    }
  }
}

// ---- one step -----------------------------------------------------------------------------------------------------
// S <- l S + k v^T, o = scale S^T q: the state is read and written once, W columns a lane, and that is all that costs time.  A
// wavefront has one head of one row: LR lanes cover a row of the state (or a block of 64 W columns), the other groups take other
// rows, and their parts of o are added up at the end.
template <typename T, int W>
__global__ __launch_bounds__(256) void attention_step_kernel(StepArgs a, int LR) {
  __shared__ float sq[4][128], sk[4][128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t head = (int64_t)blockIdx.x * 4 + wave, heads = (int64_t)a.N * a.H;
  const bool here = head < heads;
  const int n = here ? (int)(head / a.H) : 0, h = here ? (int)(head % a.H) : 0;
  if (here) {
    const T* q = static_cast<const T*>(a.q.p) + n * a.q.seq + h * a.q.head;
    const T* k = static_cast<const T*>(a.k.p) + n * a.k.seq + h * a.k.head;
    for (int d = lane; d < a.Dk; d += 64) {
      sq[wave][d] = a.scale * to_float(q[d]);
      sk[wave][d] = to_float(k[d]);
    }
  }
  __syncthreads();
  if (!here) return;
  const T* v = static_cast<const T*>(a.v.p) + n * a.v.seq + h * a.v.head;
  T* o = static_cast<T*>(const_cast<void*>(a.o.p)) + n * a.o.seq + h * a.o.head;
  const float decay = decay_pow(log2_decay(a.log_decay[h]), 1);
  const bool reset = a.reset && a.reset[n] != 0;
  const float* in = a.s_in ? a.s_in + head * a.Dk * a.Dv : nullptr;
  float* out = a.s_out + head * a.Dk * a.Dv;
  const int groups = 64 / LR, group = lane / LR;
  constexpr int AHEAD = 8;
  for (int e0 = 0; e0 < a.Dv; e0 += LR * W) {
    const int e = e0 + (lane % LR) * W;
    const bool mine = e < a.Dv;
    float vv[W], acc[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      vv[i] = mine ? to_float(v[e + i]) : 0.f;
      acc[i] = 0.f;
    }
    if (mine) {
      for (int d0 = group; d0 < a.Dk; d0 += groups * AHEAD) {
        Pack<float, W> s[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int d = min(d0 + k * groups, a.Dk - 1);
          if (in && !reset) s[k] = *reinterpret_cast<const Pack<float, W>*>(in + (int64_t)d * a.Dv + e);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int d = d0 + k * groups;
          if (d < a.Dk) {
            const float kk = sk[wave][d], qq = sq[wave][d];
#pragma unroll
            for (int i = 0; i < W; ++i) {
              const float old = in && !reset ? s[k].v[i] * decay : 0.f;
              s[k].v[i] = fmaf(kk, vv[i], old);
              acc[i] = fmaf(qq, s[k].v[i], acc[i]);
            }
            *reinterpret_cast<Pack<float, W>*>(out + (int64_t)d * a.Dv + e) = s[k];
          }
        }
      }
    }
    for (int x = 32; x >= LR; x >>= 1)
#pragma unroll
      for (int i = 0; i < W; ++i) acc[i] += __shfl_xor(acc[i], x, 64);
    if (mine && group == 0)
#pragma unroll
      for (int i = 0; i < W; ++i) o[e + i] = from_float<T>(acc[i]);
  }
}

struct WalkClass { int dkt, dvt; };
WalkClass walk_class(int D, int E) { return {D <= 32 ? 2 : D <= 64 ? 4 : 8, E <= 32 ? 2 : 4}; }

template <typename T, int DKT, int DVT>
void run_walk(const WalkArgs& w, bool vec, int tiles, unsigned blocks, hipStream_t s) {
  const dim3 grid(blocks), threads(64 * WALK_WAVES);
  if (w.states_only) {
    if (vec)
      hipLaunchKernelGGL((walk_kernel<T, DKT, DVT, true, true>), grid, threads, 0, s, w, tiles);
    else
      hipLaunchKernelGGL((walk_kernel<T, DKT, DVT, false, true>), grid, threads, 0, s, w, tiles);
  } else {
    if (vec)
      hipLaunchKernelGGL((walk_kernel<T, DKT, DVT, true, false>), grid, threads, 0, s, w, tiles);
    else
      hipLaunchKernelGGL((walk_kernel<T, DKT, DVT, false, false>), grid, threads, 0, s, w, tiles);
  }
}

template <typename T>
void dispatch_walk(const WalkArgs& w, WalkClass k, bool vec, int tiles, unsigned blocks, hipStream_t s) {
  switch (k.dkt * 8 + k.dvt) {
    case 2 * 8 + 2: run_walk<T, 2, 2>(w, vec, tiles, blocks, s); break;
    case 2 * 8 + 4: run_walk<T, 2, 4>(w, vec, tiles, blocks, s); break;
    case 4 * 8 + 2: run_walk<T, 4, 2>(w, vec, tiles, blocks, s); break;
    case 4 * 8 + 4: run_walk<T, 4, 4>(w, vec, tiles, blocks, s); break;
    case 8 * 8 + 2: run_walk<T, 8, 2>(w, vec, tiles, blocks, s); break;
    default: run_walk<T, 8, 4>(w, vec, tiles, blocks, s); break;
  }
}

// Loads of up to 16 bytes: every row of every matrix starts at a multiple of them and is a whole number of them.
bool walk_wide(const WalkArgs& w, int size) {
  const int per = 16 / size;
  auto fits = [&](const WalkMatrix& m, int width) {
    return !m.p || ((reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && width % per == 0 && m.step % per == 0 && m.seq % per == 0 && m.head % per == 0);
  };
  for (int j = 0; j < w.jobs; ++j) {
    const WalkJob& k = w.job[j];
    if (!(fits(k.a, k.D) && fits(k.b, k.D) && fits(k.c, k.E) && fits(k.o, k.E))) return false;
  }
  return true;
}

}  // namespace

int walk_waves_per_head(int D, int E) {
  const WalkClass k = walk_class(D, E);
  return (E + 16 * k.dvt - 1) / (16 * k.dvt);
}

// Pieces of a long sequence where the sequences' heads are too few to fill the chip.
int walk_segments(int64_t waves, int32_t T, int32_t* seg_len) {
  constexpr int64_t TARGET = 2048;        // two wavefronts for each of the 1024 SIMDs
  constexpr int LEAST = 64;
  int64_t m = waves > 0 ? TARGET / waves : 1;
  m = m < T / LEAST ? m : T / LEAST;
  m = m < JOIN_MAX ? m : JOIN_MAX;
  if (m <= 1) {
    *seg_len = T < 1 ? CHUNK : (T + CHUNK - 1) / CHUNK * CHUNK;
    return 1;
  }
  const int64_t len = ((T + m - 1) / m + CHUNK - 1) / CHUNK * CHUNK;
  *seg_len = (int32_t)len;
  return (int)((T + len - 1) / len);
}

hipError_t launch_walk(const WalkArgs& all, int dtype, hipStream_t stream) {
  bool done[WALK_MAX_JOBS] = {};
  const int size = dtype == RSLX_F32 ? 4 : 2;
  for (int j = 0; j < all.jobs; ++j) {
    if (done[j]) continue;
    // jobs of the same tile class share a launch: they read the same matrices
    const WalkClass k = walk_class(all.job[j].D, all.job[j].E);
    WalkArgs w = all;
    w.jobs = 0;
    int tiles = 0;
    double flops = 0, bytes = 0;
    for (int i = j; i < all.jobs; ++i) {
      const WalkClass q = walk_class(all.job[i].D, all.job[i].E);
      if (done[i] || q.dkt != k.dkt || q.dvt != k.dvt) continue;
      done[i] = true;
      w.job[w.jobs++] = all.job[i];
      const WalkJob& x = all.job[i];
      tiles = max(tiles, walk_waves_per_head(x.D, x.E));
      const double tokens = (double)all.T * all.N * all.H;
      flops += tokens * x.D * x.E * (all.states_only ? 2 : 4);
      bytes += tokens * size * (all.states_only ? x.D + x.E : 2 * x.D + 2 * x.E);
    }
    const int64_t waves = (int64_t)(w.states_only ? w.segments - 1 : w.segments) * w.N * w.H * tiles * w.jobs;
    const int64_t blocks = (waves + WALK_WAVES - 1) / WALK_WAVES;
    if (blocks > (1 << 23)) return hipErrorInvalidConfiguration;
    const bool vec = walk_wide(w, size);
    TraceScope trace(stream, w.states_only ? "linear_attention_states" : "linear_attention_walk", flops, bytes);
    if (dtype == RSLX_F32)
      dispatch_walk<float>(w, k, vec, tiles, (unsigned)blocks, stream);
    else if (dtype == RSLX_BF16)
      dispatch_walk<bf16_t>(w, k, vec, tiles, (unsigned)blocks, stream);
    else
      dispatch_walk<__half>(w, k, vec, tiles, (unsigned)blocks, stream);
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
  const int64_t heads = (int64_t)a.N * a.H, blocks = (heads + 3) / 4;
  if (blocks > (1 << 23)) return hipErrorInvalidConfiguration;
  const bool vec = a.Dv % 4 == 0;
  const int lanes = vec ? a.Dv / 4 : a.Dv;
  int LR = 1;
  while (LR < lanes && LR < 64) LR *= 2;
  const double n = (double)heads * a.Dk * a.Dv;
  TraceScope trace(stream, "linear_attention_step", 5 * n, 8 * n);
  const dim3 grid((unsigned)blocks), threads(256);
  if (dtype == RSLX_F32) {
    if (vec) hipLaunchKernelGGL((attention_step_kernel<float, 4>), grid, threads, 0, stream, a, LR);
    else hipLaunchKernelGGL((attention_step_kernel<float, 1>), grid, threads, 0, stream, a, LR);
  } else if (dtype == RSLX_BF16) {
    if (vec) hipLaunchKernelGGL((attention_step_kernel<bf16_t, 4>), grid, threads, 0, stream, a, LR);
    else hipLaunchKernelGGL((attention_step_kernel<bf16_t, 1>), grid, threads, 0, stream, a, LR);
  } else {
    if (vec) hipLaunchKernelGGL((attention_step_kernel<__half, 4>), grid, threads, 0, stream, a, LR);
    else hipLaunchKernelGGL((attention_step_kernel<__half, 1>), grid, threads, 0, stream, a, LR);
  }
  return hipGetLastError();
}

}  // namespace rslx
