// Internal interface between the entry points and the kernels of the sequence operators (linear attention with a decay for
// each head, layer norm).  Not part of the public ABI (that is include/rslx.h).
#pragma once

#include "../../include/rslx.h"
#include "kernels.h"

namespace rslx {

// ---- layer norm ---------------------------------------------------------------------------------------------------
constexpr int NORM_MAX_BLOCKS = 1024;     // workgroups of a backward launch: each leaves a row of partial sums

struct NormArgs {
  const void* x; int64_t ldx;
  void* y; int64_t ldy;                   // forward
  const void* dy; int64_t lddy;           // backward
  void* dx; int64_t lddx;                 // or null
  int64_t rows;
  int32_t cols;
  const float* weight;                    // or null: 1
  const float* bias;                      // or null: 0
  float eps;
  float* mean;                            // forward: or null
  float* rstd;
  float* partials;                        // backward: [2][blocks][cols], or null where neither gradient is asked for
  float* dweight;                         // or null
  float* dbias;
};

int norm_backward_blocks(int64_t rows, int cols);
hipError_t launch_layer_norm(const NormArgs& a, int dtype, bool backward, hipStream_t stream);

// ---- linear attention ---------------------------------------------------------------------------------------------
// One walk over the positions of every sequence (per head):
//   o_i = sum over j <= i of w(i - j) (a_i . b_j) c_j + what the state before the first position adds
// The forward pass is one (a, b, c = q, k, v), each gradient another: dq walks (do, v, k), dv (k, q, do) and dk (v, do, q), the last two from
// the sequence's end.  The state is the sum of the outer products of b and c, [D, E].
struct WalkMatrix { const void* p; int64_t step, seq, head; };
struct WalkJob {
  WalkMatrix a, b, c, o;
  int32_t D, E;                 // widths of a, b and of c, o
  int32_t reversed;             // positions count from the sequence's end, and the state carries the scale
  const float* s_in;            // state before the first position (of every segment: see segments), or null = 0
  int64_t in_row, in_col;       // its element (d, e) at d * in_row + e * in_col
  float* s_out;                 // state behind the last position, [N, H, D, E], or null
};
constexpr int WALK_MAX_JOBS = 3;
struct WalkArgs {
  WalkJob job[WALK_MAX_JOBS];
  int32_t jobs;
  int32_t T, N, H;
  float scale;
  const float* log_decay;
  const uint8_t* dones;
  const int32_t* lengths;
  int32_t segments, seg_len;    // a sequence is cut into this many pieces of seg_len positions (a multiple of 16); one piece: s_in is
                                // the caller's [N, H, D, E], more: [N, H, segments, D, E], from the two launches below
  int32_t states_only;          // no outputs: piece m leaves its own contribution in slot m + 1 of s_out [N, H, segments, D, E], and
  int32_t* cuts;                // [job][N][segments]: whether an episode ends behind one of its positions
};
int walk_segments(int64_t waves, int32_t T, int32_t* seg_len);
int walk_waves_per_head(int D, int E, int size);      // size: bytes of a value
hipError_t launch_walk(const WalkArgs& w, int dtype, hipStream_t stream);
// slot[0] = start (0 where the sequence's last step ends an episode and the walk is reversed), slot[m + 1] = decay^len_m slot[m] + slot[m + 1]
hipError_t launch_walk_join(const WalkArgs& w, const float* const* starts, hipStream_t stream);

struct StepArgs {
  WalkMatrix q, k, v, o;        // step is not used
  int32_t N, H, Dk, Dv;
  float scale;
  const float* log_decay;
  const uint8_t* reset;
  const float* s_in;
  float* s_out;
};
hipError_t launch_attention_step(const StepArgs& a, int dtype, hipStream_t stream);

}  // namespace rslx
