// Internal interface between the entry points and the kernels of the operators around a gated memory (gated linear recurrence, root-mean-square
// norm with the residual's addition, Muon step).  Not part of the public ABI (that is include/rslx.h).
#pragma once

#include "../../include/rslx.h"
#include "host.h"
#include "kernels.h"

namespace rslx {

// ---- gated linear recurrence ----------------------------------------------------------------------------------------
struct RecMatrix { void* p; int64_t step, seq; };
struct RecArgs {
  RecMatrix x, g, h;            // forward; one step: step is not used
  RecMatrix dh, dx, dg;         // backward
  int32_t T, N, D;
  const uint8_t* dones;         // one step: the reset flags
  const int32_t* lengths;
  const float* s0;              // or null = 0
  float* s_last;                // or null
  const float* ds_last;         // or null = 0
  float* ds0;                   // or null
  int32_t shared_lines;
  int32_t shape;                // how the steps are shared out (gated_recurrence.hip)
  int32_t pieces;               // of a sequence, of piece_steps steps each
  int64_t piece_steps;
  float *gates, *into, *back;   // more than one piece: the maps s -> gates s + into of every piece, then the states in front of them, and likewise
  int32_t* cuts;                // (back) on the way from the end; whether an episode ends inside; [pieces, N, D rounded up to four], [pieces, N]
};
// Carves the workspace of a call and enters its places.
void plan_recurrence(host::Carver& c, RecArgs& a, int dtype, bool backward);
hipError_t launch_recurrence(RecArgs& a, int dtype, bool backward, hipStream_t stream);
hipError_t launch_recurrence_step(const RecArgs& a, int dtype, hipStream_t stream);

// ---- root-mean-square norm --------------------------------------------------------------------------------------------
constexpr int RMS_MAX_BLOCKS = 1024;      // workgroups of a backward launch: each leaves a row of partial sums

struct RmsArgs {
  const void* x; int64_t ldx;             // forward: x; backward: total
  const void* residual; int64_t ldr;      // forward: or null; backward: dtotal or null
  const void* dy; int64_t lddy;           // backward
  void* total; int64_t ldt;               // forward: or null
  void* y; int64_t ldy;                   // forward: y; backward: dx or null
  int64_t rows;
  int32_t cols;
  const float* weight;                    // or null: 1
  float eps;
  float* scales;                          // forward in 8 bits
  float* rstd;                            // forward: or null
  float* partials;                        // backward: [blocks][cols], or null where dweight is not asked for
  float* dweight;
  int32_t past;                           // outputs go past the caches
};
int rms_backward_blocks(int64_t rows, int cols);
hipError_t launch_rms_norm(const RmsArgs& a, int dtype, bool e4m3, hipStream_t stream);
hipError_t launch_rms_norm_backward(const RmsArgs& a, int dtype, hipStream_t stream);

// ---- Muon step --------------------------------------------------------------------------------------------------------
// p <= q are a matrix's sides, X [p, q] (the transposed update where the matrix is tall), in 32 x 16 blocks of 64 lanes: see muon.hip.
struct alignas(16) MuonItem {
  const float* w_in;
  float* w_out;
  const float* grad;
  const float* m_in;
  float* m_out;
  char* base;                   // the matrix's part of the workspace (muon_item_bytes)
  int32_t rows, cols;
  float scale;
  int16_t in_pieces, large;     // whether its symmetric products are made in pieces of the contraction (plan_muon_parts), whether that with X in large tiles
};
// What every launch reads: the first one, which has it as an argument, leaves it at the start of the workspace for the others (an argument of that size
// is read from memory of the host, several times in a row).
enum MuonGrid { MUON_MOMENTUM_GRID, MUON_PACK_GRID, MUON_SYMMETRIC_GRID, MUON_PIECES_GRID, MUON_FOLD_GRID, MUON_APPLY_GRID, MUON_LARGE_GRID, MUON_GRIDS };
struct MuonTable {
  MuonItem item[RSLX_MUON_MAX_MATRICES];
  int32_t first[MUON_GRIDS][RSLX_MUON_MAX_MATRICES];     // workgroup of a launch that a matrix begins with; INT32_MAX behind the last one
  float lr, momentum, decay;
  int32_t nesterov;
  float* parts;                 // sums over pieces of the contraction, where symmetric products are cut into pieces
  int32_t pieces;
};
constexpr int MUON_NORM_BLOCKS = 512;     // workgroups at most that sum a matrix's squares
size_t muon_item_bytes(int32_t rows, int32_t cols);
size_t plan_muon_parts(MuonTable& t, int count);          // enters the pieces and whose they are; returns the floats of their sums, 0 where there are none
hipError_t launch_muon(MuonTable& t, int count, MuonTable* in_workspace, int steps, hipStream_t stream);

}  // namespace rslx
