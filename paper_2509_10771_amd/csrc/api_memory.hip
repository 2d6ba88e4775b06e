// C ABI of the operators around a gated memory: gated linear recurrence, root-mean-square norm with the residual's addition, Muon step.  Argument checks,
// workspace planning and the order of the launches; the kernels are in gated_recurrence.hip, rms_norm.hip and muon.hip.
#include "memory.h"
#include "overlap.h"

using namespace rslx;
using namespace rslx::host;

namespace {

RowSet block_of(const void* p, int64_t bytes) { return {p, bytes, {}, {p && bytes > 0 ? 1 : 0, 1, 1}}; }
RowSet floats_of(const void* p, int64_t n) { return p ? host::rows_of(p, 1, n, 1, 4) : block_of(nullptr, 0); }

// ---- gated linear recurrence ----------------------------------------------------------------------------------------
int32_t check_rec(const rslx_gated_rec* a, const char* who, bool step) {
  if (!a) return fail(RSLX_ERR_INVALID_ARG, "%s: null description", who);
  RSLX_TRY(check_dtype(a->dtype, who));
  if (a->T < 0 || a->T > RSLX_ATTN_MAX_STEPS || a->N < 0 || a->D < 1) return fail(RSLX_ERR_SHAPE, "%s: T = %d, N = %d, D = %d", who, a->T, a->N, a->D);
  const int64_t tiles = (a->N > 0 ? (int64_t)a->N : 1) * (((int64_t)a->D + 63) / 64);
  if (tiles > RSLX_REC_MAX_TILES) return fail(RSLX_ERR_SHAPE, "%s: N * ceil(D / 64) = %lld exceeds %d", who, (long long)tiles, RSLX_REC_MAX_TILES);
  if (step && (a->T != 1 || a->dones || a->lengths))
    return fail(RSLX_ERR_INVALID_ARG, "%s: one step has T = 1 and neither dones nor lengths", who);
  return RSLX_OK;
}

RowSet rows_of(const rslx_gated_rec& a, const rslx_seq_view& v) {
  const int size = type_size(a.dtype);
  return {v.data, (int64_t)a.D * size, {(wide)v.step * size, (wide)v.seq * size, 0}, {a.T, a.N, 1}};
}

int32_t check_view(const rslx_gated_rec& a, const rslx_seq_view* v, bool written, const char* who, const char* name) {
  if (!v || !v->data) return fail(RSLX_ERR_INVALID_ARG, "%s: null %s", who, name);
  if (reinterpret_cast<uintptr_t>(v->data) % type_size(a.dtype) != 0) return fail(RSLX_ERR_INVALID_ARG, "%s: %s not aligned to its type", who, name);
  if (written && overlaps_itself(rows_of(a, *v)))
    return fail(RSLX_ERR_SHAPE, "%s: rows of %s overlap (strides %lld and %lld, width %d)", who, name, (long long)v->step, (long long)v->seq, a.D);
  return RSLX_OK;
}

Named named(const rslx_gated_rec& a, const rslx_seq_view* v, const char* name) { return a.T > 0 ? Named{rows_of(a, *v), name} : Named{{}, name}; }
Named named(const rslx_gated_rec& a, const float* state, const char* name) { return {block_of(state, (int64_t)a.N * a.D * 4), name}; }

int32_t check_state(const float* s, const char* who, const char* name) {
  if (s && !aligned16(s)) return fail(RSLX_ERR_INVALID_ARG, "%s: %s not 16-byte aligned", who, name);
  return RSLX_OK;
}

RecMatrix matrix(const rslx_seq_view* v) { return v ? RecMatrix{v->data, v->step, v->seq} : RecMatrix{}; }

RecArgs rec_args(const rslx_gated_rec& a) {
  RecArgs r;
  memset(&r, 0, sizeof r);
  r.T = a.T; r.N = a.N; r.D = a.D;
  r.dones = a.dones;
  r.lengths = a.lengths;
  return r;
}

// A launch has fewer than 2^32 lanes.
int32_t check_grid(const RecArgs& r, const char* who) {
  if ((int64_t)r.N * ((r.D + 63) / 64) * r.pieces >= (int64_t)1 << 24 || (r.pieces > 1 && (int64_t)r.N * ((r.D + 3) / 4) >= (int64_t)1 << 26))
    return fail(RSLX_ERR_SHAPE, "%s: %d pieces of %d sequences of %d channels are too many", who, r.pieces, r.N, r.D);
  return RSLX_OK;
}

size_t rec_workspace(const rslx_gated_rec* a, bool backward, const char* who) {
  if (check_rec(a, who, false) != RSLX_OK) return 0;
  Carver c(nullptr);
  RecArgs r = rec_args(*a);
  plan_recurrence(c, r, a->dtype, backward);
  if (check_grid(r, who) != RSLX_OK) return 0;
  return c.off > 256 ? c.off : 256;
}

int32_t rec_plan(RecArgs& r, int dtype, bool backward, void* ws, size_t ws_bytes, const char* who) {
  Carver c(ws);
  plan_recurrence(c, r, dtype, backward);
  RSLX_TRY(check_grid(r, who));
  if (c.off > 0 && (!ws || ws_bytes < c.off)) return fail(RSLX_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, ws_bytes, c.off);
  if (c.off > 0 && !aligned16(ws)) return fail(RSLX_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", who);
  return RSLX_OK;
}

// ---- root-mean-square norm --------------------------------------------------------------------------------------------
int32_t check_rows(int32_t dtype, int64_t rows, int32_t cols, const char* who) {
  RSLX_TRY(check_dtype(dtype, who));
  if (rows < 0 || cols < 1 || cols > RSLX_NORM_MAX_COLS)
    return fail(RSLX_ERR_SHAPE, "%s: %lld rows of %d, 1 to %d columns are taken", who, (long long)rows, cols, RSLX_NORM_MAX_COLS);
  return RSLX_OK;
}

struct NormMatrix {
  const void* p;
  int64_t ld;
  int size;
  const char* name;
  RowSet rows(int64_t n, int32_t cols) const { return p ? host::rows_of(p, ld, n, cols, size) : RowSet{nullptr, 0, {}, {0, 0, 0}}; }
};

int32_t check_aligned(const NormMatrix& m, const char* who) {
  if (reinterpret_cast<uintptr_t>(m.p) % m.size) return fail(RSLX_ERR_INVALID_ARG, "%s: %s not aligned to its type", who, m.name);
  return RSLX_OK;
}

int32_t check_written(const NormMatrix& m, int64_t rows, int32_t cols, const char* who) {
  if (m.p && rows > 1 && m.ld < cols && m.ld > -(int64_t)cols)
    return fail(RSLX_ERR_SHAPE, "%s: rows of %s overlap (distance %lld, %d columns)", who, m.name, (long long)m.ld, cols);
  return RSLX_OK;
}

// An output may be one of the inputs, row by row in place; it must not overlap it otherwise (rows are loaded before earlier ones are stored).
int32_t check_in_place(const NormMatrix& out, const NormMatrix& in, int64_t rows, int32_t cols, const char* who) {
  if (!out.p || !in.p || (out.p == in.p && (rows == 1 || out.ld == in.ld))) return RSLX_OK;
  if (share_memory(out.rows(rows, cols), in.rows(rows, cols)))
    return fail(RSLX_ERR_INVALID_ARG, "%s: %s and %s overlap and are not the same matrix", who, out.name, in.name);
  return RSLX_OK;
}

int32_t rms_norm(int32_t dtype, bool e4m3, const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int32_t cols, const float* weight,
                 float eps, void* total, int64_t ldt, void* y, int64_t ldy, float* scales, float* rstd, void* stream, const char* who) {
  RSLX_TRY(check_rows(dtype, rows, cols, who));
  if (rows == 0) return RSLX_OK;
  if (!x || !y || (e4m3 && !scales)) return fail(RSLX_ERR_INVALID_ARG, "%s: null x, y or scales", who);
  const int size = type_size(dtype);
  const NormMatrix in[] = {{x, ldx, size, "x"}, {residual, ldr, size, "residual"}}, out[] = {{y, ldy, e4m3 ? 1 : size, "y"}, {total, ldt, size, "total"}};
  for (int i = 0; i < 2; ++i) {
    RSLX_TRY(check_aligned(in[i], who));
    RSLX_TRY(check_aligned(out[i], who));
    RSLX_TRY(check_written(out[i], rows, cols, who));
  }
  if (!aligned16(weight)) return fail(RSLX_ERR_INVALID_ARG, "%s: weight not 16-byte aligned", who);
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      if (i == 1 || !e4m3) RSLX_TRY(check_in_place(out[i], in[j], rows, cols, who));
  const Named all[] = {{out[0].rows(rows, cols), "y"}, {out[1].rows(rows, cols), "total"}, {floats_of(scales, rows), "scales"},
                       {floats_of(rstd, rows), "rstd"}, {floats_of(weight, cols), "weight"}};
  RSLX_TRY(check_apart(all, 4, who));
  const Named statistics[] = {all[2], all[3], {in[0].rows(rows, cols), "x"}, {in[1].rows(rows, cols), "residual"}};
  RSLX_TRY(check_apart(statistics, 2, who));
  const Named bytes[] = {all[0], statistics[2], statistics[3]};
  if (e4m3) RSLX_TRY(check_apart(bytes, 1, who));
  RmsArgs a;
  memset(&a, 0, sizeof a);
  a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.total = total; a.ldt = ldt; a.y = y; a.ldy = ldy;
  a.rows = rows; a.cols = cols;
  a.weight = weight; a.eps = eps;
  a.scales = scales; a.rstd = rstd;
  RSLX_HIP(launch_rms_norm(a, dtype, e4m3, (hipStream_t)stream));
  return RSLX_OK;
}

// ---- Muon step --------------------------------------------------------------------------------------------------------
int32_t check_muon(const rslx_muon_matrix* m, int32_t count, const rslx_muon_cfg* cfg, const char* who) {
  if (!cfg || (count > 0 && !m)) return fail(RSLX_ERR_INVALID_ARG, "%s: null %s", who, cfg ? "matrices" : "configuration");
  if (count < 0 || count > RSLX_MUON_MAX_MATRICES) return fail(RSLX_ERR_SHAPE, "%s: %d matrices, 0 to %d are taken", who, count, RSLX_MUON_MAX_MATRICES);
  if (cfg->steps < 1 || cfg->steps > RSLX_MUON_MAX_STEPS) return fail(RSLX_ERR_SHAPE, "%s: %d steps, 1 to %d are taken", who, cfg->steps, RSLX_MUON_MAX_STEPS);
  for (int i = 0; i < count; ++i)
    if (m[i].rows < 1 || m[i].rows > RSLX_MUON_MAX_DIM || m[i].cols < 1 || m[i].cols > RSLX_MUON_MAX_DIM)
      return fail(RSLX_ERR_SHAPE, "%s: matrix %d is %d x %d, 1 to %d are taken", who, i, m[i].rows, m[i].cols, RSLX_MUON_MAX_DIM);
  return RSLX_OK;
}

// The workspace: the table, then each matrix's part.
MuonTable* plan_muon(Carver& c, const rslx_muon_matrix* m, int32_t count, const rslx_muon_cfg& cfg, MuonTable& t) {
  memset(&t, 0, sizeof t);
  t.lr = cfg.lr; t.momentum = cfg.momentum; t.decay = cfg.weight_decay;
  t.nesterov = cfg.nesterov;
  MuonTable* table = c.take<MuonTable>(1);
  for (int i = 0; i < count; ++i)
    t.item[i] = {m[i].w_in, m[i].w_out, m[i].grad, m[i].m_in, m[i].m_out, c.take<char>(muon_item_bytes(m[i].rows, m[i].cols)), m[i].rows, m[i].cols, m[i].scale};
  t.parts = c.take<float>(plan_muon_parts(t, count));
  return table;
}

}  // namespace

extern "C" {

size_t rslx_gated_recurrence_workspace_bytes(const rslx_gated_rec* a) { return rec_workspace(a, false, "rslx_gated_recurrence_workspace_bytes"); }

int32_t rslx_gated_recurrence(const rslx_gated_rec* a, const rslx_seq_view* x, const rslx_seq_view* g, const float* s0_or_null, const rslx_seq_view* h,
                              float* s_last_or_null, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "rslx_gated_recurrence";
  RSLX_TRY(check_rec(a, who, false));
  if (a->N == 0) return RSLX_OK;
  if (a->T > 0) {
    RSLX_TRY(check_view(*a, x, false, who, "x"));
    RSLX_TRY(check_view(*a, g, false, who, "g"));
    RSLX_TRY(check_view(*a, h, true, who, "h"));
  }
  RSLX_TRY(check_state(s0_or_null, who, "s0"));
  RSLX_TRY(check_state(s_last_or_null, who, "s_last"));
  const Named dones{block_of(a->dones, (int64_t)a->T * a->N), "dones"}, lengths{block_of(a->lengths, (int64_t)a->N * 4), "lengths"};
  const Named s0 = named(*a, s0_or_null, "s0");
  const Named all[] = {named(*a, h, "h"), named(*a, s_last_or_null, "s_last"), named(*a, x, "x"), named(*a, g, "g"), dones, lengths};
  RSLX_TRY(check_apart(all, 2, who));
  const Named of_h[] = {all[0], s0}, of_state[] = {all[1], s0};
  RSLX_TRY(check_apart(of_h, 1, who));
  if (s0_or_null != s_last_or_null) RSLX_TRY(check_apart(of_state, 1, who));
  RecArgs r = rec_args(*a);
  r.x = matrix(x); r.g = matrix(g); r.h = matrix(h);
  RSLX_TRY(rec_plan(r, a->dtype, false, ws, ws_bytes, who));
  r.s0 = s0_or_null; r.s_last = s_last_or_null;
  RSLX_HIP(launch_recurrence(r, a->dtype, false, (hipStream_t)stream));
  return RSLX_OK;
}

size_t rslx_gated_recurrence_backward_workspace_bytes(const rslx_gated_rec* a) {
  return rec_workspace(a, true, "rslx_gated_recurrence_backward_workspace_bytes");
}

int32_t rslx_gated_recurrence_backward(const rslx_gated_rec* a, const rslx_seq_view* x, const rslx_seq_view* g, const float* s0_or_null,
                                       const rslx_seq_view* dh, const float* ds_last_or_null, const rslx_seq_view* dx, const rslx_seq_view* dg,
                                       float* ds0_or_null, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "rslx_gated_recurrence_backward";
  RSLX_TRY(check_rec(a, who, false));
  if (a->N == 0) return RSLX_OK;
  if (a->T > 0) {
    RSLX_TRY(check_view(*a, x, false, who, "x"));
    RSLX_TRY(check_view(*a, g, false, who, "g"));
    RSLX_TRY(check_view(*a, dh, false, who, "dh"));
    RSLX_TRY(check_view(*a, dx, true, who, "dx"));
    RSLX_TRY(check_view(*a, dg, true, who, "dg"));
  }
  RSLX_TRY(check_state(s0_or_null, who, "s0"));
  RSLX_TRY(check_state(ds_last_or_null, who, "ds_last"));
  RSLX_TRY(check_state(ds0_or_null, who, "ds0"));
  const Named all[] = {named(*a, dx, "dx"), named(*a, dg, "dg"), named(*a, ds0_or_null, "ds0"), named(*a, x, "x"), named(*a, g, "g"), named(*a, dh, "dh"),
                       named(*a, s0_or_null, "s0"), named(*a, ds_last_or_null, "ds_last"), {block_of(a->dones, (int64_t)a->T * a->N), "dones"},
                       {block_of(a->lengths, (int64_t)a->N * 4), "lengths"}};
  RSLX_TRY(check_apart(all, 3, who));
  RecArgs r = rec_args(*a);
  r.x = matrix(x); r.g = matrix(g); r.dh = matrix(dh); r.dx = matrix(dx); r.dg = matrix(dg);
  RSLX_TRY(rec_plan(r, a->dtype, true, ws, ws_bytes, who));
  r.s0 = s0_or_null; r.ds_last = ds_last_or_null; r.ds0 = ds0_or_null;
  RSLX_HIP(launch_recurrence(r, a->dtype, true, (hipStream_t)stream));
  return RSLX_OK;
}

int32_t rslx_gated_recurrence_step(const rslx_gated_rec* a, const rslx_seq_view* x, const rslx_seq_view* g, const uint8_t* reset_or_null,
                                   const float* s_in_or_null, float* s_out, const rslx_seq_view* h, void* stream) {
  const char* who = "rslx_gated_recurrence_step";
  RSLX_TRY(check_rec(a, who, true));
  if (a->N == 0) return RSLX_OK;
  RSLX_TRY(check_view(*a, x, false, who, "x"));
  RSLX_TRY(check_view(*a, g, false, who, "g"));
  RSLX_TRY(check_view(*a, h, true, who, "h"));
  if (!s_out) return fail(RSLX_ERR_INVALID_ARG, "%s: null s_out", who);
  RSLX_TRY(check_state(s_in_or_null, who, "s_in"));
  RSLX_TRY(check_state(s_out, who, "s_out"));
  const Named reset{block_of(reset_or_null, a->N), "reset"}, s_in = named(*a, s_in_or_null, "s_in");
  const Named out = named(*a, h, "h"), in[] = {named(*a, x, "x"), named(*a, g, "g")};
  const Named of_state[] = {named(*a, s_out, "s_out"), out, in[0], in[1], reset}, of_both[] = {of_state[0], s_in}, of_h[] = {out, s_in, reset};
  RSLX_TRY(check_apart(of_state, 1, who));
  if (s_in_or_null != s_out) RSLX_TRY(check_apart(of_both, 1, who));
  RSLX_TRY(check_apart(of_h, 1, who));
  for (const Named& v : in)                    // (a lane reads its values of x and g before it writes h)
    if (!same_rows(out.rows, v.rows) && share_memory(out.rows, v.rows))
      return fail(RSLX_ERR_INVALID_ARG, "%s: h overlaps %s, and not row by row", who, v.name);
  RecArgs r = rec_args(*a);
  r.x = matrix(x); r.g = matrix(g); r.h = matrix(h);
  r.dones = reset_or_null;
  r.s0 = s_in_or_null; r.s_last = s_out;
  RSLX_HIP(launch_recurrence_step(r, a->dtype, (hipStream_t)stream));
  return RSLX_OK;
}

int32_t rslx_rms_norm(int32_t dtype, const void* x, int64_t ldx, const void* residual_or_null, int64_t ldr, int64_t rows, int32_t cols,
                      const float* weight_or_null, float eps, void* total_or_null, int64_t ldt, void* y, int64_t ldy, float* rstd_or_null, void* stream) {
  return rms_norm(dtype, false, x, ldx, residual_or_null, ldr, rows, cols, weight_or_null, eps, total_or_null, ldt, y, ldy, nullptr, rstd_or_null, stream,
                  "rslx_rms_norm");
}

int32_t rslx_rms_norm_e4m3(int32_t dtype, const void* x, int64_t ldx, const void* residual_or_null, int64_t ldr, int64_t rows, int32_t cols,
                           const float* weight_or_null, float eps, void* total_or_null, int64_t ldt, void* y8, int64_t ldy, float* scales,
                           float* rstd_or_null, void* stream) {
  return rms_norm(dtype, true, x, ldx, residual_or_null, ldr, rows, cols, weight_or_null, eps, total_or_null, ldt, y8, ldy, scales, rstd_or_null, stream,
                  "rslx_rms_norm_e4m3");
}

size_t rslx_rms_norm_backward_workspace_bytes(int64_t rows, int32_t cols) {
  if (check_rows(RSLX_F32, rows, cols, "rslx_rms_norm_backward_workspace_bytes") != RSLX_OK) return 0;
  return (size_t)rms_backward_blocks(rows, cols) * cols * sizeof(float);
}

int32_t rslx_rms_norm_backward(int32_t dtype, const void* dy, int64_t lddy, const void* total, int64_t ldt, int64_t rows, int32_t cols,
                               const float* weight_or_null, const float* rstd, const void* dtotal_or_null, int64_t lddt, void* dx_or_null, int64_t lddx,
                               float* dweight_or_null, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "rslx_rms_norm_backward";
  RSLX_TRY(check_rows(dtype, rows, cols, who));
  if (rows > 0 && (!dy || !total || !rstd)) return fail(RSLX_ERR_INVALID_ARG, "%s: null dy, total or rstd", who);
  const int size = type_size(dtype);
  const NormMatrix in[] = {{dy, lddy, size, "dy"}, {total, ldt, size, "total"}, {dtotal_or_null, lddt, size, "dtotal"}}, out{dx_or_null, lddx, size, "dx"};
  for (const NormMatrix& m : in) RSLX_TRY(check_aligned(m, who));
  RSLX_TRY(check_aligned(out, who));
  RSLX_TRY(check_written(out, rows, cols, who));
  if (!aligned16(weight_or_null)) return fail(RSLX_ERR_INVALID_ARG, "%s: weight not 16-byte aligned", who);
  for (const NormMatrix& m : in) RSLX_TRY(check_in_place(out, m, rows, cols, who));
  const Named written[] = {{out.rows(rows, cols), "dx"}, {floats_of(dweight_or_null, cols), "dweight"},
                           {floats_of(weight_or_null, cols), "weight"}, {floats_of(rstd, rows), "rstd"}};
  RSLX_TRY(check_apart(written, 2, who));
  const Named sums[] = {written[1], {in[0].rows(rows, cols), "dy"}, {in[1].rows(rows, cols), "total"}, {in[2].rows(rows, cols), "dtotal"}};
  RSLX_TRY(check_apart(sums, 1, who));
  if (!dweight_or_null && (!dx_or_null || rows == 0)) return RSLX_OK;
  const size_t need = dweight_or_null ? rslx_rms_norm_backward_workspace_bytes(rows, cols) : 0;
  if (need > 0 && (!ws || ws_bytes < need)) return fail(RSLX_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, ws_bytes, need);
  if (need > 0 && !aligned16(ws)) return fail(RSLX_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", who);
  RmsArgs a;
  memset(&a, 0, sizeof a);
  a.x = total; a.ldx = ldt; a.dy = dy; a.lddy = lddy; a.residual = dtotal_or_null; a.ldr = lddt; a.y = dx_or_null; a.ldy = lddx;
  a.rows = rows; a.cols = cols;
  a.weight = weight_or_null;
  a.rstd = const_cast<float*>(rstd);
  a.partials = dweight_or_null ? static_cast<float*>(ws) : nullptr;
  a.dweight = dweight_or_null;
  RSLX_HIP(launch_rms_norm_backward(a, dtype, (hipStream_t)stream));
  return RSLX_OK;
}

size_t rslx_muon_step_workspace_bytes(const rslx_muon_matrix* matrices, int32_t count, const rslx_muon_cfg* cfg) {
  if (check_muon(matrices, count, cfg, "rslx_muon_step_workspace_bytes") != RSLX_OK) return 0;
  Carver c(nullptr);
  MuonTable t;
  plan_muon(c, matrices, count, *cfg, t);
  return c.off > 256 ? c.off : 256;
}

int32_t rslx_muon_step(const rslx_muon_matrix* matrices, int32_t count, const rslx_muon_cfg* cfg, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "rslx_muon_step";
  RSLX_TRY(check_muon(matrices, count, cfg, who));
  if (count == 0) return RSLX_OK;
  // everything that is written, then everything that is read, by matrix
  struct Range { uintptr_t lo, hi; int matrix; bool written; const char* name; };
  Range ranges[5 * RSLX_MUON_MAX_MATRICES];
  int n = 0;
  for (int i = 0; i < count; ++i) {
    const rslx_muon_matrix& m = matrices[i];
    if (!m.w_out || !m.grad) return fail(RSLX_ERR_INVALID_ARG, "%s: matrix %d: null w_out or grad", who, i);
    const struct { const float* p; bool written; const char* name; } all[] = {
        {m.w_out, true, "w_out"}, {m.m_out, true, "m_out"}, {m.grad, false, "grad"}, {m.w_in == m.w_out ? nullptr : m.w_in, false, "w_in"},
        {m.m_in == m.m_out ? nullptr : m.m_in, false, "m_in"}};
    for (const auto& x : all) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(x.p);
      if (at % sizeof(float)) return fail(RSLX_ERR_INVALID_ARG, "%s: matrix %d: %s not aligned to its type", who, i, x.name);
      if (x.p) ranges[n++] = {at, at + (uintptr_t)m.rows * m.cols * sizeof(float), i, x.written, x.name};
    }
  }
  // by their starts: a range meets an earlier one where it starts before the furthest end of those that are written, or, written itself, of all
  std::sort(ranges, ranges + n, [](const Range& x, const Range& y) { return x.lo < y.lo; });
  const Range *far = nullptr, *far_written = nullptr;
  for (int i = 0; i < n; ++i) {
    const Range& r = ranges[i];
    const Range* meets = r.written && far && r.lo < far->hi ? far : far_written && r.lo < far_written->hi ? far_written : nullptr;
    if (meets)
      return fail(RSLX_ERR_INVALID_ARG, "%s: %s of matrix %d overlaps %s of matrix %d", who, r.name, r.matrix, meets->name, meets->matrix);
    if (!far || r.hi > far->hi) far = &r;
    if (r.written && (!far_written || r.hi > far_written->hi)) far_written = &r;
  }
  Carver c(ws);
  MuonTable t;
  MuonTable* table = plan_muon(c, matrices, count, *cfg, t);
  if (!ws || ws_bytes < c.off) return fail(RSLX_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, ws_bytes, c.off);
  if (!aligned16(ws)) return fail(RSLX_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", who);
  RSLX_HIP(launch_muon(t, count, table, cfg->steps, (hipStream_t)stream));
  return RSLX_OK;
}

}  // extern "C"
