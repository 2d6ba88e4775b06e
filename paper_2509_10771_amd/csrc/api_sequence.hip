// C ABI of the sequence operators: linear attention with a decay for each head, layer norm.  Argument checks, workspace planning and the
// order of the launches; the kernels are in linear_attention.hip and layer_norm.hip.
#include "overlap.h"
#include "sequence.h"

using namespace rslx;
using namespace rslx::host;

namespace {

constexpr int64_t MAX_HEADS = 1 << 24;       // N * H of a call

int32_t check_attn(const rslx_linear_attn* a, const char* who, bool step) {
  if (!a) return fail(RSLX_ERR_INVALID_ARG, "%s: null description", who);
  RSLX_TRY(check_dtype(a->dtype, who));
  if (a->T < 0 || a->T > RSLX_ATTN_MAX_STEPS || a->N < 0 || a->H < 0) return fail(RSLX_ERR_SHAPE, "%s: T = %d, N = %d, H = %d", who, a->T, a->N, a->H);
  if (a->Dk < 1 || a->Dk > RSLX_ATTN_MAX_DIM || a->Dv < 1 || a->Dv > RSLX_ATTN_MAX_DIM)
    return fail(RSLX_ERR_SHAPE, "%s: head widths %d and %d, 1 to %d are taken", who, a->Dk, a->Dv, RSLX_ATTN_MAX_DIM);
  if ((int64_t)a->N * a->H > MAX_HEADS) return fail(RSLX_ERR_SHAPE, "%s: N * H = %lld exceeds %lld", who, (long long)a->N * a->H, (long long)MAX_HEADS);
  if (step && (a->T != 1 || a->dones || a->lengths))
    return fail(RSLX_ERR_INVALID_ARG, "%s: one step has T = 1 and neither dones nor lengths", who);
  if ((int64_t)a->N * a->H > 0 && !a->log_decay) return fail(RSLX_ERR_INVALID_ARG, "%s: null log_decay", who);
  return RSLX_OK;
}

RowSet rows_of(const rslx_linear_attn& a, const rslx_seq_view& v, int width) {
  const int size = type_size(a.dtype);
  return {v.data, (int64_t)width * size, {(wide)v.step * size, (wide)v.seq * size, (wide)v.head * size}, {a.T, a.N, a.H}};
}

// A matrix [T, N, H, width] behind a view; written: no two of its elements may be the same memory.
int32_t check_view(const rslx_linear_attn& a, const rslx_seq_view* v, int width, bool written, const char* who, const char* name) {
  if (!v || !v->data) return fail(RSLX_ERR_INVALID_ARG, "%s: null %s", who, name);
  if (reinterpret_cast<uintptr_t>(v->data) % type_size(a.dtype) != 0) return fail(RSLX_ERR_INVALID_ARG, "%s: %s not aligned to its type", who, name);
  if (written && overlaps_itself(rows_of(a, *v, width)))
    return fail(RSLX_ERR_SHAPE, "%s: rows of %s overlap (strides %lld, %lld and %lld, width %d)", who, name, (long long)v->step, (long long)v->seq,
                (long long)v->head, width);
  return RSLX_OK;
}

int32_t check_state(const float* s, const char* who, const char* name) {
  if (s && !aligned16(s)) return fail(RSLX_ERR_INVALID_ARG, "%s: %s not 16-byte aligned", who, name);
  return RSLX_OK;
}

bool states_overlap(const rslx_linear_attn& a, const float* x, const float* y) {
  const uintptr_t n = (uintptr_t)a.N * a.H * a.Dk * a.Dv * sizeof(float);
  const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
  return x && y && p < q + n && q < p + n;
}

Named named(const rslx_linear_attn& a, const rslx_seq_view* v, int width, const char* name) {
  return a.T > 0 ? Named{rows_of(a, *v, width), name} : Named{{}, name};
}
Named named(const rslx_linear_attn& a, const float* state, const char* name) {
  return {{state, (int64_t)a.N * a.H * a.Dk * a.Dv * (int64_t)sizeof(float), {}, {1, 1, 1}}, name};
}

WalkMatrix matrix(const rslx_seq_view* v) { return v ? WalkMatrix{v->data, v->step, v->seq, v->head} : WalkMatrix{}; }

WalkArgs walk_args(const rslx_linear_attn& a) {
  WalkArgs w;
  memset(&w, 0, sizeof w);
  w.T = a.T; w.N = a.N; w.H = a.H;
  w.scale = a.scale;
  w.log_decay = a.log_decay;
  w.dones = a.dones;
  w.lengths = a.lengths;
  w.segments = 1;
  return w;
}

void add_job(WalkArgs& w, const rslx_seq_view* x, const rslx_seq_view* y, const rslx_seq_view* z, const rslx_seq_view* out, int D, int E, bool reversed,
             const float* s_in, bool transposed, float* s_out) {
  WalkJob& j = w.job[w.jobs++];
  j.a = matrix(x); j.b = matrix(y); j.c = matrix(z); j.o = matrix(out);
  j.D = D; j.E = E;
  j.reversed = reversed ? 1 : 0;
  j.s_in = s_in;
  j.in_row = transposed ? 1 : E;
  j.in_col = transposed ? D : 1;
  j.s_out = s_out;
}

// Pieces of the sequences, and the workspace: per set of states (S; backward also its gradient) one state per piece, and where episodes end.
struct AttnPlan {
  int32_t segments, seg_len, sets;
  float* states[2];
  int32_t* cuts;
  size_t bytes;
};

void plan_attn(Carver& c, const rslx_linear_attn& a, bool backward, AttnPlan& p) {
  memset(&p, 0, sizeof p);
  p.sets = backward ? 2 : 1;
  const int64_t heads = (int64_t)a.N * a.H;
  const int size = type_size(a.dtype);
  const int64_t waves = heads * (walk_waves_per_head(a.Dk, a.Dv, size) + (backward ? 2 * walk_waves_per_head(a.Dv, a.Dk, size) : 0));
  p.segments = walk_segments(waves, a.T, &p.seg_len);
  if (p.segments > 1) {
    for (int s = 0; s < p.sets; ++s) p.states[s] = c.take<float>((size_t)heads * p.segments * a.Dk * a.Dv);
    p.cuts = c.take<int32_t>((size_t)p.sets * a.N * p.segments);
  }
  p.bytes = c.off;
}

size_t attn_workspace(const rslx_linear_attn* a, bool backward, const char* who) {
  if (check_attn(a, who, false) != RSLX_OK) return 0;
  Carver c(nullptr);
  AttnPlan p;
  plan_attn(c, *a, backward, p);
  return p.bytes > 256 ? p.bytes : 256;
}

int32_t attn_plan(const rslx_linear_attn& a, bool backward, void* ws, size_t ws_bytes, const char* who, AttnPlan& p) {
  Carver c(ws);
  plan_attn(c, a, backward, p);
  if (p.bytes > 0 && (!ws || ws_bytes < p.bytes)) return fail(RSLX_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, ws_bytes, p.bytes);
  if (p.bytes > 0 && !aligned16(ws)) return fail(RSLX_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", who);
  return RSLX_OK;
}

}  // namespace

extern "C" {

size_t rslx_linear_attention_workspace_bytes(const rslx_linear_attn* a) { return attn_workspace(a, false, "rslx_linear_attention_workspace_bytes"); }

int32_t rslx_linear_attention(const rslx_linear_attn* a, const rslx_seq_view* q, const rslx_seq_view* k, const rslx_seq_view* v,
                              const float* s0_or_null, const rslx_seq_view* o, float* s_last_or_null, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "rslx_linear_attention";
  RSLX_TRY(check_attn(a, who, false));
  if ((int64_t)a->N * a->H == 0) return RSLX_OK;
  if (a->T > 0) {
    RSLX_TRY(check_view(*a, q, a->Dk, false, who, "q"));
    RSLX_TRY(check_view(*a, k, a->Dk, false, who, "k"));
    RSLX_TRY(check_view(*a, v, a->Dv, false, who, "v"));
    RSLX_TRY(check_view(*a, o, a->Dv, true, who, "o"));
  }
  RSLX_TRY(check_state(s0_or_null, who, "s0"));
  RSLX_TRY(check_state(s_last_or_null, who, "s_last"));
  if (s0_or_null != s_last_or_null && states_overlap(*a, s0_or_null, s_last_or_null)) return fail(RSLX_ERR_INVALID_ARG, "%s: s0 and s_last overlap", who);
  const Named all[] = {named(*a, o, a->Dv, "o"), named(*a, s_last_or_null, "s_last"), named(*a, q, a->Dk, "q"), named(*a, k, a->Dk, "k"),
                       named(*a, v, a->Dv, "v")};
  RSLX_TRY(check_apart(all, 2, who));
  const Named read[] = {all[0], named(*a, s0_or_null, "s0")};
  RSLX_TRY(check_apart(read, 1, who));
  AttnPlan p;
  RSLX_TRY(attn_plan(*a, false, ws, ws_bytes, who, p));
  const hipStream_t s = (hipStream_t)stream;
  const float* start = s0_or_null;
  if (p.segments > 1) {
    WalkArgs w = walk_args(*a);
    w.segments = p.segments; w.seg_len = p.seg_len; w.states_only = 1; w.cuts = p.cuts;
    add_job(w, nullptr, k, v, nullptr, a->Dk, a->Dv, false, nullptr, false, p.states[0]);
    RSLX_HIP(launch_walk(w, a->dtype, s));
    RSLX_HIP(launch_walk_join(w, &s0_or_null, s));
    start = p.states[0];
  }
  WalkArgs w = walk_args(*a);
  w.segments = p.segments; w.seg_len = p.seg_len;
  add_job(w, q, k, v, o, a->Dk, a->Dv, false, start, false, s_last_or_null);
  RSLX_HIP(launch_walk(w, a->dtype, s));
  return RSLX_OK;
}

size_t rslx_linear_attention_backward_workspace_bytes(const rslx_linear_attn* a) {
  return attn_workspace(a, true, "rslx_linear_attention_backward_workspace_bytes");
}

int32_t rslx_linear_attention_backward(const rslx_linear_attn* a, const rslx_seq_view* q, const rslx_seq_view* k, const rslx_seq_view* v,
                                       const float* s0_or_null, const rslx_seq_view* d_o, const float* ds_last_or_null, const rslx_seq_view* dq,
                                       const rslx_seq_view* dk, const rslx_seq_view* dv, float* ds0_or_null, void* ws, size_t ws_bytes,
                                       void* stream) {
  const char* who = "rslx_linear_attention_backward";
  RSLX_TRY(check_attn(a, who, false));
  if ((int64_t)a->N * a->H == 0) return RSLX_OK;
  if (a->T > 0) {
    RSLX_TRY(check_view(*a, q, a->Dk, false, who, "q"));
    RSLX_TRY(check_view(*a, k, a->Dk, false, who, "k"));
    RSLX_TRY(check_view(*a, v, a->Dv, false, who, "v"));
    RSLX_TRY(check_view(*a, d_o, a->Dv, false, who, "do"));
    RSLX_TRY(check_view(*a, dq, a->Dk, true, who, "dq"));
    RSLX_TRY(check_view(*a, dk, a->Dk, true, who, "dk"));
    RSLX_TRY(check_view(*a, dv, a->Dv, true, who, "dv"));
  }
  RSLX_TRY(check_state(s0_or_null, who, "s0"));
  RSLX_TRY(check_state(ds_last_or_null, who, "ds_last"));
  RSLX_TRY(check_state(ds0_or_null, who, "ds0"));
  if (states_overlap(*a, ds0_or_null, ds_last_or_null) || states_overlap(*a, ds0_or_null, s0_or_null))
    return fail(RSLX_ERR_INVALID_ARG, "%s: ds0 overlaps an input", who);
  const Named all[] = {named(*a, dq, a->Dk, "dq"), named(*a, dk, a->Dk, "dk"), named(*a, dv, a->Dv, "dv"), named(*a, ds0_or_null, "ds0"),
                       named(*a, q, a->Dk, "q"), named(*a, k, a->Dk, "k"), named(*a, v, a->Dv, "v"), named(*a, d_o, a->Dv, "do"),
                       named(*a, s0_or_null, "s0"), named(*a, ds_last_or_null, "ds_last")};
  RSLX_TRY(check_apart(all, 4, who));
  AttnPlan p;
  RSLX_TRY(attn_plan(*a, true, ws, ws_bytes, who, p));
  const hipStream_t s = (hipStream_t)stream;
  const float* start[2] = {s0_or_null, ds_last_or_null};
  if (p.segments > 1) {
    WalkArgs w = walk_args(*a);
    w.segments = p.segments; w.seg_len = p.seg_len; w.states_only = 1; w.cuts = p.cuts;
    add_job(w, nullptr, k, v, nullptr, a->Dk, a->Dv, false, nullptr, false, p.states[0]);
    add_job(w, nullptr, q, d_o, nullptr, a->Dk, a->Dv, true, nullptr, false, p.states[1]);
    RSLX_HIP(launch_walk(w, a->dtype, s));
    RSLX_HIP(launch_walk_join(w, start, s));
    start[0] = p.states[0];
    start[1] = p.states[1];
  }
  WalkArgs w = walk_args(*a);
  w.segments = p.segments; w.seg_len = p.seg_len;
  add_job(w, d_o, v, k, dq, a->Dv, a->Dk, false, start[0], true, nullptr);
  add_job(w, v, d_o, q, dk, a->Dv, a->Dk, true, start[1], true, nullptr);
  add_job(w, k, q, d_o, dv, a->Dk, a->Dv, true, start[1], false, ds0_or_null);
  RSLX_HIP(launch_walk(w, a->dtype, s));
  return RSLX_OK;
}

int32_t rslx_linear_attention_step(const rslx_linear_attn* a, const rslx_seq_view* q, const rslx_seq_view* k, const rslx_seq_view* v,
                                   const uint8_t* reset_or_null, const float* s_in_or_null, float* s_out, const rslx_seq_view* o, void* stream) {
  const char* who = "rslx_linear_attention_step";
  RSLX_TRY(check_attn(a, who, true));
  if ((int64_t)a->N * a->H == 0) return RSLX_OK;
  RSLX_TRY(check_view(*a, q, a->Dk, false, who, "q"));
  RSLX_TRY(check_view(*a, k, a->Dk, false, who, "k"));
  RSLX_TRY(check_view(*a, v, a->Dv, false, who, "v"));
  RSLX_TRY(check_view(*a, o, a->Dv, true, who, "o"));
  if (!s_out) return fail(RSLX_ERR_INVALID_ARG, "%s: null s_out", who);
  RSLX_TRY(check_state(s_in_or_null, who, "s_in"));
  RSLX_TRY(check_state(s_out, who, "s_out"));
  if (s_in_or_null != s_out && states_overlap(*a, s_in_or_null, s_out)) return fail(RSLX_ERR_INVALID_ARG, "%s: s_in and s_out overlap", who);
  const Named out = named(*a, o, a->Dv, "o"), in[] = {named(*a, q, a->Dk, "q"), named(*a, k, a->Dk, "k"), named(*a, v, a->Dv, "v")};
  const Named states[] = {named(*a, s_out, "s_out"), out, in[0], in[1], in[2]}, read[] = {out, named(*a, s_in_or_null, "s_in")};
  RSLX_TRY(check_apart(states, 1, who));
  RSLX_TRY(check_apart(read, 1, who));
  for (const Named& x : in)                    // (a head's q, k and v are read before its o is written)
    if (!same_rows(out.rows, x.rows) && share_memory(out.rows, x.rows))
      return fail(RSLX_ERR_INVALID_ARG, "%s: o overlaps %s, and not row by row", who, x.name);
  StepArgs t;
  memset(&t, 0, sizeof t);
  t.q = matrix(q); t.k = matrix(k); t.v = matrix(v); t.o = matrix(o);
  t.N = a->N; t.H = a->H; t.Dk = a->Dk; t.Dv = a->Dv;
  t.scale = a->scale;
  t.log_decay = a->log_decay;
  t.reset = reset_or_null;
  t.s_in = s_in_or_null;
  t.s_out = s_out;
  RSLX_HIP(launch_attention_step(t, a->dtype, (hipStream_t)stream));
  return RSLX_OK;
}

int32_t rslx_layer_norm(int32_t dtype, const void* x, int64_t ldx, int64_t rows, int32_t cols, const float* weight_or_null,
                        const float* bias_or_null, float eps, void* y, int64_t ldy, float* mean_or_null, float* rstd_or_null, void* stream) {
  const char* who = "rslx_layer_norm";
  RSLX_TRY(check_dtype(dtype, who));
  if (rows < 0 || cols < 1 || cols > RSLX_NORM_MAX_COLS)
    return fail(RSLX_ERR_SHAPE, "%s: %lld rows of %d, 1 to %d columns are taken", who, (long long)rows, cols, RSLX_NORM_MAX_COLS);
  if (rows == 0) return RSLX_OK;
  if (!x || !y) return fail(RSLX_ERR_INVALID_ARG, "%s: null x or y", who);
  if (reinterpret_cast<uintptr_t>(x) % type_size(dtype) || reinterpret_cast<uintptr_t>(y) % type_size(dtype))
    return fail(RSLX_ERR_INVALID_ARG, "%s: x or y not aligned to its type", who);
  if (rows > 1 && ldy < cols && ldy > -cols) return fail(RSLX_ERR_SHAPE, "%s: rows of y overlap (ldy %lld, %d columns)", who, (long long)ldy, cols);
  if (!aligned16(weight_or_null) || !aligned16(bias_or_null)) return fail(RSLX_ERR_INVALID_ARG, "%s: weight or bias not 16-byte aligned", who);
  const int size = type_size(dtype);
  RSLX_TRY(check_in_place(rows_of(y, ldy, rows, cols, size), rows_of(x, ldx, rows, cols, size), who, "x and y"));
  NormArgs a;
  memset(&a, 0, sizeof a);
  a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy;
  a.rows = rows; a.cols = cols;
  a.weight = weight_or_null; a.bias = bias_or_null; a.eps = eps;
  a.mean = mean_or_null; a.rstd = rstd_or_null;
  RSLX_HIP(launch_layer_norm(a, dtype, false, (hipStream_t)stream));
  return RSLX_OK;
}

size_t rslx_layer_norm_backward_workspace_bytes(int64_t rows, int32_t cols) {
  if (rows < 0 || cols < 1 || cols > RSLX_NORM_MAX_COLS) {
    fail(RSLX_ERR_SHAPE, "rslx_layer_norm_backward_workspace_bytes: %lld rows of %d", (long long)rows, cols);
    return 0;
  }
  return (size_t)2 * norm_backward_blocks(rows, cols) * cols * sizeof(float);
}

int32_t rslx_layer_norm_backward(int32_t dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t rows, int32_t cols,
                                 const float* weight_or_null, const float* mean, const float* rstd, void* dx_or_null, int64_t lddx,
                                 float* dweight_or_null, float* dbias_or_null, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "rslx_layer_norm_backward";
  RSLX_TRY(check_dtype(dtype, who));
  if (rows < 0 || cols < 1 || cols > RSLX_NORM_MAX_COLS)
    return fail(RSLX_ERR_SHAPE, "%s: %lld rows of %d, 1 to %d columns are taken", who, (long long)rows, cols, RSLX_NORM_MAX_COLS);
  if (rows > 0 && (!dy || !x || !mean || !rstd)) return fail(RSLX_ERR_INVALID_ARG, "%s: null dy, x, mean or rstd", who);
  const int size = type_size(dtype);
  if (reinterpret_cast<uintptr_t>(dy) % size || reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(dx_or_null) % size)
    return fail(RSLX_ERR_INVALID_ARG, "%s: dy, x or dx not aligned to its type", who);
  if (dx_or_null && rows > 1 && lddx < cols && lddx > -cols)
    return fail(RSLX_ERR_SHAPE, "%s: rows of dx overlap (lddx %lld, %d columns)", who, (long long)lddx, cols);
  if (!aligned16(weight_or_null)) return fail(RSLX_ERR_INVALID_ARG, "%s: weight not 16-byte aligned", who);
  if (dx_or_null && rows > 0) {
    const RowSet out = rows_of(dx_or_null, lddx, rows, cols, size);
    RSLX_TRY(check_in_place(out, rows_of(dy, lddy, rows, cols, size), who, "dx and dy"));
    RSLX_TRY(check_in_place(out, rows_of(x, ldx, rows, cols, size), who, "dx and x"));
  }
  const bool parameters = dweight_or_null || dbias_or_null;
  if (!parameters && (!dx_or_null || rows == 0)) return RSLX_OK;
  const size_t need = parameters ? rslx_layer_norm_backward_workspace_bytes(rows, cols) : 0;
  if (need > 0 && (!ws || ws_bytes < need)) return fail(RSLX_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, ws_bytes, need);
  if (need > 0 && !aligned16(ws)) return fail(RSLX_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", who);
  NormArgs a;
  memset(&a, 0, sizeof a);
  a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.dx = dx_or_null; a.lddx = lddx;
  a.rows = rows; a.cols = cols;
  a.weight = weight_or_null;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.partials = parameters ? static_cast<float*>(ws) : nullptr;
  a.dweight = dweight_or_null; a.dbias = dbias_or_null;
  RSLX_HIP(launch_layer_norm(a, dtype, true, (hipStream_t)stream));
  return RSLX_OK;
}

}  // extern "C"
