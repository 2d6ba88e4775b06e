// Host-only exercise of the entry points around a gated memory (gated linear recurrence, RMS norm, Muon step) for a sanitizer build of the library (address +
// undefined behaviour on the host code): workspace queries at the extremes of their sizes, and the argument checks that return before anything is
// launched.  Needs no GPU; pointers that stand for device memory are never dereferenced here.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "../../include/rslx.h"

static int failures = 0;
#define CHECK(cond)                                                                                                                \
  do {                                                                                                                             \
    if (!(cond)) { std::printf("FAILED %s:%d: %s  (last error: %s)\n", __FILE__, __LINE__, #cond, rslx_last_error()); ++failures; } \
  } while (0)

static float memory[8192] __attribute__((aligned(16)));

static rslx_gated_rec rec(int32_t dtype, int32_t T, int32_t N, int32_t D) {
  rslx_gated_rec a;
  std::memset(&a, 0, sizeof a);
  a.dtype = dtype;
  a.T = T; a.N = N; a.D = D;
  return a;
}

static bool said(const char* text) { return std::strstr(rslx_last_error(), text) != nullptr; }

int main() {
  const int32_t sizes[] = {0, 1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 4096, 65535, 65537, 1 << 20, 1 << 24, 1 << 30, INT_MAX - 65, INT_MAX - 64,
                           INT_MAX - 63, INT_MAX - 31, INT_MAX - 1, INT_MAX};
  // ---- gated linear recurrence: queries, and calls that differ from them in a null pointer only ----
  for (int32_t dtype = RSLX_F32; dtype <= RSLX_F16; ++dtype)
    for (int32_t T : sizes)
      for (int32_t N : sizes)
        for (int32_t D : sizes) {
          rslx_gated_rec a = rec(dtype, T, N, D);
          const size_t forward = rslx_gated_recurrence_workspace_bytes(&a), backward = rslx_gated_recurrence_backward_workspace_bytes(&a);
          CHECK(forward == 0 || forward >= 256);
          CHECK(backward == 0 || (backward >= 256 && forward >= 256));
          const int32_t rc = rslx_gated_recurrence(&a, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr);
          CHECK(T == 0 || N == 0 || D == 0 || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_SHAPE);
        }
  const int64_t strides[] = {0, 1, -1, 8, -8, 64, INT_MAX, -(int64_t)INT_MAX, (int64_t)1 << 40, INT64_MAX / 4, INT64_MIN / 4, INT64_MAX, INT64_MIN};
  rslx_seq_view row{memory, 0, 0, 0};
  for (int32_t T : {3, 300, 4000})
    for (int64_t step : strides)
      for (int64_t seq : strides) {
        rslx_gated_rec a = rec(RSLX_BF16, T, 2, 8);
        rslx_seq_view o{memory + 1024, step, seq, 0}, in{memory, step, seq, 0};
        int32_t rc = rslx_gated_recurrence(&a, &row, &in, memory + 2048, &o, memory + 2048, memory + 4096, 1 << 13, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_WORKSPACE || rc == RSLX_ERR_HIP);
        rc = rslx_gated_recurrence_backward(&a, &row, &in, nullptr, &row, nullptr, &o, &in, nullptr, memory + 4096, 1 << 13, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_WORKSPACE || rc == RSLX_ERR_HIP);
        a = rec(RSLX_F32, 1, 2, 8);
        rc = rslx_gated_recurrence_step(&a, &in, &row, nullptr, nullptr, memory + 2048, &o, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_HIP);
      }
  rslx_gated_rec a = rec(RSLX_F32, 0, 0, 8);
  CHECK(rslx_gated_recurrence(&a, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == RSLX_OK);
  CHECK(rslx_gated_recurrence_step(nullptr, &row, &row, nullptr, nullptr, memory, &row, nullptr) == RSLX_ERR_INVALID_ARG);

  // ---- root-mean-square norm ----
  for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)3, (int64_t)1 << 20, (int64_t)1 << 40, INT64_MAX / 2, INT64_MAX - 1, INT64_MAX})
    for (int32_t cols : {1, 2, 64, 65, 512, 513, 4096, 16384}) {
      CHECK(rslx_rms_norm_backward_workspace_bytes(rows, cols) > 0);
      int32_t rc = rslx_rms_norm(RSLX_F16, memory, cols, nullptr, 0, rows, cols, memory, 1e-5f, nullptr, 0, memory, cols, memory, nullptr);
      CHECK(rows == 0 ? rc == RSLX_OK : rc == RSLX_ERR_INVALID_ARG);                            // (rstd lies in x)
      rc = rslx_rms_norm_backward(RSLX_F32, memory, 0, memory, 0, rows, cols, nullptr, memory, nullptr, 0, nullptr, 0, memory + 4096, memory, 2, nullptr);
      CHECK(rc == RSLX_ERR_WORKSPACE || rc == RSLX_ERR_INVALID_ARG);
    }
  CHECK(rslx_rms_norm_backward_workspace_bytes(-1, 8) == 0 && rslx_rms_norm_backward_workspace_bytes(4, 16385) == 0);
  for (int64_t ldx : strides)
    for (int64_t ldy : strides)
      for (int64_t rows : {(int64_t)1, (int64_t)3, (int64_t)1 << 31, (int64_t)1 << 40}) {
        int32_t rc = rslx_rms_norm(RSLX_BF16, memory, ldx, memory + 64, ldy, rows, 8, nullptr, 1e-5f, memory + 2048, ldx, memory + 1024, ldy, nullptr, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_HIP);
        rc = rslx_rms_norm_e4m3(RSLX_F32, memory, ldx, nullptr, 0, rows, 8, nullptr, 1e-5f, nullptr, 0, memory + 1024, ldy, memory + 4096, nullptr, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_HIP);
        rc = rslx_rms_norm_backward(RSLX_BF16, memory, ldx, memory + 64, ldy, rows, 8, nullptr, memory + 4096, memory + 128, ldy, memory + 1024, ldx, nullptr, nullptr, 0,
                                    nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_HIP);
      }

  // ---- Muon step ----
  rslx_muon_matrix m[RSLX_MUON_MAX_MATRICES];
  rslx_muon_cfg cfg{0.1f, 0.9f, 0.f, 1, 5};
  for (int32_t rows : sizes)
    for (int32_t cols : sizes)
      for (int32_t count : {0, 1, 2, 32}) {
        for (rslx_muon_matrix& x : m) x = {memory, memory, memory + 1024, nullptr, nullptr, rows, cols, 1.f};
        const size_t need = rslx_muon_step_workspace_bytes(m, count, &cfg);
        CHECK((need == 0) == (count > 0 && (rows < 1 || cols < 1 || rows > RSLX_MUON_MAX_DIM || cols > RSLX_MUON_MAX_DIM)));
        const int32_t rc = rslx_muon_step(m, count, &cfg, memory, 16, nullptr);
        CHECK(count == 0 ? rc == RSLX_OK : rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_WORKSPACE);
      }
  for (int32_t count : {-1, 33, INT_MAX, INT_MIN}) CHECK(rslx_muon_step_workspace_bytes(m, count, &cfg) == 0 && rslx_muon_step(m, count, &cfg, memory, 16, nullptr) == RSLX_ERR_SHAPE);
  for (int32_t steps : {0, -1, 33, INT_MAX, INT_MIN}) {
    cfg.steps = steps;
    CHECK(rslx_muon_step_workspace_bytes(m, 1, &cfg) == 0 && said("steps"));
  }
  CHECK(rslx_muon_step_workspace_bytes(m, 1, nullptr) == 0 && rslx_muon_step_workspace_bytes(nullptr, 1, &cfg) == 0);

  if (failures) { std::printf("%d checks failed\n", failures); return 1; }
  std::printf("all checks passed\n");
  return 0;
}
