// Host-only exercise of the sequence operators' entry points for a sanitizer build of the library (address + undefined behaviour
// on the host code): workspace queries at every extreme of T, N and H, and the argument checks that return before anything is launched.
// Needs no GPU; pointers that stand for device memory are never dereferenced here.
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

static float memory[4096] __attribute__((aligned(16)));

static rslx_linear_attn attn(int32_t dtype, int64_t T, int64_t N, int64_t H, int32_t Dk, int32_t Dv) {
  rslx_linear_attn a;
  std::memset(&a, 0, sizeof a);
  a.dtype = dtype;
  a.T = (int32_t)T; a.N = (int32_t)N; a.H = (int32_t)H;
  a.Dk = Dk; a.Dv = Dv;
  a.scale = 1.f;
  a.log_decay = memory;
  return a;
}

static bool said(const char* text) { return std::strstr(rslx_last_error(), text) != nullptr; }

int main() {
  const int32_t sizes[] = {0, 1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 4096, 65535, 65537, 1 << 20, 1 << 23, 1 << 24, (1 << 24) + 1, 1 << 30,
                           INT_MAX - 1024, INT_MAX - 65, INT_MAX - 64, INT_MAX - 63, INT_MAX - 32, INT_MAX - 31, INT_MAX - 30, INT_MAX - 1, INT_MAX};
  const int32_t widths[] = {1, 2, 31, 32, 33, 64, 65, 127, 128};

  // ---- workspace queries, and calls that differ from them in a null pointer only ----
  for (int32_t dtype = RSLX_F32; dtype <= RSLX_F16; ++dtype)
    for (int32_t T : sizes)
      for (int32_t N : sizes)
        for (int32_t H : {0, 1, 3, 1024, 1 << 24, INT_MAX})
          for (int w = 0; w < 9; w += (T > 4096 ? 1 : 4)) {
            rslx_linear_attn a = attn(dtype, T, N, H, widths[w], widths[8 - w]);
            const size_t forward = rslx_linear_attention_workspace_bytes(&a), backward = rslx_linear_attention_backward_workspace_bytes(&a);
            CHECK((forward == 0) == (backward == 0));
            CHECK(forward == 0 || (forward >= 256 && backward >= 256));
            CHECK(forward == 0 || T == 0 || (int64_t)N * H == 0 || rslx_linear_attention(&a, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == 1);
          }
  rslx_linear_attn a = attn(RSLX_F32, INT_MAX - 63, 1, 1, 8, 8);
  CHECK(rslx_linear_attention_workspace_bytes(&a) == 0 && said("T = 2147483584"));
  a = attn(RSLX_F32, 8, 1 << 24, 2, 8, 8);
  CHECK(rslx_linear_attention_workspace_bytes(&a) == 0 && said("N * H"));
  CHECK(rslx_linear_attention_workspace_bytes(nullptr) == 0 && rslx_linear_attention_backward_workspace_bytes(nullptr) == 0);

  // ---- views: strides at the limits of their type ----
  const int64_t strides[] = {0, 1, -1, 8, -8, 64, INT_MAX, -(int64_t)INT_MAX, (int64_t)1 << 40, INT64_MAX / 4, INT64_MIN / 4, INT64_MAX, INT64_MIN};
  a = attn(RSLX_F32, 3, 2, 4, 8, 8);
  rslx_seq_view row{memory, 0, 0, 0};
  for (int64_t step : strides)
    for (int64_t seq : strides)
      for (int64_t head : strides) {
        rslx_seq_view o{memory + 1024, step, seq, head};
        const int32_t rc = rslx_linear_attention(&a, &row, &row, &row, memory + 2048, &o, memory + 2048, nullptr, 0, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_HIP);
      }
  rslx_seq_view o{memory + 1024, 64, 32, 8}, none{nullptr, 64, 32, 8}, odd{reinterpret_cast<char*>(memory) + 2, 64, 32, 8};
  CHECK(rslx_linear_attention(&a, &row, &row, &row, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == RSLX_ERR_INVALID_ARG && said("null o"));
  CHECK(rslx_linear_attention(&a, &none, &row, &row, nullptr, &o, nullptr, nullptr, 0, nullptr) == RSLX_ERR_INVALID_ARG && said("null q"));
  CHECK(rslx_linear_attention(&a, &row, &odd, &row, nullptr, &o, nullptr, nullptr, 0, nullptr) == RSLX_ERR_INVALID_ARG && said("k not aligned"));
  CHECK(rslx_linear_attention(&a, &row, &row, &row, memory + 1, &o, nullptr, nullptr, 0, nullptr) == RSLX_ERR_INVALID_ARG && said("s0 not 16-byte"));
  CHECK(rslx_linear_attention_backward(&a, &row, &row, &row, nullptr, &row, nullptr, &o, &o, &o, nullptr, nullptr, 0, nullptr) == RSLX_ERR_INVALID_ARG && said("overlaps"));
  CHECK(rslx_linear_attention_backward(&a, &row, &row, &row, nullptr, nullptr, nullptr, &o, &o, &o, nullptr, nullptr, 0, nullptr) == RSLX_ERR_INVALID_ARG && said("null do"));
  a = attn(RSLX_F32, 4000, 1, 1, 8, 8);
  o = {memory + 1024, 8, 0, 0};
  CHECK(rslx_linear_attention(&a, &row, &row, &row, nullptr, &o, nullptr, memory, 100, nullptr) == RSLX_ERR_WORKSPACE && said("workspace 100 <"));
  CHECK(rslx_linear_attention(&a, &row, &row, &row, nullptr, &o, nullptr, memory + 1, 1 << 30, nullptr) == RSLX_ERR_INVALID_ARG && said("not 16-byte"));
  a = attn(RSLX_F32, 0, 0, 4, 8, 8);
  CHECK(rslx_linear_attention(&a, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == RSLX_OK);
  a = attn(RSLX_F32, 1, 3, 4, 8, 8);
  o = {memory + 1024, 0, 32, 8};
  CHECK(rslx_linear_attention_step(&a, &row, &row, &row, nullptr, nullptr, nullptr, &o, nullptr) == RSLX_ERR_INVALID_ARG && said("null s_out"));
  CHECK(rslx_linear_attention_step(&a, &row, &row, &o, nullptr, nullptr, memory + 1024, &o, nullptr) == RSLX_ERR_INVALID_ARG && said("s_out overlaps"));
  CHECK(rslx_linear_attention_step(nullptr, &row, &row, &row, nullptr, nullptr, memory, &o, nullptr) == RSLX_ERR_INVALID_ARG);

  // ---- layer norm ----
  for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)3, (int64_t)1 << 20, (int64_t)1 << 40, INT64_MAX / 2, INT64_MAX - 1, INT64_MAX})
    for (int32_t cols : {1, 2, 64, 65, 512, 513, 4096, 16384}) CHECK(rslx_layer_norm_backward_workspace_bytes(rows, cols) > 0);
  CHECK(rslx_layer_norm_backward_workspace_bytes(-1, 8) == 0 && rslx_layer_norm_backward_workspace_bytes(4, 16385) == 0);
  for (int64_t ldx : strides)
    for (int64_t ldy : strides)
      for (int64_t rows : {(int64_t)1, (int64_t)3, (int64_t)1 << 31, (int64_t)1 << 40}) {
        const int32_t rc = rslx_layer_norm(RSLX_BF16, memory, ldx, rows, 8, nullptr, nullptr, 1e-5f, memory + 1024, ldy, nullptr, nullptr, nullptr);
        CHECK(rc == RSLX_ERR_SHAPE || rc == RSLX_ERR_INVALID_ARG || rc == RSLX_ERR_HIP);
      }
  CHECK(rslx_layer_norm(RSLX_F32, memory, 8, 4, 8, nullptr, nullptr, 1e-5f, memory + 4, 8, nullptr, nullptr, nullptr) == RSLX_ERR_INVALID_ARG && said("x and y overlap"));
  CHECK(rslx_layer_norm_backward(RSLX_F32, memory, 8, memory, 8, 4, 8, nullptr, memory, memory, memory + 4, 8, nullptr, nullptr, nullptr, 0, nullptr) ==
        RSLX_ERR_INVALID_ARG);
  CHECK(rslx_layer_norm_backward(RSLX_F32, nullptr, 8, nullptr, 8, 0, 8, nullptr, nullptr, nullptr, nullptr, 8, nullptr, nullptr, nullptr, 0, nullptr) == RSLX_OK);

  if (failures) { std::printf("%d checks failed\n", failures); return 1; }
  std::printf("all checks passed\n");
  return 0;
}
