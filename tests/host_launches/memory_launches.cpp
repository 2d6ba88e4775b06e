// Which kernels the entry points around a gated memory launch for calls of given sizes and layouts, found on the host: this program takes the place of the HIP
// runtime's functions that register and launch kernels, and prints what it is asked to launch.  Nothing runs and no pointer is read; memory is told apart by
// addresses alone.
//
// A line of standard input is a call:
//   forward | backward | step  TYPE T N D  INSTEP INSEQ  OUTSTEP OUTSEQ     strides of x and g (g lies D values behind x) and of everything else, in values
//   muon  ROWSxCOLS,ROWSxCOLS,..
// and is answered by a line "kernel<..> GRIDxBLOCK; kernel<..> GRIDxBLOCK; ..", or by what the library said.
#include <cxxabi.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <map>
#include <sstream>
#include <string>

#include "../../include/rslx.h"

struct Size { uint32_t x, y, z; };

static std::map<const void*, std::string>& names() {      // (filled while the library is loaded, before this file's own statics are)
  static std::map<const void*, std::string> m;
  return m;
}
static std::string launched;
static Size grid_size, block_size;

extern "C" {
void __hipRegisterFunction(void**, const void* function, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[function] = name; }
int __hipPushCallConfiguration(Size grid, Size block, size_t, void*) {
  grid_size = grid;
  block_size = block;
  return 0;
}
int __hipPopCallConfiguration(Size* grid, Size* block, size_t* shared, void** stream) {
  *grid = grid_size;
  *block = block_size;
  *shared = 0;
  *stream = nullptr;
  return 0;
}
int hipLaunchKernel(const void* function, Size grid, Size block, void**, size_t, void*) {
  int status = 0;
  char* text = abi::__cxa_demangle(names()[function].c_str(), nullptr, nullptr, &status);
  std::string name = text ? text : "?";
  std::free(text);
  for (const char* skip : {"void ", "rslx::(anonymous namespace)::", "rslx::"})
    for (size_t at; (at = name.find(skip)) != std::string::npos;) name.erase(at, std::strlen(skip));
  size_t end = 0;
  for (int depth = 0; end < name.size() && (depth > 0 || name[end] != '('); ++end) depth += (name[end] == '<') - (name[end] == '>');      // without its arguments
  launched += name.substr(0, end) + " " + std::to_string((uint64_t)grid.x * grid.y * grid.z) + "x" + std::to_string(block.x) + "; ";
  return 0;
}
int hipGetLastError() { return 0; }
}

static char* place(int i) { return reinterpret_cast<char*>((uintptr_t)1 << 44) + ((int64_t)i << 40); }      // a terabyte each

int main() {
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string kind;
    in >> kind;
    launched.clear();
    int32_t rc = RSLX_ERR_INVALID_ARG;
    if (kind == "muon") {
      std::string shapes;
      in >> shapes;
      rslx_muon_matrix m[RSLX_MUON_MAX_MATRICES];
      int32_t count = 0;
      std::istringstream all(shapes);
      for (std::string one; count < RSLX_MUON_MAX_MATRICES && std::getline(all, one, ','); ++count) {
        m[count] = {nullptr, reinterpret_cast<float*>(place(2 * count)), reinterpret_cast<float*>(place(2 * count + 1)), nullptr, nullptr, 0, 0, 1.f};
        std::sscanf(one.c_str(), "%dx%d", &m[count].rows, &m[count].cols);
      }
      const rslx_muon_cfg cfg{0.1f, 0.9f, 0.f, 1, 2};
      rc = rslx_muon_step(m, count, &cfg, place(100), rslx_muon_step_workspace_bytes(m, count, &cfg), nullptr);
    } else {
      rslx_gated_rec a;
      std::memset(&a, 0, sizeof a);
      int64_t in_step, in_seq, out_step, out_seq;
      in >> a.dtype >> a.T >> a.N >> a.D >> in_step >> in_seq >> out_step >> out_seq;
      const int size = a.dtype == RSLX_F32 ? 4 : 2;
      const rslx_seq_view x{place(0), in_step, in_seq, 0}, g{place(0) + (int64_t)a.D * size, in_step, in_seq, 0};
      const rslx_seq_view p{place(1), out_step, out_seq, 0}, q{place(2), out_step, out_seq, 0}, r{place(3), out_step, out_seq, 0};
      float *s = reinterpret_cast<float*>(place(4)), *t = reinterpret_cast<float*>(place(5));
      if (kind == "forward") rc = rslx_gated_recurrence(&a, &x, &g, s, &p, t, place(6), rslx_gated_recurrence_workspace_bytes(&a), nullptr);
      else if (kind == "backward")
        rc = rslx_gated_recurrence_backward(&a, &x, &g, s, &p, t, &q, &r, nullptr, place(6), rslx_gated_recurrence_backward_workspace_bytes(&a), nullptr);
      else if (kind == "step") rc = rslx_gated_recurrence_step(&a, &x, &g, nullptr, s, t, &p, nullptr);
    }
    std::printf("%s\n", rc == RSLX_OK ? launched.c_str() : rslx_last_error());
  }
  return 0;
}
