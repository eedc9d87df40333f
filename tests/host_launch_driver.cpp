// The launches that libmoeprune makes, on the CPU: this program takes the place of the HIP runtime's launch functions, notes every
// launch's kernel and grid, and runs nothing.  A grid has to have fewer than 2^32 threads along each dimension (a launch's packet holds
// them in 32 bits), and the pieces that a job is cut into have to make up the whole of it.
// Built and run by tests/test_host_launches.py.
#include <cinttypes>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "moeprune.h"

struct Dim3 { uint32_t x, y, z; };
struct Launch { std::string kernel; Dim3 grid, block; };
static std::vector<Launch> launches;
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static struct { Dim3 grid, block; size_t lds; void* stream; } pending;

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* device, unsigned, void*, void*, void*, void*, int*) { names()[host] = device; }
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream) { pending = {grid, block, lds, stream}; return 0; }
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
  *grid = pending.grid; *block = pending.block; *lds = pending.lds; *stream = pending.stream;
  return 0;
}
int hipLaunchKernel(const void* f, Dim3 grid, Dim3 block, void**, size_t, void*) { launches.push_back({names()[f], grid, block}); return 0; }
int hipGetLastError() { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int* v, int, int) { *v = 256; return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
const char* hipGetErrorString(int) { return "?"; }
}

static int failures = 0;
#define EXPECT(cond)                                                                                     \
  do {                                                                                                   \
    if (!(cond)) { ++failures; std::printf("FAILED line %d: %s: %s\n", __LINE__, what, #cond); }         \
  } while (0)

// Every launch since the last call of this: the limits, and how many workgroups the kernels of a name had in all.
static std::map<std::string, int64_t> check(const char* what) {
  std::map<std::string, int64_t> blocks;
  for (const Launch& l : launches) {
    const uint32_t g[3] = {l.grid.x, l.grid.y, l.grid.z}, b[3] = {l.block.x, l.block.y, l.block.z};
    for (int d = 0; d < 3; ++d) {
      EXPECT(g[d] > 0 && b[d] > 0);
      if ((uint64_t)g[d] * b[d] >> 32) {
        ++failures;
        std::printf("FAILED %s: %s: dimension %d has %" PRIu64 " threads\n", what, l.kernel.c_str(), d, (uint64_t)g[d] * b[d]);
      }
      EXPECT(d == 0 || g[d] <= 65535);
    }
    for (const char* n : {"transpose_kernel", "branch_gradients_kernel", "silu_product_kernel", "distill_topk_kernel", "token_logprobs_kernel"})
      if (l.kernel.find(n) != std::string::npos) blocks[n] += (int64_t)l.grid.x * l.grid.y;
  }
  EXPECT(!launches.empty());
  launches.clear();
  return blocks;
}

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int main() {
  auto at = [](int64_t i) { return (void*)((uintptr_t)(i + 1) << 44); };   // never read
  auto f = [&](int64_t i) { return (float*)at(i); };
  const size_t room = ~(size_t)0;

  // ---- one expert's block: rows by the hundred million, and products of rows and columns beyond 2^34
  struct { int64_t T; int H, F; moep_dtype dt; } shapes[] = {
      {((int64_t)1 << 28) + 52, 4, 4, MOEP_F32}, {((int64_t)1 << 30) - 64, 4, 4, MOEP_F32}, {(int64_t)1 << 29, 8, 4, MOEP_F32},
      {1250000, 64, 14336, MOEP_F32}, {(int64_t)1 << 30, 64, 64, MOEP_BF16}, {(int64_t)1 << 29, 4096, 14336, MOEP_BF16},
      {((int64_t)1 << 30) - 1, 128, 64, MOEP_BF16}, {777, 1024, 3584, MOEP_BF16}, {1501, 512, 1024, MOEP_F32}, {1, 64, 64, MOEP_BF16}};
  for (auto& q : shapes) {
    char what[96];
    std::snprintf(what, sizeof what, "T %" PRId64 " H %d F %d dtype %d", q.T, q.H, q.F, (int)q.dt);
    EXPECT(expert_ffn_forward_workspace(q.T, q.H, q.F, q.dt, 1) > 0 && expert_ffn_backward_workspace(q.T, q.H, q.F, q.dt) > 0);
    EXPECT(expert_ffn_forward(at(1), at(2), at(3), at(4), q.T, q.H, q.F, q.dt, at(5), f(6), at(7), room, nullptr) == MOEP_OK);
    std::map<std::string, int64_t> n = check(what);
    if (q.dt == MOEP_F32) EXPECT(n["silu_product_kernel"] == up(q.T * q.F / 4, 256));
    for (int wanted = 1; wanted < 4; ++wanted) {             // dx, the weights' gradients, both
      void* dx = wanted & 1 ? at(8) : nullptr;
      const bool weights = wanted & 2;
      EXPECT(expert_ffn_backward(at(1), at(2), at(3), at(4), at(5), f(6), q.T, q.H, q.F, q.dt, dx, weights ? at(9) : nullptr,
                                 weights ? at(10) : nullptr, weights ? at(11) : nullptr, at(7), room, nullptr) == MOEP_OK);
      n = check(what);
      // workgroups: N^2 rows by 256 columns of what is transposed; along the tokens the rows are padded
      const int64_t rows = q.dt == MOEP_BF16 ? 64 : 16;
      const int64_t fixed = up(q.H, rows) * up(q.F, 256) + (dx ? 2 * up(q.F, rows) * up(q.H, 256) : 0);
      const int64_t tokens = (n["transpose_kernel"] - fixed) / (weights ? 2 : 1);
      EXPECT(weights ? (n["transpose_kernel"] - fixed) % 2 == 0 && tokens % up(q.H, 256) == 0 : n["transpose_kernel"] == fixed);
      if (weights) EXPECT(tokens / up(q.H, 256) >= up(q.T, rows));
      const int64_t row_blocks = weights ? tokens / up(q.H, 256) : up(q.T, rows);
      EXPECT(n["branch_gradients_kernel"] == row_blocks * up(q.F, 256) || n["branch_gradients_kernel"] == row_blocks * up(q.F, 64));
    }
  }
  {
    const char* what = "fp32 rows beyond a grid of 64-row tiles";
    EXPECT(expert_ffn_forward_workspace((int64_t)1 << 30, 4, 4, MOEP_F32, 1) == 0 && expert_ffn_backward_workspace((int64_t)1 << 30, 4, 4, MOEP_F32) == 0);
    EXPECT(expert_ffn_forward(at(1), at(2), at(3), at(4), (int64_t)1 << 30, 4, 4, MOEP_F32, at(5), f(6), at(7), room, nullptr) == MOEP_EUNSUPPORTED);
    EXPECT(expert_ffn_backward(at(1), at(2), at(3), at(4), at(5), f(6), (int64_t)1 << 30, 4, 4, MOEP_F32, at(8), at(9), at(10), at(11), at(7), room, nullptr) == MOEP_EUNSUPPORTED);
    EXPECT(launches.empty());
  }

  // ---- logits: rows of every workgroup size, as many as there can be
  for (moep_dtype dt : {MOEP_F32, MOEP_BF16})
    for (int64_t T : {(int64_t)1, ((int64_t)1 << 22) - 1, (int64_t)1 << 22, ((int64_t)1 << 22) + 1001, (int64_t)1 << 30})
      for (int64_t V : {3, 4096, 8000, 50000, 131072, 1000000}) {
        char what[96];
        std::snprintf(what, sizeof what, "%" PRId64 " rows of %" PRId64 " logits, dtype %d", T, V, (int)dt);
        EXPECT(moe_token_logprobs(at(1), V, (int64_t*)at(2), T, V, dt, 2, f(3), f(4), f(5), (int32_t*)at(6), nullptr) == MOEP_OK);
        EXPECT(check(what)["token_logprobs_kernel"] == T);
        EXPECT(moe_distill_topk(at(1), V, (int32_t*)at(2), f(3), T, V, 4, dt, 1.f, nullptr, f(4), f(5), at(6), V, nullptr) == MOEP_OK);
        EXPECT(check(what)["distill_topk_kernel"] == T);
        EXPECT(moe_distill_topk_backward(at(1), V, (int32_t*)at(2), f(3), f(4), f(5), T, V, 4, dt, 1.f, at(6), V, nullptr) == MOEP_OK);
        EXPECT(check(what)["distill_topk_kernel"] == T);
      }
  if (!failures) std::printf("all checks passed\n");
  return failures != 0;
}
