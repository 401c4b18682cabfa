// Host-only checks of inner_step.cpp (built and run by tests/test_inner_plans.py): the kernel launchers are stand-ins that
// record what would be launched, device memory is host memory, the current device is whatever a check makes it.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "inner_internal.h"

static int current_device = 0;
extern "C" hipError_t hipGetDevice(int* device) { *device = current_device; return hipSuccess; }
extern "C" hipError_t hipMalloc(void** ptr, size_t size) {
  *ptr = std::malloc(size < (64u << 20) ? size : (64u << 20));      // what lies behind the tables only kernels touch
  return hipSuccess;
}
extern "C" hipError_t hipFree(void* ptr) { std::free(ptr); return hipSuccess; }
extern "C" hipError_t hipMemcpy(void* dst, const void* src, size_t size, hipMemcpyKind) { std::memcpy(dst, src, size); return hipSuccess; }

namespace noloco {
static int launched = 0;
static bool say = false;          // print what is launched: the last step's products, tile by tile, and small matrices
static void told(int tile, const NsArgs& args) {
  uint32_t last = 0;
  for (int i = 0; say && i < kNsClasses && args.table->end[i] != 0xffffffffu; ++i) {
    const NsClass& c = args.table->cls[i];
    std::printf("%d %u %u %u %u\n", tile, c.tall ? c.n : c.m, c.tall ? c.m : c.n, (args.table->end[i] - last) / c.per_item, c.splits);
    last = args.table->end[i];
  }
}
int launch_ns_sums(const NsArgs&, const NsArrays&, uint32_t, void*) { ++launched; return 0; }
int launch_ns_start(const NsArgs&, const NsArrays&, int, uint32_t, void*) { ++launched; return 0; }
int launch_ns_product(const NsArgs& args, const NsArrays&, int kind, int tile, int, int, float, float, float, uint32_t, void*) {
  ++launched;
  if (kind == kNsLast) told(tile, args);
  return 0;
}
int launch_ns_small(const NsArgs& args, const NsArrays&, const NsSteps&, int, uint32_t, uint32_t, void*) {
  ++launched;
  told(0, args);
  return 0;
}
int launch_embed_lookup(const EmbedArgs&, void*) { ++launched; return 0; }
int launch_embed_gradient(const EmbedArgs&, void*) { ++launched; return 0; }
}  // namespace noloco

#define CHECK(cond) do { if (!(cond)) { std::printf("CHECK failed at line %d: %s\n", __LINE__, #cond); return 1; } } while (0)

using namespace noloco;

static const float kSteps[6] = {1.5f, -.5f, 0.f, 1.5f, -.5f, 0.f};
static char* memory(size_t at) {
  static char here[1 << 16] __attribute__((aligned(256)));
  return here + at;
}

// A call on another GPU than its plan's would use that GPU's memory there.
static int check_devices() {
  const noloco_matrix matrix = {0, 4, 4, 4, 1.f};
  const noloco_newton_schulz method = {2, kSteps, 0.f, NOLOCO_PRODUCTS_AUTO};
  const noloco_muon_hparams hparams = {.1f, .9f, 0.f, 1};
  noloco_muon_plan *plan = nullptr, *none = nullptr;
  noloco_embedding_plan* table = nullptr;
  current_device = 1;
  CHECK(noloco_muon_plan_create(&matrix, 1, 64, 1, 0, &plan) == NOLOCO_OK);
  CHECK(noloco_muon_plan_create(nullptr, 0, 64, 1, 0, &none) == NOLOCO_OK);
  CHECK(noloco_embedding_plan_create(0, 4, 4, 64, 1, 8, &table) == NOLOCO_OK);
  char *a = memory(0), *b = memory(4096), *c = memory(8192);
  float* const momentum = reinterpret_cast<float*>(c);
  for (int device : {1, 0, 1}) {
    current_device = device;
    launched = 0;
    const noloco_status want = device == 1 ? NOLOCO_OK : NOLOCO_ERR_INVALID_ARG;
    CHECK(noloco_orthogonalize(plan, a, NOLOCO_F32, b, NOLOCO_F32, &method, nullptr) == want);
    CHECK(noloco_muon_step(plan, a, NOLOCO_F32, b, NOLOCO_F32, momentum, &hparams, &method, nullptr) == want);
    CHECK(noloco_embed_lookup(table, a, NOLOCO_F32, b, NOLOCO_I32, 8, 1.f, c, NOLOCO_F32, nullptr) == want);
    CHECK(noloco_embed_gradient(table, a, NOLOCO_F32, b, NOLOCO_I32, 8, 1.f, c, NOLOCO_F32, 0, nullptr) == want);
    CHECK((launched > 0) == (device == 1));
    // what launches nothing does not ask for the device
    CHECK(noloco_orthogonalize(none, a, NOLOCO_F32, b, NOLOCO_F32, &method, nullptr) == NOLOCO_OK);
    CHECK(noloco_embed_lookup(table, a, NOLOCO_F32, nullptr, NOLOCO_I32, 0, 1.f, nullptr, NOLOCO_F32, nullptr) == NOLOCO_OK);
  }
  CHECK(noloco_muon_plan_destroy(plan) == NOLOCO_OK && noloco_muon_plan_destroy(none) == NOLOCO_OK);
  CHECK(noloco_embedding_plan_destroy(table) == NOLOCO_OK);
  return 0;
}

// Every number of tokens that a plan takes is a grid that HIP takes: less than 2^32 threads and at most 65536 workgroups in a
// dimension.
static int check_lookup_grid() {
  for (int bit = 0; bit < 31; ++bit)
    for (int64_t all : {(1ll << bit) - 1, 1ll << bit, (1ll << bit) + 1, (1ll << bit) + 12345, (2ll << bit) - 1}) {
      if (all < 1 || all > 0x7fffffff) continue;
      const LookupGrid grid = lookup_grid(all);
      const uint64_t tokens = uint64_t(grid.x) * grid.y * kLookupTokens;
      CHECK(uint64_t(grid.x) * 256 < 1ull << 32 && grid.x >= 1 && grid.y >= 1 && grid.y <= 65536);
      CHECK(tokens >= uint64_t(all) && tokens - all < grid.y * uint64_t(kLookupTokens));
      CHECK(all > 1 << 27 || grid.y == 1);
    }
  return 0;
}

// Arrays of nothing share no memory, wherever they begin.
static int check_empty_arrays() {
  noloco_embedding_plan* table = nullptr;
  CHECK(noloco_embedding_plan_create(0, 4, 4, 64, 1, 8, &table) == NOLOCO_OK);
  char* const a = memory(0);
  CHECK(noloco_embed_lookup(table, a, NOLOCO_F32, a + 32, NOLOCO_I32, 0, 1.f, a + 64, NOLOCO_F32, nullptr) == NOLOCO_OK);
  CHECK(noloco_embed_gradient(table, a + 64, NOLOCO_F32, a + 64, NOLOCO_I32, 0, 1.f, a, NOLOCO_F32, 1, nullptr) == NOLOCO_OK);
  launched = 0;
  CHECK(noloco_embed_gradient(table, a + 64, NOLOCO_F32, a + 64, NOLOCO_I32, 0, 1.f, a, NOLOCO_F32, 0, nullptr) == NOLOCO_OK && launched == 1);
  CHECK(noloco_embed_lookup(table, a, NOLOCO_F32, a + 32, NOLOCO_I32, 1, 1.f, memory(4096), NOLOCO_F32, nullptr) == NOLOCO_ERR_INVALID_ARG);
  CHECK(noloco_embed_lookup(table, a, NOLOCO_F32, memory(4096), NOLOCO_I32, 1, 1.f, a + 64, NOLOCO_F32, nullptr) == NOLOCO_ERR_INVALID_ARG);
  CHECK(noloco_embedding_plan_destroy(table) == NOLOCO_OK);
  return 0;
}

// Reads W, the products to take and matrices (offset, rows, cols, row_stride) from standard input, and prints for every shape of
// matrices the tile they are planned for (0: in one workgroup), their rows and columns, how many there are, and
// the parts of X X^T; then how many launches an orthogonalisation of two steps takes.
static int print_plan() {
  int W = 0, products = 0, count = 0;
  CHECK(std::scanf("%d %d %d", &W, &products, &count) == 3);
  std::vector<noloco_matrix> matrices(count);
  int64_t end = 0;
  for (noloco_matrix& m : matrices) {
    long long v[4];
    CHECK(std::scanf("%lld %lld %lld %lld", v, v + 1, v + 2, v + 3) == 4);
    m = {v[0], v[1], v[2], v[3], 1.f};
    end = std::max<int64_t>(end, v[0] + (v[1] - 1) * v[3] + v[2]);
  }
  const int64_t stride = (end + 63) / 64 * 64;
  noloco_muon_plan* plan = nullptr;
  CHECK(noloco_muon_plan_create(matrices.data(), count, stride, W, 0, &plan) == NOLOCO_OK);
  const noloco_newton_schulz method = {2, kSteps, 0.f, products};
  char* const x = memory(0);
  char* const y = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(x) + uint64_t(W) * stride * 8 + 4096) / 256 * 256);
  say = true;
  launched = 0;
  CHECK(noloco_orthogonalize(plan, x, NOLOCO_F32, y, NOLOCO_BF16, &method, nullptr) == NOLOCO_OK);
  std::printf("launches %d\n", launched);
  CHECK(noloco_muon_plan_destroy(plan) == NOLOCO_OK);
  return 0;
}

int main(int argc, char** argv) {
  const char* const what = argc > 1 ? argv[1] : "";
  int failed = 1;
  if (std::strcmp(what, "devices") == 0) failed = check_devices();
  else if (std::strcmp(what, "lookup_grid") == 0) failed = check_lookup_grid();
  else if (std::strcmp(what, "empty_arrays") == 0) failed = check_empty_arrays();
  else if (std::strcmp(what, "plan") == 0) failed = print_plan();
  else std::printf("what to check?\n");
  if (failed == 0) std::printf("ok\n");
  return failed;
}
