// Host-only exercise of inner_step.cpp under AddressSanitizer and UBSan (built and run by tests/test_inner_host.py): the
// kernel launchers are stand-ins that record what would be launched, device memory is host memory.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#include "inner_internal.h"

static int mallocs = 0, frees = 0, fail_malloc = 0;
static size_t allocated = 0;
extern "C" hipError_t hipGetDevice(int* device) { *device = 0; return hipSuccess; }
extern "C" hipError_t hipMalloc(void** ptr, size_t size) {
  if (fail_malloc) return hipErrorOutOfMemory;
  ++mallocs;
  allocated = size;
  // The tables at its start are read and written; the workspace behind them only by kernels.
  *ptr = std::malloc(size < (64u << 20) ? size : (64u << 20));
  return hipSuccess;
}
extern "C" hipError_t hipFree(void* ptr) { ++frees; std::free(ptr); return hipSuccess; }
extern "C" hipError_t hipMemcpy(void* dst, const void* src, size_t size, hipMemcpyKind) { std::memcpy(dst, src, size); return hipSuccess; }

namespace noloco {
struct Launch { int what, kind, tile, planes, step; uint32_t groups; NsArgs args; uint32_t lds; };
static std::vector<Launch> launches;
static int fail_at = -1;
static int record(const Launch& l) {
  if (static_cast<int>(launches.size()) == fail_at) return 1;
  launches.push_back(l);
  return 0;
}
int launch_ns_sums(const NsArgs& args, const NsArrays&, uint32_t groups, void*) { return record({0, 0, 0, 0, 0, groups, args, 0}); }
int launch_ns_start(const NsArgs& args, const NsArrays&, int planes, uint32_t groups, void*) { return record({1, 0, 0, planes, 0, groups, args, 0}); }
int launch_ns_product(const NsArgs& args, const NsArrays&, int kind, int tile, int planes, int step, float, float, float, uint32_t groups, void*) {
  return record({2, kind, tile, planes, step, groups, args, 0});
}
int launch_ns_small(const NsArgs& args, const NsArrays&, const NsSteps& steps, int planes, uint32_t groups, uint32_t lds, void*) {
  return record({3, 0, 0, planes, steps.count, groups, args, lds});
}
static int lookups = 0, gradients = 0;
int launch_embed_lookup(const EmbedArgs&, void*) { ++lookups; return 0; }
int launch_embed_gradient(const EmbedArgs&, void*) { ++gradients; return 0; }
}  // namespace noloco

#define CHECK(cond) do { if (!(cond)) { std::printf("CHECK failed at line %d: %s\n", __LINE__, #cond); return 1; } } while (0)

using namespace noloco;

// Every launch covers each of its items' parts once, items lie apart in the workspace, and all items of all matrices
// come up in exactly one batch.
static int check_plan(const std::vector<noloco_matrix>& matrices, int64_t stride, int32_t W, int64_t room, int32_t out_dtype) {
  noloco_muon_plan* plan = nullptr;
  CHECK(noloco_muon_plan_create(matrices.data(), static_cast<int32_t>(matrices.size()), stride, W, room, &plan) == NOLOCO_OK);
  int64_t elements, bytes;
  int32_t batches[2];
  CHECK(noloco_muon_plan_info(plan, &elements, &bytes, &batches[0], &batches[1]) == NOLOCO_OK);
  CHECK(bytes >= 0 && static_cast<size_t>(bytes) <= allocated);
  launches.clear();
  const float k[6] = {1.5f, -.5f, 0.f, 1.5f, -.5f, 0.f};
  const noloco_newton_schulz method = {2, k, 0.f, out_dtype == NOLOCO_BF16 ? NOLOCO_PRODUCTS_F16 : NOLOCO_PRODUCTS_PAIRS};
  static char here[256] __attribute__((aligned(256)));
  char* const x = here;
  char* const y = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(here) + uintptr_t(W) * stride * 8 + 4096) / 256 * 256);
  CHECK(noloco_orthogonalize(plan, x, NOLOCO_F32, y, out_dtype, &method, nullptr) == NOLOCO_OK);
  const int planes = out_dtype == NOLOCO_BF16 ? 1 : 2;
  std::map<int64_t, int> seen;
  size_t in_batch = 0, batch = 0;
  for (size_t l = 0; l < launches.size(); ++l) {
    const Launch& launch = launches[l];
    if (launch.what == 3) {
      CHECK(in_batch == 0 && launch.planes == planes && launch.step == 2 && launch.lds <= kNsSmallLds);
      ++batch;
    } else {
      CHECK(launch.what == (in_batch == 0 ? 0 : (in_batch == 1 ? 1 : 2)));
    }
    if (launch.what == 2) {
      const int kinds[6] = {kNsGram, kNsSquare, kNsApply, kNsGram, kNsSquare, kNsLast};
      CHECK(launch.kind == kinds[in_batch - 2] && launch.planes == planes && launch.step == static_cast<int>(in_batch - 2) / 3);
    }
    if (launch.what != 3 && ++in_batch == 8) { in_batch = 0; ++batch; }
    CHECK(launch.groups > 0 && launch.groups <= (1u << 22) + (1u << 21));
    CHECK(launch.args.first_end == launch.args.table->end[0] && std::memcmp(&launch.args.first, &launch.args.table->cls[0], sizeof(NsClass)) == 0);
    uint32_t last = 0;
    uint64_t end_of_last = 0;
    for (int i = 0; i < kNsClasses && launch.args.table->end[i] != 0xffffffffu; ++i) {
      const NsClass& c = launch.args.table->cls[i];
      const uint32_t groups = launch.args.table->end[i] - last;
      CHECK(groups > 0 && groups % c.per_item == 0);
      const uint32_t items = groups / c.per_item;
      last = launch.args.table->end[i];
      CHECK(c.m <= c.n && c.mp >= c.m && c.np >= c.n && c.mp % 64 == 0 && c.np % 64 == 0);
      CHECK(ns_x_bytes(c.mp, c.np, planes) >> 32 == 0);
      if (launch.what == 3) {
        CHECK(c.per_item == 1 && c.m <= 128 && ns_small_bytes(c.m, c.n, planes) <= launch.lds);
      } else {
        CHECK(c.item_bytes == ns_item_bytes(c.mp, c.np, planes) && c.base >= end_of_last);
        end_of_last = c.base + c.item_bytes * items;
        CHECK(end_of_last <= static_cast<uint64_t>(bytes));
      }
      if (launch.what == 2) {
        const uint32_t mt = c.mp / launch.tile, nt = c.np / launch.tile;
        CHECK(c.mp % launch.tile == 0 && c.np % launch.tile == 0);
        CHECK(c.per_item == (launch.kind >= kNsApply ? mt * nt : mt * (mt + 1) / 2));
        CHECK(c.splits >= 1 && c.splits <= launch.args.splits && c.splits * uint64_t(64 / planes) <= c.n + 64 / planes);
        CHECK(c.splits == 1 || (launch.tile == kNsSplitTile && c.splits * (uint64_t(mt) * (mt + 1) / 2) * kNsSplitBytes <= ns_x_bytes(c.mp, c.np, planes)));
      }
      if (launch.what == 1) CHECK(c.per_item == c.mp / 64 * (c.np / 64));
      if (launch.what == 0 || launch.what == 3) {
        CHECK(c.per_item >= 1 && c.per_item <= kNsChunks);
        for (uint32_t j = 0; j < items; ++j) {
          const NsItem& item = launch.args.items[c.first_item + j];
          if (launch.what == 0) CHECK(reinterpret_cast<const char*>(launch.args.sums + uint64_t(c.first_sum + j + 1) * kNsChunks) <= launch.args.workspace);
          ++seen[item.offset];
        }
      }
    }
    CHECK(last == launch.groups);
  }
  CHECK(in_batch == 0 && batch == static_cast<size_t>(batches[planes - 1]));
  size_t wanted = 0;
  for (const noloco_matrix& m : matrices)
    if (m.rows > 0 && m.cols > 0)
      for (int32_t w = 0; w < W; ++w, ++wanted) CHECK(seen[w * stride + m.offset] == 1);
  CHECK(seen.size() == wanted);
  // products by the result's type, pairs where small matrices are all there is
  if (!launches.empty()) {
    bool small = true;
    for (const noloco_matrix& m : matrices) {
      const int64_t lo = std::min(m.rows, m.cols), hi = std::max(m.rows, m.cols);
      auto fits = [&](int planes) { return lo <= 128 && lo * ((hi + 7) / 8 * 8) <= static_cast<int64_t>(ns_small_numbers(planes)) && ns_small_bytes(lo, hi, planes) <= kNsSmallLds; };
      small = small && (fits(2) || (lo <= 64 && !fits(1)));
    }
    const noloco_newton_schulz by_type = {2, k, 0.f, NOLOCO_PRODUCTS_AUTO};
    launches.clear();
    CHECK(noloco_orthogonalize(plan, x, NOLOCO_F32, y, out_dtype, &by_type, nullptr) == NOLOCO_OK);
    for (const Launch& launch : launches)
      if (launch.what >= 2) CHECK(launch.planes == (out_dtype == NOLOCO_BF16 && !small ? 1 : 2));
  }
  // a launch that the runtime refuses ends the call
  if (!launches.empty()) {
    launches.clear();
    fail_at = 0;
    CHECK(noloco_orthogonalize(plan, x, NOLOCO_F32, y, out_dtype, &method, nullptr) == NOLOCO_ERR_DEVICE);
    CHECK(launches.empty());
    fail_at = -1;
  }
  CHECK(noloco_muon_plan_destroy(plan) == NOLOCO_OK);
  return 0;
}

static noloco_status method_status(const std::vector<float>& k, int32_t steps) {
  noloco_matrix m = {0, 4, 4, 4, 1.f};
  noloco_muon_plan* plan = nullptr;
  if (noloco_muon_plan_create(&m, 1, 64, 1, 0, &plan) != NOLOCO_OK) return NOLOCO_ERR_DEVICE;
  static char x[512] __attribute__((aligned(256)));
  const noloco_newton_schulz method = {steps, k.data(), 0.f, NOLOCO_PRODUCTS_AUTO};
  const noloco_status st = noloco_orthogonalize(plan, x, NOLOCO_F32, x, NOLOCO_F32, &method, nullptr);
  noloco_muon_plan_destroy(plan);
  return st;
}

int main() {
  std::mt19937 rng(1);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  for (int round = 0; round < 60; ++round) {
    std::vector<noloco_matrix> matrices;
    int64_t at = pick(0, 9);
    const int count = pick(0, 80), most = round % 3 == 0 ? 1200 : 200;
    for (int i = 0; i < count; ++i) {
      noloco_matrix m = {at, pick(0, most), pick(1, most), 0, 1.f};
      if (i > 0 && pick(0, 2) == 0) { m.rows = matrices.back().rows; m.cols = matrices.back().cols; }
      m.row_stride = m.cols + (pick(0, 1) ? pick(0, 5) : 0);
      at += m.rows * m.row_stride + pick(0, 7);
      matrices.push_back(m);
    }
    const int64_t stride = (at + 64) / 64 * 64;
    const int64_t rooms[3] = {0, 1, 40 << 20};
    if (check_plan(matrices, stride, pick(1, 5), rooms[round % 3], round % 2 ? NOLOCO_F32 : NOLOCO_BF16)) return 1;
  }
  // the largest shapes, and tall and wide ones
  if (check_plan({{0, 16384, 16384, 16384, 1.f}}, 1ll << 28, 1, 0, NOLOCO_F32)) return 1;
  if (check_plan({{0, 1, 1 << 22, 1 << 22, 1.f}, {1 << 22, 1 << 22, 1, 1, 1.f}}, 1ll << 23, 2, 0, NOLOCO_F32)) return 1;
  if (check_plan({{0, 64, 1 << 22, 1 << 22, 1.f}}, 1ll << 28, 1, 0, NOLOCO_F32)) return 1;

  // columns of one tensor side by side are no overlap; matrices inside each other's gaps neither
  noloco_muon_plan* plan = nullptr;
  const noloco_matrix side[3] = {{0, 10, 5, 15, 1.f}, {5, 10, 5, 15, 1.f}, {10, 10, 5, 15, 1.f}};
  CHECK(noloco_muon_plan_create(side, 3, 192, 2, 0, &plan) == NOLOCO_OK);
  CHECK(noloco_muon_plan_destroy(plan) == NOLOCO_OK);
  const noloco_matrix crossed[2] = {{0, 10, 5, 15, 1.f}, {5, 3, 11, 45, 1.f}};
  CHECK(noloco_muon_plan_create(crossed, 2, 192, 2, 0, &plan) == NOLOCO_ERR_SEGMENT_OVERLAP && plan == nullptr);
  fail_malloc = 1;
  CHECK(noloco_muon_plan_create(side, 3, 192, 2, 0, &plan) == NOLOCO_ERR_DEVICE && plan == nullptr);
  noloco_embedding_plan* table = nullptr;
  CHECK(noloco_embedding_plan_create(0, 10, 4, 64, 2, 100, &table) == NOLOCO_ERR_DEVICE && table == nullptr);
  fail_malloc = 0;

  // which coefficients binary16 has room for
  CHECK(method_status({3.4445f, -4.7750f, 2.0315f}, 1) == NOLOCO_OK);
  std::vector<float> five;
  for (int i = 0; i < 5; ++i) five.insert(five.end(), {3.4445f, -4.7750f, 2.0315f});
  CHECK(method_status(five, 5) == NOLOCO_OK);
  CHECK(method_status({8.2872f, -23.5959f, 17.3004f}, 1) == NOLOCO_OK);
  CHECK(method_status({15.6f, 0.f, 0.f}, 1) == NOLOCO_ERR_UNSUPPORTED);
  CHECK(method_status({2.7f, 0.f, 0.f}, 1) == NOLOCO_OK);
  CHECK(method_status({2.8f, 0.f, 0.f}, 1) == NOLOCO_ERR_UNSUPPORTED);          // the result leaves the range
  CHECK(method_status({0.f, 0.f, 0.f}, 1) == NOLOCO_OK);
  CHECK(method_status({0.f, -80.f, 80.f}, 1) == NOLOCO_ERR_UNSUPPORTED);        // P leaves its range between the ends
  CHECK(method_status({NAN, 0.f, 0.f}, 1) == NOLOCO_ERR_INVALID_ARG);
  CHECK(method_status({1.f, INFINITY, 0.f}, 1) == NOLOCO_ERR_INVALID_ARG);
  CHECK(method_status({1.f, 0.f, 0.f}, 0) == NOLOCO_ERR_INVALID_ARG);

  // embedding: sizes of the scratch, and calls that launch nothing
  CHECK(noloco_embedding_plan_create(3, 10, 4, 64, 2, 100, &table) == NOLOCO_OK);
  CHECK(allocated >= 2 * 2 * 100 * 8 + 2 * 4 * 2 * 4 * 4);
  static char buffer[4096] __attribute__((aligned(256)));
  CHECK(noloco_embed_lookup(table, buffer, NOLOCO_F32, nullptr, NOLOCO_I32, 0, 1.f, nullptr, NOLOCO_F32, nullptr) == NOLOCO_OK && lookups == 0);
  CHECK(noloco_embed_gradient(table, nullptr, NOLOCO_F32, nullptr, NOLOCO_I32, 0, 1.f, buffer, NOLOCO_F32, 1, nullptr) == NOLOCO_OK && gradients == 0);
  CHECK(noloco_embed_gradient(table, nullptr, NOLOCO_F32, nullptr, NOLOCO_I32, 0, 1.f, buffer, NOLOCO_F32, 0, nullptr) == NOLOCO_OK && gradients == 1);
  CHECK(noloco_embed_lookup(table, buffer, NOLOCO_F32, buffer + 1024, NOLOCO_I32, 4, 1.f, buffer + 2048, NOLOCO_F32, nullptr) == NOLOCO_OK && lookups == 1);
  CHECK(noloco_embedding_plan_destroy(table) == NOLOCO_OK);
  CHECK(noloco_embedding_plan_destroy(nullptr) == NOLOCO_OK && noloco_muon_plan_destroy(nullptr) == NOLOCO_OK);
  CHECK(mallocs == frees);
  std::printf("inner host driver: ok\n");
  return 0;
}
