// Host-only exercise of model_step.cpp under AddressSanitizer and UBSan (built and run by tests/test_model_host.py): the kernel
// launchers are stand-ins that check what would be launched against the plan's workspace; no memory is read through.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <limits>
#include <random>
#include <vector>

#include "model_internal.h"

static int device = 0, mallocs = 0, frees = 0, fail_malloc = 0;
static uint64_t room_at = 0, room = 0;
extern "C" hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
extern "C" hipError_t hipMalloc(void** ptr, size_t size) {
  if (fail_malloc) return hipErrorOutOfMemory;
  ++mallocs;
  *ptr = std::malloc(1);
  room_at = reinterpret_cast<uint64_t>(*ptr);
  room = size;
  return hipSuccess;
}
extern "C" hipError_t hipFree(void* ptr) { ++frees; std::free(ptr); return hipSuccess; }

static int bad = 0, launches = 0, fail_launch = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("EXPECT failed at line %d: %s\n", __LINE__, #cond); ++bad; } } while (0)
static bool inside(const void* p, uint64_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  return at >= room_at && at - room_at <= room && bytes <= room - (at - room_at);
}

namespace noloco {
static std::vector<ProductArgs> products;
static std::vector<SlopeArgs> slopes;
static std::vector<LogProbArgs> log_probs;
static int launch() { ++launches; return fail_launch; }
int launch_layer_norm(const NormArgs& a, void*) {
  EXPECT(a.groups >= 1 && a.tokens > 0 && a.weight >= 0);
  return launch();
}
int launch_layer_norm_gradient(const NormArgs& a, void*) {
  EXPECT(a.groups >= 1 && inside(a.partial, uint64_t(a.W) * a.groups * 2 * a.width * 4));
  return launch();
}
int launch_product(const ProductArgs& a, const ProductPlan& p, char* at, void*) {
  products.push_back(a);
  EXPECT(inside(at, p.bytes));
  EXPECT(p.splits >= 1 && p.splits <= 32 && (p.tile == 0 || p.tile == 32 || p.tile == 128 || p.tile == 256));
  const uint64_t sizes[2] = {a.m, a.n};
  uint64_t end = 0;
  for (int i = 0; i < 2; ++i) {
    const Operand& o = i == 0 ? a.a : a.b;
    if (p.tile == 0) continue;
    const uint64_t rows = o.along_k ? sizes[i] : a.k, wide = ((o.along_k ? a.k : sizes[i]) + 7) / 8 * 8;
    EXPECT(p.packed[i] || (o.bf16 && o.ld % 8 == 0 && o.worker_stride % 8 == 0 && reinterpret_cast<uint64_t>(o.p) % 16 == 0 && (!o.along_k || a.k % 8 == 0)));
    EXPECT(!p.packed[i] || p.packed_at[i] >= end);
    if (p.packed[i]) end = p.packed_at[i] + uint64_t(a.W) * rows * wide * 2 * p.parts[i];
  }
  if (p.f16) {
    EXPECT(p.largest_at >= end && p.exponents_at >= p.largest_at + uint64_t(a.W) * 2 * kPackParts * 4);
    end = p.exponents_at + uint64_t(a.W) * 8;
  }
  if (p.splits > 1) {
    EXPECT(p.parts_at >= end && p.splits <= (uint64_t(a.k) + 63) / 64 * (p.parts[0] + p.parts[1] - 1));
    end = p.parts_at + p.splits * uint64_t(a.W) * a.m * ((a.n + 7) / 8 * 8) * 4;
  }
  EXPECT(end <= p.bytes);
  return launch();
}
int launch_slope(const SlopeArgs& a, void*) {
  slopes.push_back(a);
  const uint64_t numbers = uint64_t(a.W) * a.tokens * a.outputs * (a.dz_bf16 ? 2 : 4), sums = uint64_t(a.W) * a.groups * a.outputs * 4;
  EXPECT(a.dz == nullptr || inside(a.dz, numbers));
  EXPECT(a.partial == nullptr || inside(a.partial, sums));
  if (a.dz != nullptr && a.partial != nullptr) EXPECT(static_cast<char*>(a.dz) + numbers <= reinterpret_cast<char*>(a.partial));
  return launch();
}
int launch_log_probs(const LogProbArgs& a, void*) {
  log_probs.push_back(a);
  EXPECT(a.part >= 1 && a.part <= kLogChunk && uint64_t(a.num_parts) * a.part >= a.vocab && uint64_t(a.num_parts - 1) * a.part < a.vocab);
  if (a.num_parts > 1) {
    const uint64_t parts = uint64_t(a.rows) * a.num_parts;
    EXPECT(inside(a.parts, parts * sizeof(LogPart)) && inside(a.keys, parts * a.top * 8));
    EXPECT(reinterpret_cast<char*>(a.parts) + parts * sizeof(LogPart) <= reinterpret_cast<char*>(a.keys));
  }
  return launch();
}
int launch_log_probs_gradient(const LogProbArgs&, void*) { return launch(); }
}  // namespace noloco

#define CHECK(cond) do { if (!(cond) || bad) { std::printf("CHECK failed at line %d: %s\n", __LINE__, #cond); return 1; } } while (0)

using namespace noloco;

static char* at(uint64_t v) { return reinterpret_cast<char*>(v << 43); }     // arrays far from each other

static int norms() {
  const noloco_norm given[] = {{0, 1000, 1000}, {2000, -1, 17}, {3000, 30000, 20000}};
  noloco_layer_norm_plan* plan = nullptr;
  std::mt19937 gen(1);
  for (int32_t W : {1, 3, 700, 5000}) {
    CHECK(noloco_layer_norm_plan_create(given, 3, 50048, W, 5000, &plan) == NOLOCO_OK);
    float* const stats = reinterpret_cast<float*>(at(4));
    for (int k = 0; k < 60; ++k) {
      const int32_t norm = k % 3;
      const int64_t T = k < 3 ? 5000 : 1 + gen() % 5000;
      CHECK(noloco_layer_norm(plan, norm, at(1), 0, at(2), 1, T, 1e-5f, at(3), 0, stats, nullptr) == NOLOCO_OK);
      CHECK(noloco_layer_norm_gradient(plan, norm, at(5), 1, at(1), 0, at(2), 1, stats, T, nullptr, at(3), 0, at(6), 0, k & 1, nullptr) == NOLOCO_OK);
    }
    // what is refused
    auto forward = [&](int32_t norm, void* x, void* theta, int64_t T, float eps, void* out, float* s, int32_t t1 = 0) {
      return noloco_layer_norm(plan, norm, x, t1, theta, 0, T, eps, out, 0, s, nullptr);
    };
    const int before = launches;
    CHECK(forward(3, at(1), at(2), 1, 0.f, at(3), nullptr) == NOLOCO_ERR_INVALID_ARG && forward(-1, at(1), at(2), 1, 0.f, at(3), nullptr) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1), at(2), 5001, 0.f, at(3), nullptr) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1), at(2), -1, 0.f, at(3), nullptr) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, nullptr, at(2), 1, 0.f, at(3), nullptr) == NOLOCO_ERR_NULL && forward(0, at(1), nullptr, 1, 0.f, at(3), nullptr) == NOLOCO_ERR_NULL);
    CHECK(forward(0, at(1), at(2), 1, 0.f, nullptr, nullptr) == NOLOCO_ERR_NULL && forward(0, at(1), at(2), 1, -1.f, at(3), nullptr) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1), at(2), 1, std::numeric_limits<float>::quiet_NaN(), at(3), nullptr) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1) + 8, at(2), 1, 0.f, at(3), nullptr) == NOLOCO_ERR_ALIGNMENT && forward(0, at(1), at(2) + 128, 1, 0.f, at(3), nullptr) == NOLOCO_ERR_ALIGNMENT);
    CHECK(forward(0, at(1), at(2), 1, 0.f, at(1), nullptr) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1), at(2), 1, 0.f, at(2), nullptr) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1), at(2), 1, 0.f, at(3), reinterpret_cast<float*>(at(3))) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1), at(2), 1, 0.f, at(3), nullptr, 2) == NOLOCO_ERR_INVALID_ARG);
    auto back = [&](void* dout, void* x, const float* s, void* add, void* dx, void* grad, int32_t acc) {
      return noloco_layer_norm_gradient(plan, 0, dout, 0, x, 0, at(2), 0, s, 2, add, dx, 0, grad, 0, acc, nullptr);
    };
    CHECK(back(nullptr, at(1), stats, nullptr, at(3), at(6), 0) == NOLOCO_ERR_NULL && back(at(5), nullptr, stats, nullptr, at(3), at(6), 0) == NOLOCO_ERR_NULL);
    CHECK(back(at(5), at(1), nullptr, nullptr, at(3), at(6), 0) == NOLOCO_ERR_NULL && back(at(5), at(1), stats, nullptr, nullptr, at(6), 0) == NOLOCO_ERR_NULL);
    CHECK(back(at(5), at(1), stats, nullptr, at(3), at(6), 2) == NOLOCO_ERR_INVALID_ARG && back(at(5), at(1), stats, nullptr, at(5), at(6), 0) == NOLOCO_ERR_INVALID_ARG);
    CHECK(back(at(5), at(1), stats, nullptr, at(3), at(2), 0) == NOLOCO_ERR_INVALID_ARG && back(at(5), at(1), stats, at(3) + 16, at(3), at(6), 0) == NOLOCO_ERR_INVALID_ARG);
    CHECK(back(at(5), at(1), stats, at(6), at(3), at(6), 0) == NOLOCO_ERR_INVALID_ARG && back(at(5), at(1), stats, nullptr, at(3), at(6) + 64, 0) == NOLOCO_ERR_ALIGNMENT);
    device = 1;
    CHECK(forward(0, at(1), at(2), 1, 0.f, at(3), nullptr) == NOLOCO_ERR_INVALID_ARG && back(at(5), at(1), stats, nullptr, at(3), at(6), 0) == NOLOCO_ERR_INVALID_ARG);
    device = 0;
    CHECK(launches == before);
    CHECK(back(at(5), at(1), stats, at(3), at(3), at(6), 0) == NOLOCO_OK);
    fail_launch = 1;
    CHECK(back(at(5), at(1), stats, at(3), at(3), at(6), 0) == NOLOCO_ERR_DEVICE && forward(0, at(1), at(2), 1, 0.f, at(3), nullptr) == NOLOCO_ERR_DEVICE);
    fail_launch = 0;
    CHECK(noloco_layer_norm_plan_destroy(plan) == NOLOCO_OK);
  }
  return 0;
}

static int matrices() {
  const noloco_linear_layer given[] = {{0, 100, 200, 200, 20000, 0}, {100000, 300, 40, 301, -1, 1}, {3, 1, 1, 1, 5, 0}};
  noloco_linear_plan* plan = nullptr;
  std::mt19937 gen(2);
  for (int64_t asked : {int64_t(0), int64_t(1), int64_t(3000000)}) {
    CHECK(noloco_linear_plan_create(given, 3, 150016, 7, 3000, asked, &plan) == NOLOCO_OK);
    for (int k = 0; k < 300; ++k) {
      const int32_t layer = k % 3, act = gen() % 5, acc = gen() & 1;
      const int64_t T = k < 9 ? 3000 : gen() % 3001;
      const int32_t t[5] = {int32_t(gen() & 1), int32_t(gen() & 1), int32_t(gen() & 1), int32_t(gen() & 1), int32_t(gen() & 1)};
      const noloco_linear_layer& l = given[layer];
      products.clear();
      CHECK(noloco_linear(plan, layer, at(1), t[0], at(2), t[1], T, act, nullptr, at(7), at(3), t[2], nullptr) == NOLOCO_OK);
      int64_t of_out = 0;
      for (const ProductArgs& p : products) {
        CHECK(p.m == T && p.n == l.outputs && p.k == l.inputs && p.b.along_k == l.transposed);
        CHECK(p.out == at(3) + of_out * T * l.outputs * (t[2] ? 2 : 4) && p.before == at(7) + of_out * T * l.outputs * (t[2] ? 2 : 4));
        CHECK(p.a.p == at(1) + of_out * T * l.inputs * (t[0] ? 2 : 4) && p.b.p == at(2) + (l.offset + of_out * 150016) * (t[1] ? 2 : 4));
        CHECK(l.bias < 0 || p.bias == at(2) + (l.bias + of_out * 150016) * (t[1] ? 2 : 4));
        of_out += p.W;
      }
      CHECK(of_out == (T > 0 ? 7 : 0));
      products.clear();
      slopes.clear();
      const bool dx = gen() & 1, grad = gen() & 1;
      CHECK(noloco_linear_gradient(plan, layer, at(1), t[0], at(4), t[1], at(2), t[2], T, act, at(5), nullptr, dx ? at(3) : nullptr, t[3], grad ? at(6) : nullptr,
                                   t[4], acc, nullptr) == NOLOCO_OK);
      // every worker's products once
      int64_t of_dx = 0, of_grad = 0;
      for (const ProductArgs& p : products) {
        const bool for_grad = p.out_ld == l.row_stride && p.out_stride == 150016;
        const int64_t first = for_grad ? of_grad : of_dx;
        const char* base = for_grad ? at(6) + (l.offset + first * 150016) * (t[4] ? 2 : 4) : at(3) + first * T * l.inputs * (t[3] ? 2 : 4);
        CHECK(p.out == base);
        (for_grad ? of_grad : of_dx) += p.W;
        CHECK(act != 0 || (for_grad ? (l.transposed ? p.a.p : p.b.p) : p.a.p) == at(1) + first * T * l.outputs * (t[0] ? 2 : 4));
      }
      CHECK(of_dx == (dx && T > 0 ? 7 : 0) && of_grad == (grad && (T > 0 || !acc) ? 7 : 0));
      int64_t sloped = 0;
      for (const SlopeArgs& s : slopes) sloped += s.W;
      CHECK(sloped == ((of_dx > 0 || of_grad > 0) && (act != 0 || (grad && l.bias >= 0)) ? 7 : 0));
    }
    const int before = launches;
    auto forward = [&](int32_t layer, void* x, void* theta, int64_t T, int32_t act, void* residual, void* z, void* out, int32_t t1 = 0) {
      return noloco_linear(plan, layer, x, t1, theta, 0, T, act, residual, z, out, 0, nullptr);
    };
    CHECK(forward(3, at(1), at(2), 1, 0, nullptr, nullptr, at(3)) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1), at(2), 3001, 0, nullptr, nullptr, at(3)) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1), at(2), 1, 5, nullptr, nullptr, at(3)) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1), at(2), 1, -1, nullptr, nullptr, at(3)) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, nullptr, at(2), 1, 0, nullptr, nullptr, at(3)) == NOLOCO_ERR_NULL && forward(0, at(1), at(2), 1, 0, nullptr, nullptr, nullptr) == NOLOCO_ERR_NULL);
    CHECK(forward(0, at(1), at(2), 1, 0, nullptr, nullptr, at(3), 7) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1) + 4, at(2), 1, 0, nullptr, nullptr, at(3)) == NOLOCO_ERR_ALIGNMENT);
    CHECK(forward(0, at(1), at(2), 1, 0, at(3) + 16, nullptr, at(3)) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1), at(2), 1, 0, nullptr, at(3), at(3)) == NOLOCO_ERR_INVALID_ARG);
    CHECK(forward(0, at(1), at(2), 1, 0, at(4), at(4), at(3)) == NOLOCO_ERR_INVALID_ARG && forward(0, at(1), at(2), 1, 0, nullptr, at(2), at(3)) == NOLOCO_ERR_INVALID_ARG);
    auto back = [&](void* dout, void* x, void* z, int32_t act, void* add, void* dx, void* grad) {
      return noloco_linear_gradient(plan, 0, dout, 0, x, 0, at(2), 0, 2, act, z, add, dx, 0, grad, 0, 0, nullptr);
    };
    CHECK(back(nullptr, at(4), nullptr, 0, nullptr, at(3), at(6)) == NOLOCO_ERR_NULL && back(at(1), nullptr, nullptr, 0, nullptr, at(3), at(6)) == NOLOCO_ERR_NULL);
    CHECK(back(at(1), at(4), nullptr, 1, nullptr, at(3), at(6)) == NOLOCO_ERR_NULL && back(at(1), at(4), nullptr, 0, nullptr, at(1), at(6)) == NOLOCO_ERR_INVALID_ARG);
    CHECK(back(at(1), at(4), nullptr, 0, at(3) + 16, at(3), at(6)) == NOLOCO_ERR_INVALID_ARG && back(at(1), at(4), nullptr, 0, nullptr, at(3), at(4)) == NOLOCO_ERR_INVALID_ARG);
    CHECK(back(at(1), at(4), at(3), 1, nullptr, at(3), at(6)) == NOLOCO_ERR_INVALID_ARG && back(at(1), at(4), nullptr, 0, nullptr, at(3), at(2)) == NOLOCO_ERR_INVALID_ARG);
    device = 1;
    CHECK(forward(0, at(1), at(2), 1, 0, nullptr, nullptr, at(3)) == NOLOCO_ERR_INVALID_ARG && back(at(1), at(4), nullptr, 0, nullptr, at(3), at(6)) == NOLOCO_ERR_INVALID_ARG);
    device = 0;
    CHECK(launches == before);
    CHECK(back(at(1), nullptr, nullptr, 0, at(3), at(3), nullptr) == NOLOCO_OK && forward(0, at(1), at(2), 1, 0, at(3), nullptr, at(3)) == NOLOCO_OK);
    fail_launch = 1;
    CHECK(back(at(1), at(4), nullptr, 0, nullptr, at(3), at(6)) == NOLOCO_ERR_DEVICE && forward(0, at(1), at(2), 1, 0, nullptr, nullptr, at(3)) == NOLOCO_ERR_DEVICE);
    fail_launch = 0;
    CHECK(noloco_linear_plan_destroy(plan) == NOLOCO_OK);
  }
  return 0;
}

static int losses() {
  std::mt19937 gen(3);
  for (int64_t vocab : {1, 7, 4096, 50257, 65536, 65537, 262144, 1 << 24})
    for (int32_t W : {1, 3}) {
      const int64_t most = vocab > 300000 ? 20 : 2000;
      noloco_log_prob_plan* plan = nullptr;
      CHECK(noloco_log_prob_plan_create(vocab, vocab + 3, W, most, 32, &plan) == NOLOCO_OK);
      float* const f[6] = {reinterpret_cast<float*>(at(3)), reinterpret_cast<float*>(at(4)), reinterpret_cast<float*>(at(5)), reinterpret_cast<float*>(at(6)),
                           reinterpret_cast<float*>(at(7)), reinterpret_cast<float*>(at(8))};
      int32_t* const ids = reinterpret_cast<int32_t*>(at(9));
      for (int64_t T = 1; T <= most; T += T < 600 ? 1 : 97)
        CHECK(noloco_token_log_probs(plan, at(1), T & 1, at(2), 2 + (T & 1), T, f[0], f[1], f[2], T % 33, ids, f[3], nullptr) == NOLOCO_OK);
      CHECK(noloco_token_log_probs(plan, at(1), 0, at(2), 2, most, f[0], f[1], f[2], 32, ids, f[3], nullptr) == NOLOCO_OK);
      const int before = launches;
      auto forward = [&](void* logits, void* tokens, int64_t T, float* lp, float* h, int32_t top, int32_t* top_ids, int32_t t1 = 0, int32_t t2 = 2) {
        return noloco_token_log_probs(plan, logits, t1, tokens, t2, T, lp, h, f[2], top, top_ids, f[3], nullptr);
      };
      CHECK(forward(nullptr, at(2), 1, f[0], f[1], 0, nullptr) == NOLOCO_ERR_NULL && forward(at(1), nullptr, 1, f[0], f[1], 0, nullptr) == NOLOCO_ERR_NULL);
      CHECK(forward(at(1), at(2), 1, nullptr, f[1], 0, nullptr) == NOLOCO_ERR_NULL && forward(at(1), at(2), 1, f[0], f[1], 1, nullptr) == NOLOCO_ERR_NULL);
      CHECK(forward(at(1), at(2), most + 1, f[0], f[1], 0, nullptr) == NOLOCO_ERR_INVALID_ARG && forward(at(1), at(2), 1, f[0], f[1], 33, ids) == NOLOCO_ERR_INVALID_ARG);
      CHECK(forward(at(1), at(2), 1, f[0], f[0], 0, nullptr) == NOLOCO_ERR_INVALID_ARG && forward(at(1), at(2), 1, f[0], f[1], 1, reinterpret_cast<int32_t*>(f[3])) == NOLOCO_ERR_INVALID_ARG);
      CHECK(forward(at(1), at(2), 1, reinterpret_cast<float*>(at(1)), f[1], 0, nullptr) == NOLOCO_ERR_INVALID_ARG && forward(at(1), at(2), 1, f[0], f[1], 0, nullptr, 2) == NOLOCO_ERR_INVALID_ARG);
      CHECK(forward(at(1), at(2), 1, f[0], f[1], 0, nullptr, 0, 1) == NOLOCO_ERR_INVALID_ARG && forward(at(1) + 8, at(2), 1, f[0], f[1], 0, nullptr) == NOLOCO_ERR_ALIGNMENT);
      CHECK(forward(at(1), at(2) + 4, 1, f[0], f[1], 0, nullptr, 0, 3) == NOLOCO_ERR_ALIGNMENT);
      auto back = [&](const float* norms, const float* by, const float* dh, const float* h, void* out, int32_t type) {
        return noloco_token_log_probs_gradient(plan, at(1), 1, at(2), 2, 1, norms, by, dh, h, out, type, nullptr);
      };
      CHECK(back(nullptr, f[1], nullptr, nullptr, at(10), 0) == NOLOCO_ERR_NULL && back(f[0], nullptr, nullptr, nullptr, at(10), 0) == NOLOCO_ERR_NULL);
      CHECK(back(f[0], f[1], f[2], nullptr, at(10), 0) == NOLOCO_ERR_NULL && back(f[0], f[1], nullptr, nullptr, nullptr, 0) == NOLOCO_ERR_NULL);
      CHECK(back(f[0], f[1], nullptr, nullptr, at(1), 0) == NOLOCO_ERR_INVALID_ARG && back(f[0], f[1], nullptr, nullptr, f[1], 0) == NOLOCO_ERR_INVALID_ARG);
      device = 1;
      CHECK(back(f[0], f[1], nullptr, nullptr, at(1), 1) == NOLOCO_ERR_INVALID_ARG && forward(at(1), at(2), 1, f[0], f[1], 0, nullptr) == NOLOCO_ERR_INVALID_ARG);
      device = 0;
      CHECK(launches == before);
      CHECK(back(f[0], f[1], nullptr, nullptr, at(1), 1) == NOLOCO_OK && launches == before + 1);
      CHECK(noloco_log_prob_plan_destroy(plan) == NOLOCO_OK);
    }
  return 0;
}

static int creation() {
  const noloco_norm norm{0, -1, 4};
  const noloco_linear_layer layer{0, 4, 4, 4, -1, 0};
  noloco_layer_norm_plan* a = reinterpret_cast<noloco_layer_norm_plan*>(1);
  noloco_linear_plan* b = reinterpret_cast<noloco_linear_plan*>(1);
  noloco_log_prob_plan* c = reinterpret_cast<noloco_log_prob_plan*>(1);
  fail_malloc = 1;
  CHECK(noloco_layer_norm_plan_create(&norm, 1, 64, 1, 1, &a) == NOLOCO_ERR_DEVICE && a == nullptr);
  CHECK(noloco_linear_plan_create(&layer, 1, 64, 1, 1, 0, &b) == NOLOCO_ERR_DEVICE && b == nullptr);
  CHECK(noloco_log_prob_plan_create(4, 4, 1, 1, 0, &c) == NOLOCO_ERR_DEVICE && c == nullptr);
  fail_malloc = 0;
  CHECK(noloco_layer_norm_plan_create(nullptr, 1, 64, 1, 1, &a) == NOLOCO_ERR_NULL && noloco_linear_plan_create(nullptr, 1, 64, 1, 1, 0, &b) == NOLOCO_ERR_NULL);
  CHECK(noloco_layer_norm_plan_create(&norm, 1, 64, 1, 1, nullptr) == NOLOCO_ERR_NULL && noloco_linear_plan_create(&layer, 1, 64, 1, 1, 0, nullptr) == NOLOCO_ERR_NULL);
  CHECK(noloco_log_prob_plan_create(4, 4, 1, 1, 0, nullptr) == NOLOCO_ERR_NULL);
  CHECK(noloco_layer_norm_plan_create(nullptr, 0, 64, 1, 1, &a) == NOLOCO_OK && noloco_linear_plan_create(nullptr, 0, 64, 1, 1, 0, &b) == NOLOCO_OK);
  CHECK(noloco_layer_norm_plan_destroy(a) == NOLOCO_OK && noloco_linear_plan_destroy(b) == NOLOCO_OK);
  CHECK(noloco_layer_norm_plan_destroy(nullptr) == NOLOCO_OK && noloco_linear_plan_destroy(nullptr) == NOLOCO_OK && noloco_log_prob_plan_destroy(nullptr) == NOLOCO_OK);
  // a bias between a matrix's rows, and one that reaches into them
  for (int64_t bias = 0; bias < 60; ++bias)
    for (int32_t outputs = 1; outputs < 8; ++outputs) {
      const noloco_linear_layer l{7, 4, outputs, 11, bias, 0};
      bool shares = false;
      for (int r = 0; r < 4; ++r) shares = shares || (bias < 7 + r * 11 + outputs && 7 + r * 11 < bias + outputs);
      const noloco_status st = noloco_linear_plan_create(&l, 1, 128, 1, 1, 0, &b);
      CHECK(st == (shares ? NOLOCO_ERR_SEGMENT_OVERLAP : NOLOCO_OK));
      CHECK(noloco_linear_plan_destroy(b) == NOLOCO_OK);
    }
  return 0;
}

int main() {
  std::setvbuf(stdout, nullptr, _IONBF, 0);
  if (creation() || norms() || matrices() || losses()) return 1;
  CHECK(mallocs == frees && bad == 0);
  std::printf("model host driver: ok\n");
  return 0;
}
