// Which way the products of a call go: model_step.cpp with stand-ins for the HIP runtime and the kernel launchers (built and run by
// tests/product_plans.py). Reads calls from standard input, one a line, and prints their products; no memory is read through.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "model_internal.h"

extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
extern "C" hipError_t hipMalloc(void** ptr, size_t size) {
  std::printf("room %zu\n", size);
  *ptr = std::aligned_alloc(256, 256);
  return hipSuccess;
}
extern "C" hipError_t hipFree(void* ptr) { std::free(ptr); return hipSuccess; }

namespace noloco {

int launch_layer_norm(const NormArgs&, void*) { return 0; }
int launch_layer_norm_gradient(const NormArgs&, void*) { return 0; }
int launch_slope(const SlopeArgs&, void*) { return 0; }
int launch_log_probs(const LogProbArgs&, void*) { return 0; }
int launch_log_probs_gradient(const LogProbArgs&, void*) { return 0; }

// Neighbouring numbers that the end of a product takes at once.
static int end_of(const ProductArgs& a) {
  for (int n : {8, 4}) {
    auto fits = [n](const void* p, int32_t bf16, int64_t steps) {
      return p == nullptr || (reinterpret_cast<uintptr_t>(p) % (bf16 ? 2 * n : 16) == 0 && steps % (bf16 ? n : 4) == 0);
    };
    const int64_t steps = a.out_stride | a.out_ld;
    if (fits(a.out, a.out_bf16, steps) && fits(a.more, a.out_bf16, steps) && fits(a.before, a.out_bf16, steps) && fits(a.bias, a.bias_bf16, a.bias_stride)) return n;
  }
  return 1;
}

int launch_product(const ProductArgs& a, const ProductPlan& p, char*, void*) {
  const bool adds = p.tile > 0 && p.splits == 1 && end_of(a) == 8 && a.activation == NOLOCO_ACT_NONE && a.before == nullptr && a.bias == nullptr && a.n % 8 == 0 &&
                    (a.more != nullptr || a.accumulate);
  std::printf("product tile %d f16 %d parts %d %d splits %u along %d %d packed %d %d end %d adds %d m %u n %u k %u W %d\n", p.tile, p.tile > 0 ? p.f16 : 0, p.parts[0],
              p.parts[1], p.splits, a.a.along_k, a.b.along_k, p.tile > 0 ? p.packed[0] : 0, p.tile > 0 ? p.packed[1] : 0, end_of(a), adds ? 1 : 0, a.m, a.n, a.k, a.W);
  return 0;
}

}  // namespace noloco

static char* at(uint64_t v) { return reinterpret_cast<char*>(v << 43); }     // arrays far from each other

int main() {
  long long W, T, room, offset, inputs, outputs, row_stride, bias, stride;
  int transposed, act, types[5], accumulate, more, gradient;
  while (std::scanf("%d %lld %lld %lld %lld %lld %lld %lld %lld %d %lld %d %d %d %d %d %d %d %d", &gradient, &W, &T, &room, &offset, &inputs, &outputs, &row_stride, &bias,
                    &transposed, &stride, &act, types, types + 1, types + 2, types + 3, types + 4, &accumulate, &more) == 19) {
    const noloco_linear_layer layer{offset, inputs, outputs, row_stride, bias, transposed};
    noloco_linear_plan* plan = nullptr;
    if (noloco_linear_plan_create(&layer, 1, stride, static_cast<int32_t>(W), T, room, &plan) != NOLOCO_OK) return 1;
    const noloco_status st =
        gradient ? noloco_linear_gradient(plan, 0, at(1), types[0], at(2), types[1], at(3), types[2], T, act, act ? at(4) : nullptr, more ? at(5) : nullptr, at(6),
                                          types[3], at(7), types[4], accumulate, nullptr)
                 : noloco_linear(plan, 0, at(1), types[0], at(3), types[1], T, act, more ? at(5) : nullptr, at(4), at(6), types[2], nullptr);
    if (st != NOLOCO_OK) return 2;
    std::printf("done\n");
    noloco_linear_plan_destroy(plan);
  }
  return 0;
}
