// dz = dout act'(before), the gradient before a matrix's activation, and its sums over the tokens, the bias's gradient (kernels and
// their launcher).
#include "activations.h"
#include "device_numbers.h"
#include "model_internal.h"

namespace noloco {
namespace {


// A workgroup takes 64 N columns of a group of tokens, every wave a fourth of them.
template <typename E, typename Z, int N>
__global__ __launch_bounds__(256) void linear_slope(SlopeArgs a) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = (blockIdx.x * 64 + lane) * N;
  const int64_t w = blockIdx.z, each = (a.tokens + a.groups - 1) / a.groups;
  const int64_t first = blockIdx.y * each, last = first + each < a.tokens ? first + each : a.tokens;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  if (column < a.outputs) {
    for (int64_t t = first + wave; t < last; t += 4) {
      const int64_t at = (w * a.tokens + t) * a.outputs + column;
      float d[N];
      Stored<E, N>::load(static_cast<const E*>(a.dout) + at, d);
      if (a.before != nullptr) {
        float z[N];
        Stored<E, N>::load(static_cast<const E*>(a.before) + at, z);
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] *= slope_of(a.activation, z[i]);
        if (a.dz != nullptr) Stored<Z, N>::store(static_cast<Z*>(a.dz) + at, d);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += d[i];
    }
  }
  if (a.partial == nullptr) return;
  __shared__ float waves[4][64 * N];
#pragma unroll
  for (int i = 0; i < N; ++i) waves[wave][i * 64 + lane] = sum[i];
  __syncthreads();
  if (wave != 0 || column >= a.outputs) return;
  float* const to = a.partial + (w * a.groups + blockIdx.y) * static_cast<int64_t>(a.outputs) + column;
#pragma unroll
  for (int i = 0; i < N; ++i)
    to[i] = (waves[0][i * 64 + lane] + waves[1][i * 64 + lane]) + (waves[2][i * 64 + lane] + waves[3][i * 64 + lane]);
}

__global__ __launch_bounds__(256) void linear_slope_join(SlopeArgs a) {
  __shared__ float quarter[4][64];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = blockIdx.x * 64 + lane;
  const int64_t w = blockIdx.y;
  const uint32_t from = a.groups * wave / 4, to = a.groups * (wave + 1) / 4;
  float sum = 0.f;
  if (column < a.outputs && a.tokens > 0) {
    const float* p = a.partial + w * a.groups * static_cast<int64_t>(a.outputs) + column;
#pragma unroll 8
    for (uint32_t g = from; g < to; ++g) sum += p[static_cast<int64_t>(a.outputs) * g];
  }
  quarter[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || column >= a.outputs) return;
  sum = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
  const int64_t at = w * a.stride + column;
  if (a.accumulate) {
    float old;
    load_numbers<1>(a.grad, at, a.grad_bf16, &old);
    sum += old;
  }
  store_numbers<1>(a.grad, at, a.grad_bf16, &sum);
}

}  // namespace

int launch_slope(const SlopeArgs& args, void* stream) {
  if (args.tokens > 0) {
    auto with = [&](auto e, auto z) {
      typedef decltype(e) E;
      typedef decltype(z) Z;
      const uint32_t n = args.outputs % 8 == 0 ? 8 : (args.outputs % 4 == 0 ? 4 : 1);
      const dim3 grid((args.outputs + 64 * n - 1) / (64 * n), args.groups, args.W);
      if (n == 8) return enqueue(linear_slope<E, Z, 8>, grid, 256, 0, stream, args);
      if (n == 4) return enqueue(linear_slope<E, Z, 4>, grid, 256, 0, stream, args);
      return enqueue(linear_slope<E, Z, 1>, grid, 256, 0, stream, args);
    };
    int st;
    if (args.dout_bf16) st = args.dz_bf16 ? with(uint16_t{}, uint16_t{}) : with(uint16_t{}, float{});
    else st = args.dz_bf16 ? with(float{}, uint16_t{}) : with(float{}, float{});
    if (st != 0) return st;
  }
  if (args.grad == nullptr) return 0;
  return enqueue(linear_slope_join, dim3((args.outputs + 63) / 64, args.W), 256, 0, stream, args);
}

}  // namespace noloco
