// dz = dout act'(before), the gradient before a matrix's activation, and its sums over the tokens, the bias's gradient (kernels and
// their launcher).
#include "activations.h"
#include "device_numbers.h"
#include "model_internal.h"

namespace noloco {
namespace {


__device__ __forceinline__ void put_bias(const SlopeArgs& a, int64_t w, uint32_t column, float sum) {
  const int64_t at = w * a.stride + column;
  if (a.accumulate) {
    float old;
    load_numbers<1>(a.grad, at, a.grad_bf16, &old);
    sum += old;
  }
  store_numbers<1>(a.grad, at, a.grad_bf16, &sum);
}

// A workgroup takes 64 N columns of a group of tokens; its waves (four, or sixteen where there is one group) take the tokens in turn, a
// few at a time whose numbers are on their way together.  Bound by memory, with an activation nearly as much by its slope's instructions: 2 x 4096 x 16384 through the
// normal distribution's 167 us (4.8 TB/s).
template <typename E, typename Z, int N, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void linear_slope(SlopeArgs a) {
  constexpr int kAhead = N == 8 ? 2 : 4;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = (blockIdx.x * 64 + lane) * N;
  const int64_t w = blockIdx.z, each = (a.tokens + a.groups - 1) / a.groups;
  const int64_t first = blockIdx.y * each, last = first + each < a.tokens ? first + each : a.tokens;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  if (column < a.outputs) {
    for (int64_t t = first + wave; t < last; t += kAhead * WAVES) {
      float d[kAhead][N], z[kAhead][N];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (t + k * WAVES >= last) break;
        const int64_t at = (w * a.tokens + t + k * WAVES) * a.outputs + column;
        Stored<E, N>::load(static_cast<const E*>(a.dout) + at, d[k]);
        if (a.before != nullptr) Stored<E, N>::load(static_cast<const E*>(a.before) + at, z[k]);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (t + k * WAVES >= last) break;
        if (a.before != nullptr) {
          times_slope<N>(a.activation, z[k], d[k]);
          Stored<Z, N>::store(static_cast<Z*>(a.dz) + (w * a.tokens + t + k * WAVES) * a.outputs + column, d[k]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += d[k][i];
      }
    }
  }
  if (a.grad == nullptr) return;
  __shared__ float waves[WAVES][64 * N];
#pragma unroll
  for (int i = 0; i < N; ++i) waves[wave][lane * N + i] = sum[i];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < 64 * N; i += WAVES * 64) {
    const uint32_t mine = blockIdx.x * 64 * N + i;
    if (mine >= a.outputs) break;
    float all = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < WAVES; ++k) all += waves[k][i];
    if (a.groups == 1) put_bias(a, w, mine, all); else a.partial[(w * a.groups + blockIdx.y) * static_cast<int64_t>(a.outputs) + mine] = all;
  }
}

// The groups' sums, in their order.
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
  put_bias(a, w, column, sum);
}

}  // namespace

int launch_slope(const SlopeArgs& args, void* stream) {
  if (args.tokens > 0) {
    auto with = [&](auto e, auto z) {
      typedef decltype(e) E;
      typedef decltype(z) Z;
      const uint32_t n = args.outputs % 8 == 0 ? 8 : (args.outputs % 4 == 0 ? 4 : 1);
      const dim3 grid((args.outputs + 64 * n - 1) / (64 * n), args.groups, args.W);
      auto with_waves = [&](auto numbers) {
        constexpr int N = decltype(numbers)::value;
        return args.groups == 1 ? enqueue(linear_slope<E, Z, N, 16>, grid, 1024, 0, stream, args) : enqueue(linear_slope<E, Z, N, 4>, grid, 256, 0, stream, args);
      };
      return n == 8 ? with_waves(Number<8>{}) : (n == 4 ? with_waves(Number<4>{}) : with_waves(Number<1>{}));
    };
    int st;
    if (args.dout_bf16) st = args.dz_bf16 ? with(uint16_t{}, uint16_t{}) : with(uint16_t{}, float{});
    else st = args.dz_bf16 ? with(float{}, uint16_t{}) : with(float{}, float{});
    if (st != 0) return st;
  }
  if (args.grad == nullptr || (args.groups == 1 && args.tokens > 0)) return 0;
  return enqueue(linear_slope_join, dim3((args.outputs + 63) / 64, args.W), 256, 0, stream, args);
}

}  // namespace noloco
