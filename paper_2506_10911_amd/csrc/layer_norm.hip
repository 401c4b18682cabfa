// Layer norm and its gradient (kernels and their launchers).
//
//   out = (x - mean) rstd g + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   dx  = add + rstd (d g - mean(d g) - xh mean(d g xh)),  xh = (x - mean) rstd
//   g's gradient = sum over tokens of d xh, b's = sum of d
//
// All are bound by memory: a row is read once and held in registers, by a wave up to 1024 numbers, by a workgroup of 256
// or 1024 threads up to 16384 (the gradient, which holds more, 8192); longer ones are read again from the caches.  The next row is
// asked for before the present one is worked on (by one after the other 8 x 8192 rows of 768 in bf16 took 56 us, their gradient
// 193; so 36 and 79, at 5.7 and 5.1 TB/s; 2 x 8192 rows of 4096 150, so 81).  The variance is summed from the held distances to the mean, so that a mean far from zero
// costs no digits.  Workgroups of one worker keep its weights in registers over all their rows, and sum their rows' shares of
// the weights' gradients there; a second launch adds the workgroups' sums in their order.
#include "device_numbers.h"
#include "model_internal.h"

namespace noloco {
namespace {

// Thread `lane` of the L that hold a row has its vectors lane, lane + L, ... of N numbers, K of them.
template <int N, int K, int L> struct Row {
  static constexpr int kNumbers = N * K;
  float v[kNumbers];
  __device__ __forceinline__ static bool there(uint32_t lane, int k, uint32_t width) { return (lane + k * L) * N < width; }
  __device__ __forceinline__ void load(const void* p, int64_t at, bool bf16, uint32_t lane, uint32_t width) {
    auto each = [&](auto element) {
      typedef decltype(element) E;
      const E* from = static_cast<const E*>(p) + at;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (there(lane, k, width)) {
          Stored<E, N>::load(from + (lane + k * L) * N, v + k * N);
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) v[k * N + i] = 0.f;
        }
      }
    };
    if (bf16) each(uint16_t{}); else each(float{});
  }
  __device__ __forceinline__ void store(void* p, int64_t at, bool bf16, uint32_t lane, uint32_t width) const {
    auto each = [&](auto element) {
      typedef decltype(element) E;
      E* to = static_cast<E*>(p) + at;
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (there(lane, k, width)) Stored<E, N>::store(to + (lane + k * L) * N, v + k * N);
    };
    if (bf16) each(uint16_t{}); else each(float{});
  }
};

// A row on its way: as it lies in memory, so that nobody waits for it before it is widened.  Where types differ (E is void) it is
// widened as it comes.
template <typename E, int N, int K, int L> struct Coming {
  static constexpr int kVector = Stored<E, N>::kVector;
  typedef E vector __attribute__((ext_vector_type(kVector)));
  vector raw[K][N / kVector];
  __device__ __forceinline__ void ask(const void* p, int64_t at, bool, uint32_t lane, uint32_t width) {
    const E* const from = static_cast<const E*>(p) + at;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!Row<N, K, L>::there(lane, k, width)) continue;
#pragma unroll
      for (int i = 0; i < N / kVector; ++i) raw[k][i] = *reinterpret_cast<const vector*>(from + (lane + k * L) * N + i * kVector);
    }
  }
  // The row as numbers; zeros where the thread has none.
  __device__ __forceinline__ void take(Row<N, K, L>& row, uint32_t lane, uint32_t width) const {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float x;
        if constexpr (sizeof(E) == 2) x = widen(raw[k][i / kVector][i % kVector]); else x = raw[k][i / kVector][i % kVector];
        row.v[k * N + i] = Row<N, K, L>::there(lane, k, width) ? x : 0.f;
      }
  }
};
template <int N, int K, int L> struct Coming<void, N, K, L> {
  Row<N, K, L> row;
  __device__ __forceinline__ void ask(const void* p, int64_t at, bool bf16, uint32_t lane, uint32_t width) { row.load(p, at, bf16, lane, width); }
  __device__ __forceinline__ void take(Row<N, K, L>& to, uint32_t, uint32_t) const { to = row; }
};

// E: the type of x and out (and of dout), or void.
template <typename E, int N, int K, int L>
__global__ __launch_bounds__(L < 256 ? 256 : L) void layer_norm_held(NormArgs a) {
  typedef Row<N, K, L> R;
  constexpr uint32_t kThreads = L < 256 ? 256 : L, kRows = kThreads / L;
  __shared__ float shared[2][L > 64 ? L / 64 : 1];
  const uint32_t lane = threadIdx.x % L, width = a.width;
  const int64_t w = blockIdx.y, first = w * a.tokens, step = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / L;
  if (t >= a.tokens) return;              // whole waves, and whole workgroups where these hold a row
  R weight, bias, x;
  Coming<E, N, K, L> coming;
  coming.ask(a.x, (first + t) * width, a.x_bf16, lane, width);
  weight.load(a.theta, w * a.stride + a.weight, a.theta_bf16, lane, width);
  if (a.bias >= 0) {
    bias.load(a.theta, w * a.stride + a.bias, a.theta_bf16, lane, width);
  } else {
#pragma unroll
    for (int i = 0; i < R::kNumbers; ++i) bias.v[i] = 0.f;
  }
  const float count = static_cast<float>(width);
  for (; t < a.tokens; t += step) {
    coming.take(x, lane, width);
    if (t + step < a.tokens) coming.ask(a.x, (first + t + step) * width, a.x_bf16, lane, width);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < R::kNumbers; ++i) sum += x.v[i];
    sum_all<L, 1>(&sum, shared[0]);
    const float mean = sum / count;
    float squares = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float& d = x.v[k * N + i];
        d = R::there(lane, k, width) ? d - mean : 0.f;
        squares += d * d;
      }
    sum_all<L, 1>(&squares, shared[1]);
    const float rstd = 1.f / sqrtf(squares / count + a.eps);
#pragma unroll
    for (int i = 0; i < R::kNumbers; ++i) x.v[i] = x.v[i] * rstd * weight.v[i] + bias.v[i];
    x.store(a.out, (first + t) * width, a.out_bf16, lane, width);
    if (a.stats != nullptr && lane == 0) {
      a.stats[(first + t) * 2] = mean;
      a.stats[(first + t) * 2 + 1] = rstd;
    }
  }
}

// Rows that no workgroup holds: read three times, from the caches.
__global__ __launch_bounds__(1024) void layer_norm_wide(NormArgs a) {
  __shared__ float shared[2][16];
  const int64_t w = blockIdx.y;
  const float count = static_cast<float>(a.width);
  for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const int64_t at = (w * a.tokens + t) * a.width;
    float sum = 0.f, x;
    for (uint32_t i = threadIdx.x; i < a.width; i += 1024) {
      load_numbers<1>(a.x, at + i, a.x_bf16, &x);
      sum += x;
    }
    sum_all<1024, 1>(&sum, shared[0]);
    const float mean = sum / count;
    float squares = 0.f;
    for (uint32_t i = threadIdx.x; i < a.width; i += 1024) {
      load_numbers<1>(a.x, at + i, a.x_bf16, &x);
      squares += (x - mean) * (x - mean);
    }
    sum_all<1024, 1>(&squares, shared[1]);
    const float rstd = 1.f / sqrtf(squares / count + a.eps);
    for (uint32_t i = threadIdx.x; i < a.width; i += 1024) {
      float weight, bias = 0.f;
      load_numbers<1>(a.x, at + i, a.x_bf16, &x);
      load_numbers<1>(a.theta, w * a.stride + a.weight + i, a.theta_bf16, &weight);
      if (a.bias >= 0) load_numbers<1>(a.theta, w * a.stride + a.bias + i, a.theta_bf16, &bias);
      x = (x - mean) * rstd * weight + bias;
      store_numbers<1>(a.out, at + i, a.out_bf16, &x);
    }
    if (a.stats != nullptr && threadIdx.x == 0) {
      a.stats[(w * a.tokens + t) * 2] = mean;
      a.stats[(w * a.tokens + t) * 2 + 1] = rstd;
    }
  }
}

template <typename E, int N, int K, int L>
__global__ __launch_bounds__(L < 256 ? 256 : L) void layer_norm_gradient_held(NormArgs a) {
  typedef Row<N, K, L> R;
  constexpr uint32_t kThreads = L < 256 ? 256 : L, kRows = kThreads / L;
  __shared__ float shared[2][2 * (L > 64 ? L / 64 : 1)];
  const uint32_t lane = threadIdx.x % L, sub = threadIdx.x / L, width = a.width;
  const int64_t w = blockIdx.y, first = w * a.tokens, step = static_cast<int64_t>(gridDim.x) * kRows;
  R weight, of_weight, of_bias;
  weight.load(a.theta, w * a.stride + a.weight, a.theta_bf16, lane, width);
#pragma unroll
  for (int i = 0; i < R::kNumbers; ++i) of_weight.v[i] = of_bias.v[i] = 0.f;
  const float count = static_cast<float>(width);
  int turn = 0;
  Coming<E, N, K, L> coming_x, coming_d, coming_add;
  float mean = 0.f, rstd = 0.f;
  auto ask = [&](int64_t t) {
    const int64_t at = (first + t) * width;
    coming_x.ask(a.x, at, a.x_bf16, lane, width);
    coming_d.ask(a.dout, at, a.dout_bf16, lane, width);
    if (a.add != nullptr) coming_add.ask(a.add, at, a.out_bf16, lane, width);
    mean = a.stats[(first + t) * 2];
    rstd = a.stats[(first + t) * 2 + 1];
  };
  int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + sub;
  if (t < a.tokens) ask(t);
  for (; t < a.tokens; t += step) {
    R x, d, add;
    coming_x.take(x, lane, width);
    coming_d.take(d, lane, width);
    if (a.add != nullptr) {
      coming_add.take(add, lane, width);
    } else {
#pragma unroll
      for (int i = 0; i < R::kNumbers; ++i) add.v[i] = 0.f;
    }
    const float mine = mean, scale = rstd;
    if (t + step < a.tokens) ask(t + step);
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = k * N + i;
        x.v[e] = R::there(lane, k, width) ? (x.v[e] - mine) * scale : 0.f;
        of_weight.v[e] += d.v[e] * x.v[e];
        of_bias.v[e] += d.v[e];
        d.v[e] *= weight.v[e];
        sums[0] += d.v[e];
        sums[1] += d.v[e] * x.v[e];
      }
    sum_all<L, 2>(sums, shared[turn]);
    turn ^= 1;
    sums[0] /= count;
    sums[1] /= count;
#pragma unroll
    for (int i = 0; i < R::kNumbers; ++i) x.v[i] = add.v[i] + scale * (d.v[i] - sums[0] - x.v[i] * sums[1]);
    x.store(a.out, (first + t) * width, a.out_bf16, lane, width);
  }
  if (a.grad == nullptr) return;
  // The workgroup's rows together, in their order.
  if constexpr (kRows > 1) {
    __shared__ float joined[kRows][L * R::kNumbers];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      R& mine = which == 0 ? of_weight : of_bias;
      if (which == 1) __syncthreads();
#pragma unroll
      for (int i = 0; i < R::kNumbers; ++i) joined[sub][i * L + lane] = mine.v[i];
      __syncthreads();
      if (sub == 0) {
#pragma unroll
        for (int i = 0; i < R::kNumbers; ++i)
#pragma unroll
          for (uint32_t s = 1; s < kRows; ++s) mine.v[i] += joined[s][i * L + lane];
      }
    }
  }
  if (sub == 0) {
    const int64_t to = (w * a.groups + blockIdx.x) * 2 * static_cast<int64_t>(width);
    of_weight.store(a.partial, to, false, lane, width);
    if (a.bias >= 0) of_bias.store(a.partial, to + width, false, lane, width);
  }
}

__global__ __launch_bounds__(1024) void layer_norm_gradient_wide(NormArgs a) {
  __shared__ float shared[2][32];
  const int64_t w = blockIdx.y;
  const float count = static_cast<float>(a.width);
  int turn = 0;
  for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const int64_t at = (w * a.tokens + t) * a.width;
    const float mean = a.stats[(w * a.tokens + t) * 2], rstd = a.stats[(w * a.tokens + t) * 2 + 1];
    float sums[2] = {0.f, 0.f}, x, d, weight;
    for (uint32_t i = threadIdx.x; i < a.width; i += 1024) {
      load_numbers<1>(a.x, at + i, a.x_bf16, &x);
      load_numbers<1>(a.dout, at + i, a.dout_bf16, &d);
      load_numbers<1>(a.theta, w * a.stride + a.weight + i, a.theta_bf16, &weight);
      sums[0] += d * weight;
      sums[1] += d * weight * ((x - mean) * rstd);
    }
    sum_all<1024, 2>(sums, shared[turn]);
    turn ^= 1;
    sums[0] /= count;
    sums[1] /= count;
    for (uint32_t i = threadIdx.x; i < a.width; i += 1024) {
      float add = 0.f;
      load_numbers<1>(a.x, at + i, a.x_bf16, &x);
      load_numbers<1>(a.dout, at + i, a.dout_bf16, &d);
      load_numbers<1>(a.theta, w * a.stride + a.weight + i, a.theta_bf16, &weight);
      if (a.add != nullptr) load_numbers<1>(a.add, at + i, a.out_bf16, &add);
      x = add + rstd * (d * weight - sums[0] - (x - mean) * rstd * sums[1]);
      store_numbers<1>(a.out, at + i, a.out_bf16, &x);
    }
  }
}

// The weights' gradients of wide rows: a thread takes a column of every `groups`th token.
__global__ __launch_bounds__(256) void layer_norm_columns(NormArgs a) {
  const uint32_t column = blockIdx.x * 256 + threadIdx.x;
  const int64_t w = blockIdx.z;
  if (column >= a.width) return;
  float of_weight = 0.f, of_bias = 0.f, x, d;
  for (int64_t t = blockIdx.y; t < a.tokens; t += a.groups) {
    const int64_t row = w * a.tokens + t, at = row * a.width + column;
    load_numbers<1>(a.x, at, a.x_bf16, &x);
    load_numbers<1>(a.dout, at, a.dout_bf16, &d);
    of_weight += d * ((x - a.stats[row * 2]) * a.stats[row * 2 + 1]);
    of_bias += d;
  }
  float* const to = a.partial + (w * a.groups + blockIdx.y) * 2 * static_cast<int64_t>(a.width) + column;
  to[0] = of_weight;
  to[a.width] = of_bias;
}

// A worker's groups together, 4 to 7 us: a workgroup takes 64 columns, its four waves a quarter of the groups each.
__global__ __launch_bounds__(256) void layer_norm_join(NormArgs a) {
  __shared__ float quarter[4][64];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = blockIdx.z;
  const uint32_t column = blockIdx.x * 64 + lane;
  const int64_t w = blockIdx.y;
  const uint32_t from = a.groups * wave / 4, to = a.groups * (wave + 1) / 4;
  float sum = 0.f;
  if (column < a.width && a.tokens > 0) {
    const float* p = a.partial + (w * a.groups * 2 + which) * static_cast<int64_t>(a.width) + column;
#pragma unroll 8
    for (uint32_t g = from; g < to; ++g) sum += p[2 * static_cast<int64_t>(a.width) * g];
  }
  quarter[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || column >= a.width) return;
  sum = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
  const int64_t at = w * a.stride + (which == 0 ? a.weight : a.bias) + column;
  if (a.accumulate) {
    float old;
    load_numbers<1>(a.grad, at, a.grad_bf16, &old);
    sum += old;
  }
  store_numbers<1>(a.grad, at, a.grad_bf16, &sum);
}

// Vectors of eight or four where weights and rows allow, of those the one that leaves fewer threads without numbers (768 by
// 64 threads: three vectors of four each, or one and a half of eight).
// MOST: numbers of a thread of 1024, whose registers are 128.
template <int MOST, typename Launch> int with_shape(const NormArgs& a, const Launch& launch) {
  const int64_t places = a.width | a.weight | (a.bias >= 0 ? a.bias : 0);
  auto with_threads = [&](auto threads) {
    constexpr int L = decltype(threads)::value;
    constexpr bool kWhole = L < 1024 || MOST == 16;
    auto vectors = [&](int n) { return (static_cast<int>(a.width) / n + L - 1) / L; };
    const int four = vectors(4), eight = vectors(8);
    if (places % 8 == 0 && eight * 8 <= four * 4) {
      if (eight == 1) return launch(Number<8>{}, Number<1>{}, threads);
      if constexpr (kWhole) return launch(Number<8>{}, Number<2>{}, threads);
    }
    if (places % 4 == 0) {
      if (four == 1) return launch(Number<4>{}, Number<1>{}, threads);
      if (four == 2) return launch(Number<4>{}, Number<2>{}, threads);
      if constexpr (kWhole) return four == 3 ? launch(Number<4>{}, Number<3>{}, threads) : launch(Number<4>{}, Number<4>{}, threads);
    }
    const int one = vectors(1);
    if (one <= 2) return launch(Number<1>{}, Number<2>{}, threads);
    if (one <= 4) return launch(Number<1>{}, Number<4>{}, threads);
    if constexpr (kWhole)
      if (one > 8) return launch(Number<1>{}, Number<16>{}, threads);
    return launch(Number<1>{}, Number<8>{}, threads);
  };
  if (a.width <= 1024) return with_threads(Number<64>{});
  return a.width <= 4096 ? with_threads(Number<256>{}) : with_threads(Number<1024>{});
}

}  // namespace

int launch_layer_norm(const NormArgs& args, void* stream) {
  // eight workgroups of 256 threads a CU, which take as many rows each as there are
  const int64_t rows = args.width <= 1024 ? 4 : 1, most = std::max<int64_t>(1, (args.width > 4096 ? 512 : 2048) / args.W);
  const dim3 grid(static_cast<uint32_t>(std::min((args.tokens + rows - 1) / rows, most)), args.W);
  if (args.width > kNormHeld) return enqueue(layer_norm_wide, grid, 1024, 0, stream, args);
  return with_shape<16>(args, [&](auto n, auto k, auto threads) {
    constexpr int N = decltype(n)::value, K = decltype(k)::value, L = decltype(threads)::value;
    auto with = [&](auto kernel) { return enqueue(kernel, grid, L < 256 ? 256 : L, 0, stream, args); };
    if (args.x_bf16 != args.out_bf16) return with(layer_norm_held<void, N, K, L>);
    return args.x_bf16 ? with(layer_norm_held<uint16_t, N, K, L>) : with(layer_norm_held<float, N, K, L>);
  });
}

int launch_layer_norm_gradient(const NormArgs& args, void* stream) {
  const dim3 grid(args.groups, args.W);
  if (args.tokens > 0) {
    int st;
    if (args.width > kNormGradientHeld) {
      st = enqueue(layer_norm_gradient_wide, grid, 1024, 0, stream, args);
      if (st == 0 && args.grad != nullptr)
        st = enqueue(layer_norm_columns, dim3((args.width + 255) / 256, args.groups, args.W), 256, 0, stream, args);
    } else {
      st = with_shape<8>(args, [&](auto n, auto k, auto threads) {
        constexpr int N = decltype(n)::value, K = decltype(k)::value, L = decltype(threads)::value;
        auto with = [&](auto kernel) { return enqueue(kernel, grid, L < 256 ? 256 : L, 0, stream, args); };
        if (args.x_bf16 != args.out_bf16 || args.x_bf16 != args.dout_bf16) return with(layer_norm_gradient_held<void, N, K, L>);
        return args.x_bf16 ? with(layer_norm_gradient_held<uint16_t, N, K, L>) : with(layer_norm_gradient_held<float, N, K, L>);
      });
    }
    if (st != 0) return st;
  }
  if (args.grad == nullptr) return 0;
  return enqueue(layer_norm_join, dim3((args.width + 63) / 64, args.W, args.bias >= 0 ? 2 : 1), 256, 0, stream, args);
}

}  // namespace noloco
