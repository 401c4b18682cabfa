// What noloco_linear applies and its slope, in binary32.  Device code only.
#pragma once

#include "device_numbers.h"
#include "noloco.h"

namespace noloco {
namespace {

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// 1 / (1 + exp(-x)); 0 where exp(-x) leaves binary32.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + exp_of(-x)); }

// The normal distribution below z, and its density.  The tail 1 - Phi(|z|) = erfc(|z| / sqrt(2)) / 2 is exp(-z^2 / 2) t Q(t) with
// t = 1 / (1 + 0.35 |z| / sqrt(2)); Q is a polynomial that was fitted to this form for the least relative error over |z| < 20
// (1.0e-8, Chebyshev points, reweighted least squares).  In binary32 the result is off by 5e-7 of itself beside exp's own error.
// erfcf is some 100 instructions with branches, this one 18, which is what a tile's end spends most of its time on where activations are
// asked for.
struct Normal { float tail, density; };          // tail: 1 - Phi(|z|)
__device__ __forceinline__ Normal normal(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.24748737f, fabsf(z), 1.f)), e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
  const float q[10] = {0.0987347926f, 0.0987040906f, 0.0928540676f, 0.0806080689f, 0.0587978355f,
                       0.0695167604f, -0.0445770242f, 0.113392267f, -0.0889537405f, 0.0209228872f};
  float sum = q[9];
#pragma unroll
  for (int i = 8; i >= 0; --i) sum = fmaf(sum, t, q[i]);
  return {e * (t * sum), 0.39894228040143268f * e};
}

// z without its infinities (of both signs, or the negative one), whose product with a factor that has become zero would be NaN: act(-infinity)
// is 0, as act's values before it are.  One instruction; a NaN may come out as a number, but the factor is NaN then.  (fminf and fmaxf are two
// each: 8 x 4096 x 2048 x 8192 through the normal distribution 1236 us, so 1223.)
__device__ __forceinline__ float size_of(float z) { return __builtin_amdgcn_fmed3f(fabsf(z), 0.f, 3.402823466e38f); }
__device__ __forceinline__ float not_lowest(float z) { return __builtin_amdgcn_fmed3f(z, -3.402823466e38f, __builtin_inff()); }

// act(z) in place of z, for N numbers.
template <int N> __device__ __forceinline__ void activate(int32_t activation, float* v) {
  auto each = [&](auto act) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act(v[i]);
  };
  switch (activation) {
    case NOLOCO_ACT_RELU: return each([](float z) { return z > 0.f || z != z ? z : 0.f; });
    case NOLOCO_ACT_GELU: return each([](float z) { return fmaf(-size_of(z), normal(z).tail, fmaxf(z, 0.f)); });
    case NOLOCO_ACT_GELU_TANH: return each([](float z) { return not_lowest(z) * sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z)); });
    case NOLOCO_ACT_SILU: return each([](float z) { return not_lowest(z) * sigmoid(z); });
    default: return;
  }
}

// d act'(z) in place of d.
template <int N> __device__ __forceinline__ void times_slope(int32_t activation, const float* z, float* d) {
  auto each = [&](auto slope) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= slope(z[i]);
  };
  switch (activation) {
    case NOLOCO_ACT_RELU: return each([](float z) { return z != z ? z : (z > 0.f ? 1.f : 0.f); });
    case NOLOCO_ACT_GELU:
      return each([](float z) {
        const Normal n = normal(z);
        const float below = z > 0.f ? 1.f - n.tail : n.tail;
        return n.density > 0.f ? fmaf(z, n.density, below) : below;
      });
    case NOLOCO_ACT_GELU_TANH:
      return each([](float z) {
        const float s = sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z)), by = s * (1.f - s);
        return by > 0.f ? s + z * by * (1.5957691216057308f * (1.f + 0.134145f * z * z)) : s;
      });
    case NOLOCO_ACT_SILU:
      return each([](float z) {
        const float s = sigmoid(z), by = s * (1.f - s);
        return by > 0.f ? s * (1.f + z * (1.f - s)) : s;
      });
    default: return;
  }
}

}  // namespace
}  // namespace noloco
