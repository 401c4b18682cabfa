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
// erfcf is some 100 instructions with branches, this one 20.
struct Normal { float below, density; };
__device__ __forceinline__ Normal normal(float z) {
  const float x = fabsf(z), t = __builtin_amdgcn_rcpf(1.f + 0.24748737f * x), e = exp_of(-0.5f * z * z);
  const float q[10] = {0.0987347926f, 0.0987040906f, 0.0928540676f, 0.0806080689f, 0.0587978355f,
                       0.0695167604f, -0.0445770242f, 0.113392267f, -0.0889537405f, 0.0209228872f};
  float sum = q[9];
#pragma unroll
  for (int i = 8; i >= 0; --i) sum = fmaf(sum, t, q[i]);
  const float tail = e > 0.f ? e * (t * sum) : (z == z ? 0.f : z);
  return {z > 0.f ? 1.f - tail : tail, 0.39894228040143268f * e};
}

__device__ __forceinline__ float activate(int32_t activation, float z) {
  switch (activation) {
    case NOLOCO_ACT_RELU: return z > 0.f || z != z ? z : 0.f;
    case NOLOCO_ACT_GELU: return z * normal(z).below;
    case NOLOCO_ACT_GELU_TANH: return z * sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z));
    case NOLOCO_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}

__device__ __forceinline__ float slope_of(int32_t activation, float z) {
  switch (activation) {
    case NOLOCO_ACT_RELU: return z != z ? z : (z > 0.f ? 1.f : 0.f);
    case NOLOCO_ACT_GELU: {
      const Normal n = normal(z);
      return n.density > 0.f ? n.below + z * n.density : n.below;
    }
    case NOLOCO_ACT_GELU_TANH: {
      const float s = sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z)), by = s * (1.f - s);
      return by > 0.f ? s + z * by * (1.5957691216057308f * (1.f + 0.134145f * z * z)) : s;
    }
    case NOLOCO_ACT_SILU: {
      const float s = sigmoid(z);
      return s > 0.f ? s * (1.f + z * (1.f - s)) : s;
    }
    default: return 1.f;
  }
}

}  // namespace
}  // namespace noloco
