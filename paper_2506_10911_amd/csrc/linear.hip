// Matrices with bias, activation and residual, and their gradient (kernels and their launchers).
//
//   z = x M + bias, out = act(z) + residual;  dz = dout act'(z), dx = dz M^T + add, M's gradient = x^T dz
//
// All three are products sum over k of A(m, k) B(n, k), whose operands lie with their numbers along k or along m (n) next to
// each other.  The matrix cores take bf16.  A bf16 operand goes in as it is.  A float operand is rounded to bf16 where the
// result is bf16 (its own rounding is as large), and is taken apart into three bf16 where the result is float: high, middle
// and low eight bits, which together are the number; of the products of parts the six (or three, beside a bf16 operand) are
// summed that reach 2^-16 of the largest, and what is left out is below binary32's own rounding.
#include <type_traits>

#include "device_numbers.h"
#include "model_internal.h"

namespace noloco {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint16_t ushort8 __attribute__((ext_vector_type(8)));

#define lds_memory __attribute__((address_space(3)))

__device__ __forceinline__ float activate(int32_t activation, float z) {
  switch (activation) {
    case NOLOCO_ACT_RELU: return z > 0.f || z != z ? z : 0.f;
    case NOLOCO_ACT_GELU: return 0.5f * z * erfcf(z * -0.70710678118654752f);
    case NOLOCO_ACT_GELU_TANH: return z / (1.f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
    case NOLOCO_ACT_SILU: return z / (1.f + expf(-z));
    default: return z;
  }
}

__device__ __forceinline__ float slope_of(int32_t activation, float z) {
  switch (activation) {
    case NOLOCO_ACT_RELU: return z != z ? z : (z > 0.f ? 1.f : 0.f);
    case NOLOCO_ACT_GELU: return 0.5f * erfcf(z * -0.70710678118654752f) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    case NOLOCO_ACT_GELU_TANH: {
      const float s = 1.f / (1.f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
      const float by = s * (1.f - s);
      return s + (by > 0.f ? z * by * (1.5957691216057308f * (1.f + 0.134145f * z * z)) : 0.f);
    }
    case NOLOCO_ACT_SILU: {
      const float s = 1.f / (1.f + expf(-z));
      return s > 0.f ? s * (1.f + z * (1.f - s)) : 0.f;
    }
    default: return 1.f;
  }
}

// The end of a product for N neighbouring numbers of a row.
template <int N> __device__ __forceinline__ void finish(const ProductArgs& a, int64_t w, uint32_t m, uint32_t n, float* v) {
  const int64_t at = w * a.out_stride + m * a.out_ld + n;
  if (a.bias != nullptr) {
    float bias[N];
    load_numbers<N>(a.bias, w * a.bias_stride + n, a.bias_bf16, bias);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += bias[i];
  }
  if (a.before != nullptr) store_numbers<N>(a.before, at, a.out_bf16, v);
  if (a.activation != NOLOCO_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activate(a.activation, v[i]);
  }
  if (a.more != nullptr || a.accumulate) {
    float more[N];
    load_numbers<N>(a.accumulate ? a.out : a.more, at, a.out_bf16, more);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += more[i];
  }
  store_numbers<N>(a.out, at, a.out_bf16, v);
}

// Do four neighbouring numbers of everything that the end of a product touches lie at a multiple of their size?
__device__ __forceinline__ bool ends_in_fours(const ProductArgs& a) {
  auto fits = [](const void* p, int32_t bf16) { return reinterpret_cast<uintptr_t>(p) % (bf16 ? 8 : 16) == 0; };
  return ((a.out_stride | a.out_ld) & 3) == 0 && fits(a.out, a.out_bf16) && fits(a.more, a.out_bf16) && fits(a.before, a.out_bf16) &&
         (a.bias == nullptr || ((a.bias_stride & 3) == 0 && fits(a.bias, a.bias_bf16)));
}

// ---------------------------------------------------------------------------
// Products of any operands
// ---------------------------------------------------------------------------

constexpr int kTile = 128, kDepth = 32;
constexpr int kPlane = kTile * kDepth * 2;       // bytes of one part of an operand's stage

// Sixteen neighbouring numbers of an operand, as they come from memory; those that are not there are zeros.
template <typename E> struct Sixteen {
  E v[16];
  __device__ __forceinline__ void load(const E* p, int there, bool whole) {
    if (whole) {
      constexpr int kVector = 16 / sizeof(E);
      typedef E vector __attribute__((ext_vector_type(kVector)));
#pragma unroll
      for (int i = 0; i < 16; i += kVector) {
        const vector x = *reinterpret_cast<const vector*>(p + i);
#pragma unroll
        for (int k = 0; k < kVector; ++k) v[i + k] = x[k];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = i < there ? p[i] : E(0);
    }
  }
  // Part `part` of PARTS of numbers first .. first + 7.
  template <int PARTS> __device__ __forceinline__ ushort8 part(int part, int first) const {
    ushort8 out;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(E) == 2) {
        out[i] = v[first + i];
      } else if constexpr (PARTS == 1) {
        out[i] = narrow(v[first + i]);
      } else {
        // cut, not rounded: each rest is exact, and the third has at most eight bits
        float x = v[first + i];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (k < part) x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        out[i] = static_cast<uint16_t>(__float_as_uint(x) >> 16);
      }
    }
    return out;
  }
};

// 128 x 128 of the result by four waves, each 64 x 64 in blocks of 32 x 32.  Operands come through registers, where they are
// taken apart, one stage of 32 k ahead of the products.
//
// Numbers along k: rows of 64 bytes, 16-byte chunk q of row r at q ^ (r >> 2 & 3), so that 16 lanes meet 16 quarters of the
// LDS's banks.  Numbers along m: rows of 256 bytes, one k each, chunk q of row k at q ^ (k & 3) << 2, turned by the LDS's
// transposing reads.
template <typename TA, typename TB, bool ALONG_A, bool ALONG_B, int PA, int PB>
__global__ __launch_bounds__(256) void product_any(ProductArgs a) {
  __shared__ __align__(1024) char lds[(PA + PB) * kPlane];
  const uint32_t thread = threadIdx.x, lane = thread & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const uint32_t wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  const uint32_t tiles_m = (a.m + kTile - 1) / kTile;
  const uint32_t m0 = blockIdx.x % tiles_m * kTile, n0 = blockIdx.x / tiles_m * kTile;
  const int64_t w = blockIdx.y;
  const TA* const pa = static_cast<const TA*>(a.a.p) + w * a.a.worker_stride;
  const TB* const pb = static_cast<const TB*>(a.b.p) + w * a.b.worker_stride;

  auto load = [&](auto& into, const auto* p, int64_t ld, auto along, uint32_t first, uint32_t size, uint32_t k0) {
    typedef typename std::remove_reference<decltype(*p)>::type E;
    const bool aligned = ((reinterpret_cast<uintptr_t>(p) | static_cast<uint64_t>(ld) * sizeof(E)) & 15) == 0;
    const uint32_t row = first + (along ? thread >> 1 : (thread & 7) * 16), k = k0 + (along ? (thread & 1) * 16 : thread >> 3);
    const int64_t there = along ? (row < size ? static_cast<int64_t>(a.k) - k : 0) : (k < a.k ? static_cast<int64_t>(size) - row : 0);
    const int64_t at = along ? row * ld + k : k * ld + row;
    into.load(p + (there > 0 ? at : 0), static_cast<int>(there < 0 ? 0 : there < 16 ? there : 16), aligned && there >= 16);
  };
  auto put = [&](const auto& from, auto along, auto parts, char* to) {
    constexpr int P = decltype(parts)::value;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t row = along ? thread >> 1 : thread >> 3, q = along ? (thread & 1) * 2 + h : (thread & 7) * 2 + h;
        const uint32_t at = along ? row * 64 + ((q ^ (row >> 2 & 3)) << 4) : row * 256 + ((q ^ (row & 3) << 2) << 4);
        *reinterpret_cast<ushort8*>(to + p * kPlane + at) = from.template part<P>(p, h * 8);
      }
  };
  // Fragment: number lane % 32 of a block of 32, eight k from 8 (lane / 32) on.
  const uint32_t of32 = lane & 31, half = lane >> 5;
  auto fragment = [&](const char* plane, auto along, uint32_t first, int slice) {
    if (along) {
      const uint32_t row = first + of32, q = slice * 2 + half;
      return *reinterpret_cast<const bf16x8*>(plane + row * 64 + ((q ^ (row >> 2 & 3)) << 4));
    } else {
      const uint32_t k = slice * 16 + half * 8 + (lane >> 2 & 3), byte = first * 2 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
      const char* const at = plane + k * 256 + (((byte >> 4) ^ (k & 3) << 2) << 4) + (byte & 15);
      const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(at));
      const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(at + 4 * 256));
      return __builtin_bit_cast(bf16x8, static_cast<short8v>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)));
    }
  };
  typedef typename std::conditional<ALONG_A, Yes, No>::type AlongA;
  typedef typename std::conditional<ALONG_B, Yes, No>::type AlongB;
  Sixteen<TA> next_a;
  Sixteen<TB> next_b;
  float16v acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  if (a.k > 0) {
    load(next_a, pa, a.a.ld, AlongA{}, m0, a.m, 0);
    load(next_b, pb, a.b.ld, AlongB{}, n0, a.n, 0);
  }
  for (uint32_t k0 = 0; k0 < a.k; k0 += kDepth) {
    put(next_a, AlongA{}, Number<PA>{}, lds);
    put(next_b, AlongB{}, Number<PB>{}, lds + PA * kPlane);
    __syncthreads();
    if (k0 + kDepth < a.k) {
      load(next_a, pa, a.a.ld, AlongA{}, m0, a.m, k0 + kDepth);
      load(next_b, pb, a.b.ld, AlongB{}, n0, a.n, k0 + kDepth);
    }
#pragma unroll
    for (int slice = 0; slice < kDepth / 16; ++slice) {
      bf16x8 fa[PA][2], fb[PB][2];
#pragma unroll
      for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[p][i] = fragment(lds + p * kPlane, AlongA{}, wm + i * 32, slice);
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int j = 0; j < 2; ++j) fb[p][j] = fragment(lds + (PA + p) * kPlane, AlongB{}, wn + j * 32, slice);
      // the small products first
#pragma unroll
      for (int both = 2; both >= 0; --both)
#pragma unroll
        for (int p = 0; p <= both; ++p) {
          if (p >= PA || both - p >= PB) continue;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[both - p][j], fa[p][i], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();
  }

  // Block (i, j), element e of a lane: m = 32 i + of32, n = 32 j + 8 (e / 4) + 4 half + e % 4.
  const bool fours = ends_in_fours(a);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const uint32_t m = m0 + wm + i * 32 + of32, n = n0 + wn + j * 32 + e * 2 + half * 4;
        if (m >= a.m || n >= a.n) continue;
        float v[4] = {acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        if (fours && n + 4 <= a.n) {
          finish<4>(a, w, m, n, v);
        } else {
#pragma unroll 1
          for (uint32_t c = 0; c < 4 && n + c < a.n; ++c) {
            float one = c == 0 ? v[0] : (c == 1 ? v[1] : (c == 2 ? v[2] : v[3]));
            finish<1>(a, w, m, n + c, &one);
          }
        }
      }
}

// ---------------------------------------------------------------------------
// dz and its sums over the tokens
// ---------------------------------------------------------------------------

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

int launch_product(const ProductArgs& args, void* stream) {
  if (args.m == 0 || args.n == 0) return 0;
  const dim3 grid((args.m + kTile - 1) / kTile * ((args.n + kTile - 1) / kTile), args.W);
  auto with_layout = [&](auto ta, auto tb, auto pa, auto pb) {
    typedef decltype(ta) TA;
    typedef decltype(tb) TB;
    constexpr int PA = decltype(pa)::value, PB = decltype(pb)::value;
    if (args.a.along_k) {
      return args.b.along_k ? enqueue(product_any<TA, TB, true, true, PA, PB>, grid, 256, 0, stream, args)
                            : enqueue(product_any<TA, TB, true, false, PA, PB>, grid, 256, 0, stream, args);
    }
    return enqueue(product_any<TA, TB, false, false, PA, PB>, grid, 256, 0, stream, args);
  };
  const uint16_t half = 0;
  const float whole = 0.f;
  const Number<1> one;
  const Number<3> three;
  if (args.a.bf16) {
    if (args.b.bf16) return with_layout(half, half, one, one);
    return args.out_bf16 ? with_layout(half, whole, one, one) : with_layout(half, whole, one, three);
  }
  if (args.b.bf16) return args.out_bf16 ? with_layout(whole, half, one, one) : with_layout(whole, half, three, one);
  return args.out_bf16 ? with_layout(whole, whole, one, one) : with_layout(whole, whole, three, three);
}

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
