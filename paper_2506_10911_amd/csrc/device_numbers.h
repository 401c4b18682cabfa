// What the kernels of layer norm, matrices and log probabilities share: launching, numbers as they are stored, sums over
// a wave.  Device code only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace noloco {
namespace {

template <typename T> struct same { typedef T type; };
template <typename... KArgs>
int enqueue(void (*kernel)(KArgs...), dim3 grid, uint32_t block, uint32_t lds, void* stream, typename same<KArgs>::type... args) {
  void* argv[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), argv, lds, static_cast<hipStream_t>(stream));
}

template <int N> struct Number { static constexpr int value = N; };
struct Yes { constexpr operator bool() const { return true; } };
struct No { constexpr operator bool() const { return false; } };

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ uint16_t narrow(float v) {   // to bf16, nearest, ties to even; NaN stays NaN
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// N neighbouring numbers as stored (float, or bf16 as uint16_t), in vectors of up to 16 bytes.
template <typename E, int N> struct Stored {
  static constexpr int kVector = N == 1 ? 1 : (sizeof(E) == 2 && N % 8 == 0 ? 8 : 4);
  static_assert(N % kVector == 0, "vectors");
  typedef E vector __attribute__((ext_vector_type(kVector)));
  __device__ __forceinline__ static void load(const E* p, float* v) { load<false>(p, v); }
  __device__ __forceinline__ static void store(E* p, const float* v) { store<false>(p, v); }
  // What nobody reads again soon: past the caches that others fill.
  __device__ __forceinline__ static void load_once(const E* p, float* v) { load<true>(p, v); }
  __device__ __forceinline__ static void store_once(E* p, const float* v) { store<true>(p, v); }
  template <bool ONCE> __device__ __forceinline__ static void load(const E* p, float* v) {
#pragma unroll
    for (int i = 0; i < N; i += kVector) {
      E raw[kVector];
      if constexpr (kVector == 1) {
        raw[0] = *p;
      } else {
        const vector* const from = reinterpret_cast<const vector*>(p + i);
        const vector x = ONCE ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
        for (int k = 0; k < kVector; ++k) raw[k] = x[k];
      }
#pragma unroll
      for (int k = 0; k < kVector; ++k) {
        if constexpr (sizeof(E) == 2) v[i + k] = widen(raw[k]); else v[i + k] = raw[k];
      }
    }
  }
  template <bool ONCE> __device__ __forceinline__ static void store(E* p, const float* v) {
#pragma unroll
    for (int i = 0; i < N; i += kVector) {
      E raw[kVector];
#pragma unroll
      for (int k = 0; k < kVector; ++k) {
        if constexpr (sizeof(E) == 2) raw[k] = narrow(v[i + k]); else raw[k] = v[i + k];
      }
      if constexpr (kVector == 1) {
        *p = raw[0];
      } else {
        vector x;
#pragma unroll
        for (int k = 0; k < kVector; ++k) x[k] = raw[k];
        vector* const to = reinterpret_cast<vector*>(p + i);
        if constexpr (ONCE) __builtin_nontemporal_store(x, to); else *to = x;
      }
    }
  }
};

// The same where the type is known at run time only (a branch of the whole wave).
template <int N> __device__ __forceinline__ void load_numbers(const void* p, int64_t at, bool bf16, float* v) {
  if (bf16) Stored<uint16_t, N>::load(static_cast<const uint16_t*>(p) + at, v);
  else Stored<float, N>::load(static_cast<const float*>(p) + at, v);
}
template <int N> __device__ __forceinline__ void store_numbers(void* p, int64_t at, bool bf16, const float* v) {
  if (bf16) Stored<uint16_t, N>::store(static_cast<uint16_t*>(p) + at, v);
  else Stored<float, N>::store(static_cast<float*>(p) + at, v);
}

// Sums and largest numbers over the lanes of a wave, the same in all of them: within sixteen lanes by moves between lanes (pairs,
// fours, eights mirrored, sixteens mirrored), then over the four sixteens.  Through the LDS (__shfl_xor) a sum is six round trips.
template <int CONTROL> __device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, 15, 15, true));
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ float wave_sum(float v) {
  v += moved<0xB1>(v);
  v += moved<0x4E>(v);
  v += moved<0x141>(v);
  v += moved<0x140>(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ float wave_largest(float v) {
  v = fmaxf(v, moved<0xB1>(v));
  v = fmaxf(v, moved<0x4E>(v));
  v = fmaxf(v, moved<0x141>(v));
  v = fmaxf(v, moved<0x140>(v));
  return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}

// v[0], v[1] summed over the workgroup's L threads (a wave, or whole waves: then `shared` has 2 * L / 64 floats and is free
// again behind the next barrier that all threads pass).
template <int L, int COUNT> __device__ __forceinline__ void sum_all(float* v, float* shared) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) v[i] = wave_sum(v[i]);
  if constexpr (L > 64) {
    constexpr int kWaves = L / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i) shared[(threadIdx.x >> 6) * COUNT + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v[i] += shared[w * COUNT + i];
    }
  }
}

}  // namespace
}  // namespace noloco
