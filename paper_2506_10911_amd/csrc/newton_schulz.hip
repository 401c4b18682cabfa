// Newton-Schulz orthogonalisation of many matrices at once (kernels and their launchers).
//
// X_0 = U / (|U|_F + eps), transposed if U is tall, so that X is m x n with m <= n; a step is
//   A = X X^T          m x m, symmetric
//   P = a + b A + c A^2   m x m, symmetric
//   X <- P X
// which takes every singular value s of X to s (a + b s^2 + c s^4).  All three are matrix products with both
// operands in binary16 and sums in binary32.  |X_0| <= 1 and the polynomial keeps X small, so binary16's range is
// enough and its eleven bits beat bf16's eight at the same rate.  One binary16 a number is exact enough for bf16
// results (a few 2^-12 of the result's norm); for float results a number is a pair of binary16, high and low half, of
// which three products are taken (high high, high low, low high): 22 bits.
//
// With one binary16 a number the diagonals of A and P keep what it leaves of them, and the next product adds it: where n is much
// more than m all singular values are alike and A is nearly its diagonal, so that its rounding is a relative error of every
// singular value, and some steps' polynomials have slopes of ten there (without it 32 x 512 is 0.003 of the norm off and
// 4 x 1024 0.006, with it 0.0007; square ones 0.0012 and 0.0009).
//
// A and P are symmetric: only tiles on and below the diagonal are computed, each written to both its places.
// X stays row-major throughout: X X^T reads rows along their length, and P X reads X through the LDS's
// transposing reads, so that no transposed copy of X is ever stored.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "inner_internal.h"

namespace noloco {
namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

#define lds_memory __attribute__((address_space(3)))

// 16 bytes a lane from a buffer to the LDS, at `to` + 16 times the lane, past the registers.  The compiler does not count
// these loads (it would wait for all of them in front of every transposing read): who reads what they bring waits for
// vmcnt itself.  m0 is a register that the compiler keeps nothing in and that a clobber list may not name; its own
// instructions that read it, each behind a write of its own, are none in these kernels.
__device__ __forceinline__ uint4v buffer_words(const void* p, uint32_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  auto same = [](uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v))); };
  return uint4v{same(static_cast<uint32_t>(at)), same(static_cast<uint32_t>(at >> 32) & 0xffffu), same(bytes), 0x00020000u};
}
__device__ __forceinline__ void load_to_lds(uint4v buffer, uint32_t lane_offset, uint32_t offset, uint32_t to) {
  offset = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(offset)));
  to = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(to)));
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
               :: "v"(lane_offset), "s"(buffer), "s"(offset), "s"(to) : "memory");
}

// Enqueue a kernel and return the launch status itself.
template <typename T> struct same { typedef T type; };
template <typename... KArgs>
int enqueue_with(uint32_t lds, void (*kernel)(KArgs...), dim3 grid, uint32_t block, void* stream, typename same<KArgs>::type... args) {
  void* argv[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), argv, lds, static_cast<hipStream_t>(stream));
}
template <typename... KArgs>
int enqueue(void (*kernel)(KArgs...), uint32_t grid, uint32_t block, void* stream, typename same<KArgs>::type... args) {
  return enqueue_with(0, kernel, dim3(grid), block, stream, args...);
}

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ uint16_t narrow(float v) {   // to bf16, nearest, ties to even; NaN stays NaN
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// Tables that no kernel writes are read through the scalar cache.
#define scalar_memory __attribute__((address_space(4)))
__device__ __forceinline__ NsItem item_at(const NsArgs& args, uint32_t i) {
  const scalar_memory NsItem* p = (const scalar_memory NsItem*)args.items + i;
  return {p->offset, p->row_stride, p->scale, 0};
}

// Which class and item workgroup `group` works on, and which workgroup of the item it is.
struct Place { NsClass cls; uint32_t item, part; };
__device__ __forceinline__ Place locate(const NsArgs& args, uint32_t group) {
  Place p{args.first, 0, 0};
  uint32_t begin = 0;
  if (group >= args.first_end) {
    const scalar_memory NsTable* table = (const scalar_memory NsTable*)args.table;
    uint32_t cls = 0;
#pragma unroll
    for (int i = 0; i < kNsClasses - 1; ++i) {
      const uint32_t end = table->end[i];
      const bool past = end <= group;
      cls += past ? 1u : 0u;
      begin = past ? end : begin;
    }
    const scalar_memory NsClass* c = table->cls + cls;
    p.cls = {c->base, c->item_bytes, c->per_item, c->first_item, c->first_sum, c->m, c->n, c->mp, c->np, c->tall, c->splits, 0};
  }
  const uint32_t at = group - begin;
  p.item = at / p.cls.per_item;
  p.part = at - p.item * p.cls.per_item;
  return p;
}

struct Yes { constexpr operator bool() const { return true; } };
struct No { constexpr operator bool() const { return false; } };
template <int N> struct Number { static constexpr int value = N; };

// What is orthogonalised: x, the momentum, or the gradient that looks one step ahead.
__device__ __forceinline__ float direction(float g, float moved, float mu, bool nesterov) {
  return nesterov ? g + mu * moved : moved;
}

template <bool BF16> struct Stored { typedef float type; };
template <> struct Stored<true> { typedef uint16_t type; };

// N neighbouring numbers of type E (float, or bf16 as stored) as floats.
template <typename E, int N> struct Numbers {
  typedef E vector __attribute__((ext_vector_type(4)));
  float v[N];
  __device__ __forceinline__ void load(const E* p) {
    E raw[N];
    if constexpr (N == 4) {
      const vector x = *reinterpret_cast<const vector*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = x[i];
    } else {
      raw[0] = *p;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(E) == 2) v[i] = widen(raw[i]); else v[i] = raw[i];
    }
  }
  __device__ __forceinline__ void store(E* p) const {
    E raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(E) == 2) raw[i] = narrow(v[i]); else raw[i] = v[i];
    }
    if constexpr (N == 4) *reinterpret_cast<vector*>(p) = vector{raw[0], raw[1], raw[2], raw[3]};
    else *p = raw[0];
  }
};

// The result v of one element goes to where it belongs.
template <typename Out> __device__ __forceinline__ void put_result(const NsArrays& arrays, Out* at, float by, float v) {
  if (arrays.update) {
    float old;
    if constexpr (sizeof(Out) == 2) old = widen(*at); else old = *at;
    v = old * arrays.keep - by * v;
  }
  if constexpr (sizeof(Out) == 2) *at = narrow(v); else *at = v;
}

// ---------------------------------------------------------------------------
// Small matrices: everything in one workgroup
// ---------------------------------------------------------------------------

// X [mp][np], A and P [mp][mp] stay in the LDS from the first step to the last, rows 16 bytes longer than their numbers,
// so that 16 rows of a fragment begin in 16 different quarters of the banks.  Blocks of 32 x 32: those of A and P on and
// below the diagonal are dealt to the waves (of A with one or three blocks several waves share one's k); of P X a wave
// takes 32 columns of X, which nobody else reads, holds them in registers and writes their next values in their place.
//
// Numbers come and go in chunks of eight, a thread every 512th chunk: eight along X's row, 16 bytes of the LDS.  (Results of
// a tall matrix leave as four columns of two rows, since half a wave would write 128 bytes of a row only.)  They are read
// once: until the norm is known the LDS holds them as binary16 with a power of two for each chunk, or, where there is room
// for pairs, the two halves of a binary32 number in the places of high and low half.
//
// What bounds it: each workgroup waits for its own chain.  1152 matrices of 64 x 768 in binary16, float in and bf16 out, take
// 257 us (1.3 TB/s): four and a half rounds, in each of which all CUs load at once (14 us), then compute (six to seven us a
// step), then write.  The matrix cores are busy 10 % of the cycles, the LDS 32 %.  A second workgroup a CU has no room while X
// is in the LDS; asking for the next matrix before the steps needs registers that are not there.  (X in registers, 48 a lane at
// 64 x 768, would leave room for two: not built.)  With launches for each product instead: 637 us.  24 matrices of
// 64 x 64 to 64 x 256 in pairs: 34 us, with launches 99.
template <int PLANES, bool BF16, bool MOMENTUM, typename Out>
__global__ __launch_bounds__(kNsSmallThreads) void ns_small(NsArgs args, NsArrays arrays, NsSteps steps) {
  extern __shared__ __align__(16) char lds[];
  constexpr uint32_t kThreads = kNsSmallThreads, kWaves = kThreads / 64;
  constexpr float kUnitGram = ns_unit_a(PLANES) / (ns_unit_x(PLANES) * ns_unit_x(PLANES));
  constexpr int kAhead = 4;
  typedef typename Stored<BF16>::type In;
  typedef uint16_t ushort8 __attribute__((ext_vector_type(8)));
  const uint32_t thread = threadIdx.x, lane = thread & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const Place place = locate(args, blockIdx.x);
  const NsItem item = item_at(args, place.cls.first_item + place.item);
  const uint32_t m = place.cls.m, n = place.cls.n, mp = (m + 31) / 32 * 32, np = (n + 31) / 32 * 32;
  const bool tall = place.cls.tall != 0;
  const uint32_t x_row = np * 2 * PLANES + 16, a_row = mp * 2 * PLANES + 16;
  double* const part = reinterpret_cast<double*>(lds);
  char* const x = lds + kNsSmallSums;
  char* const gram = x + mp * x_row;
  char* const poly = gram + mp * a_row;
  float* const shares = reinterpret_cast<float*>(poly + mp * a_row);
  auto spot = [](uint32_t j) { return PLANES == 1 ? j * 2 : (j / 32) * 128 + (j % 32) * 2; };   // of number j in a row

  // Chunk by chunk: where its first number is in X and in the matrix (the matrix's first for a chunk that is not there).
  // kWay: 0 eight along X's row, one by one; 1 the same in vectors, eight columns of a row; 2 four columns of two rows.
  const uint32_t along = (n + 7) / 8;
  const bool aligned = (static_cast<uint64_t>(item.offset) | static_cast<uint64_t>(item.row_stride)) % 4 == 0;
  const bool row_vectors = !tall && aligned && n % 8 == 0, tall_vectors = tall && aligned && m % 4 == 0 && n % 2 == 0;
  const int64_t apart = tall ? item.row_stride : 1;
  struct Spot { bool there; uint32_t i, j; int64_t at; };
  struct Walk { uint32_t all, divisor, up, over, chunk, high, low; };
  auto walk_of = [&](auto way) {
    Walk w;
    w.divisor = decltype(way)::value == 2 ? m / 4 : (tall ? m : along);
    w.all = decltype(way)::value == 2 ? m / 4 * (n / 2) : m * along;
    w.up = kThreads / w.divisor;
    w.over = kThreads - w.up * w.divisor;
    w.chunk = thread;
    w.high = thread / w.divisor;
    w.low = thread - w.high * w.divisor;
    return w;
  };
  auto next_chunk = [&](auto way, Walk& w) {
    Spot c;
    c.there = w.chunk < w.all;
    c.i = c.there ? (decltype(way)::value == 2 ? w.low * 4 : (tall ? w.low : w.high)) : 0;
    c.j = c.there ? (decltype(way)::value == 2 ? w.high * 2 : (tall ? w.high : w.low) * 8) : 0;
    c.at = item.offset + (tall ? c.j * item.row_stride + c.i : c.i * item.row_stride + c.j);
    w.chunk += kThreads;
    w.high += w.up;
    w.low += w.over;
    if (w.low >= w.divisor) { w.low -= w.divisor; ++w.high; }
    return c;
  };
  // Number e of a chunk from its first one on, in the matrix, and whether it is there; all eight of them in a plane of the LDS.
  auto offset_of = [&](auto way, int e) {
    return decltype(way)::value == 2 ? (e / 4) * apart + e % 4 : (decltype(way)::value == 1 ? e : e * apart);
  };
  auto real = [&](auto way, const Spot& c, int e) { return decltype(way)::value == 0 ? c.there && c.j + e < n : c.there; };
  auto put = [&](const Spot& c, int plane, ushort8 v) {
    if (c.there) *reinterpret_cast<ushort8*>(x + c.i * x_row + spot(c.j) + plane * 64) = v;
  };
  auto get = [&](auto way, const Spot& c, int plane) {
    const char* const from = x + c.i * x_row + spot(c.j) + plane * 64;
    ushort8 v;
    if constexpr (decltype(way)::value == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t two = *reinterpret_cast<const uint32_t*>(from + k * x_row);
        v[k] = static_cast<uint16_t>(two);
        v[4 + k] = static_cast<uint16_t>(two >> 16);
      }
    } else {
      v = *reinterpret_cast<const ushort8*>(from);
    }
    return v;
  };

  // Nobody's rows and eights of columns of X are zeros.
  for (uint32_t at = m * x_row + thread * 16; at < mp * x_row; at += kThreads * 16) *reinterpret_cast<uint4v*>(x + at) = uint4v{0, 0, 0, 0};
  for (uint32_t row = thread; row < m; row += kThreads)
    for (uint32_t j = along * 8; j < np; j += 8)
#pragma unroll
      for (int p = 0; p < PLANES; ++p) *reinterpret_cast<uint4v*>(x + row * x_row + spot(j) + p * 64) = uint4v{0, 0, 0, 0};

  // Momentum, the sum of squares, and the numbers to the LDS.  Four chunks are on their way while one is worked on.
  // A chunk's squares are summed with its power of two taken out: gradients are small enough for squares to leave
  // binary32's range.
  double sum = 0.;
  uint8_t* const powers = reinterpret_cast<uint8_t*>(gram);        // of the chunks, as long as there is no A
  const uint32_t all_chunks = m * along;
  auto load = [&](auto way) {
    constexpr int V = decltype(way)::value != 0 ? 4 : 1;
    Walk walk = walk_of(way);
    Spot c[kAhead];
    Numbers<In, V> g[kAhead][8 / V];
    Numbers<float, V> moved[kAhead][8 / V];
    auto ask = [&](int k) {
      c[k] = next_chunk(way, walk);
#pragma unroll
      for (int e = 0; e < 8; e += V) {
        const int64_t from = c[k].at + (real(way, c[k], e) ? offset_of(way, e) : 0);
        g[k][e / V].load(static_cast<const In*>(arrays.in) + from);
        if constexpr (MOMENTUM) moved[k][e / V].load(arrays.momentum + from);
      }
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ask(k);
#pragma unroll 1
    for (uint32_t done = 0; done < all_chunks; done += kAhead * kThreads) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (done + k * kThreads >= all_chunks) break;
      const Spot here = c[k];
      float u[8];
      int most = -127;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = g[k][e / V].v[e % V];
        if constexpr (MOMENTUM) {
          float& v = moved[k][e / V].v[e % V];
          v = arrays.mu * v + u[e];
          u[e] = direction(u[e], v, arrays.mu, arrays.nesterov != 0);
        }
        if (!real(way, here, e)) u[e] = 0.f;
        most = max(most, static_cast<int>(__float_as_uint(u[e]) >> 23 & 255) - 127);
      }
      if constexpr (MOMENTUM) {
#pragma unroll
        for (int e = 0; e < 8; e += V)
          if (real(way, here, e)) moved[k][e / V].store(arrays.momentum + here.at + offset_of(way, e));
      }
      if (done + (k + kAhead) * kThreads < all_chunks) ask(k);
      float squares = 0.f, scaled[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        scaled[e] = ldexpf(u[e], 14 - most);
        squares += scaled[e] * scaled[e];
      }
      sum += ldexp(static_cast<double>(squares), 2 * (most - 14));
      if constexpr (PLANES == 1) {
        if (here.there) powers[done + k * kThreads + thread] = static_cast<uint8_t>(most + 127);
        half8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = static_cast<_Float16>(scaled[e]);
        put(here, 0, __builtin_bit_cast(ushort8, h));
      } else {
        ushort8 high, low;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          high[e] = static_cast<uint16_t>(__float_as_uint(u[e]) >> 16);
          low[e] = static_cast<uint16_t>(__float_as_uint(u[e]));
        }
        put(here, 0, high);
        put(here, 1, low);
      }
    }
    }
  };
  if (row_vectors) load(Number<1>{}); else load(Number<0>{});
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_down(sum, d);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  double squares = 0.;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) squares += part[w];
  const double norm = sqrt(squares) + static_cast<double>(arrays.eps);
  float near;
  {
    // X_0 = u * ns_unit_x / norm, the factor as a number near 1 and a power of two, which float has room for whatever the norm.
    // A matrix of zeros stays one.  Single binary16 are rounded already, and so that X_0 is not rounded twice it stays without
    // the number near 1 (0.5 to 1), which the first step's polynomial takes in.
    int power = 0;
    near = norm == 0. ? 0.f : static_cast<float>(frexp(static_cast<double>(ns_unit_x(PLANES)) / norm, &power));
    if (!(norm <= 1.7976931348623157e308)) near = __builtin_nanf("");
    const Number<0> way;           // in the LDS both ways are the same
    Walk walk = walk_of(way);
#pragma unroll 2
    for (uint32_t done = 0; done < all_chunks; done += kThreads) {
      const Spot c = next_chunk(way, walk);
      half8 high, low;
      if constexpr (PLANES == 1) {
        const int chunk_power = power + static_cast<int>(c.there ? powers[done + thread] : 0) - 127 - 14;
        const half8 h = __builtin_bit_cast(half8, get(way, c, 0));
#pragma unroll
        for (int e = 0; e < 8; ++e) high[e] = static_cast<_Float16>(ldexpf(static_cast<float>(h[e]), chunk_power));
      } else {
        const ushort8 hi = get(way, c, 0), lo = get(way, c, 1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = ldexpf(__uint_as_float(static_cast<uint32_t>(hi[e]) << 16 | lo[e]) * near, power);
          high[e] = static_cast<_Float16>(v);
          low[e] = static_cast<_Float16>(v - static_cast<float>(high[e]));
        }
        put(c, 1, __builtin_bit_cast(ushort8, low));
      }
      put(c, 0, __builtin_bit_cast(ushort8, high));
    }
  }
  __syncthreads();

  // fragments: row (or column) lane % 32, eight k from 8 (lane / 32) on
  const uint32_t of32 = lane & 31, half = lane >> 5;
  struct Fragment { half8 p[PLANES]; };
  auto plain = [&](const char* rows32, uint32_t row, uint32_t slice) {     // 16 k from 16 slice on of 32 rows
    Fragment f;
    const char* at = rows32 + of32 * row + (PLANES == 1 ? slice * 32 : (slice >> 1) * 128 + (slice & 1) * 32) + half * 16;
#pragma unroll
    for (int p = 0; p < PLANES; ++p) f.p[p] = *reinterpret_cast<const half8*>(at + p * 64);
    return f;
  };
  auto multiply = [](const Fragment& a, const Fragment& b, float16v d) {
    if constexpr (PLANES == 2) {
      d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[1], b.p[0], d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[0], b.p[1], d, 0, 0, 0);
    }
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[0], b.p[0], d, 0, 0, 0);
  };
  auto nothing = [] {
    float16v d;
#pragma unroll
    for (int e = 0; e < 16; ++e) d[e] = 0.f;
    return d;
  };
  // Of a block, d[e] is row 8 (e / 4) + 4 half + e % 4, column of32.  Four rows' numbers from `quad` = e / 4 on, written as part
  // of a row of the block's transpose, which begins at number j of `row`; and as they stand.
  auto write_four = [&](char* row, uint32_t j, uint32_t quad, float4v v) {
    const half4 high = __builtin_convertvector(v, half4);
    char* at = row + spot(j) + (quad * 8 + half * 4) * 2;
    *reinterpret_cast<half4*>(at) = high;
    if constexpr (PLANES == 2) *reinterpret_cast<half4*>(at + 64) = __builtin_convertvector(v - __builtin_convertvector(high, float4v), half4);
  };
  auto write_column = [&](char* block_rows, uint32_t row_bytes, uint32_t j, uint32_t quad, float4v v) {
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      char* at = block_rows + (quad * 8 + half * 4 + e) * row_bytes + spot(j);
      const _Float16 high = static_cast<_Float16>(v[e]);
      *reinterpret_cast<_Float16*>(at) = high;
      if constexpr (PLANES == 2) *reinterpret_cast<_Float16*>(at + 64) = static_cast<_Float16>(v[e] - static_cast<float>(high));
    }
  };
  auto four_of = [](const float16v& d, int quad) { return float4v{d[quad * 4], d[quad * 4 + 1], d[quad * 4 + 2], d[quad * 4 + 3]}; };

  const uint32_t blocks = mp / 32, pairs = blocks * (blocks + 1) / 2;
  auto below = [](uint32_t t, uint32_t& bi, uint32_t& bj) {     // block t on and below the diagonal, bj <= bi
    bi = 0;
    while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
    bj = t - bi * (bi + 1) / 2;
  };
  // Sum over slices [k, end) of block (bi, bj) of the product of a matrix with its transpose.
  auto block_product = [&](const char* matrix, uint32_t row_bytes, uint32_t bi, uint32_t bj, uint32_t k, uint32_t end) {
    float16v d = nothing();
    const char *r = matrix + bj * 32 * row_bytes, *c = matrix + bi * 32 * row_bytes;
    constexpr uint32_t kAtOnce = PLANES == 1 ? 4 : 2;
    if (bi == bj) {
      for (; k + kAtOnce <= end; k += kAtOnce) {
        Fragment a[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) a[i] = plain(r, row_bytes, k + i);
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) d = multiply(a[i], a[i], d);
      }
    } else {
      for (; k + kAtOnce <= end; k += kAtOnce) {
        Fragment a[kAtOnce], b[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
          a[i] = plain(r, row_bytes, k + i);
          b[i] = plain(c, row_bytes, k + i);
        }
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) d = multiply(a[i], b[i], d);
      }
    }
    for (; k < end; ++k) d = multiply(plain(r, row_bytes, k), plain(c, row_bytes, k), d);
    return d;
  };

  // The symmetric product of `from` with its transpose, block by block; result(bi, bj, quad, d) makes four of its numbers
  // what is written to both their places in `to`.  With one or three blocks of long rows all waves share their k, and then
  // their results.  What single binary16 leave of a number on the diagonal and the three beside
  // it goes into the row's last 16 bytes.
  auto rest = [&](const char* matrix, uint32_t row) { return reinterpret_cast<const float*>(matrix + row * a_row + mp * 2)[row & 3]; };
  auto symmetric = [&](const char* from, uint32_t row_bytes, uint32_t slices, char* to, bool share_k, auto result) {
    auto write = [&](uint32_t bi, uint32_t bj, uint32_t quad, float4v v) {
      write_four(to + (bi * 32 + of32) * a_row, bj * 32, quad, v);
      if (bi != bj) write_column(to + bj * 32 * a_row, a_row, bi * 32 + of32, quad, v);
      else if constexpr (PLANES == 1) {
        uint32_t fours = of32 & ~3u;
        asm("" : "+v"(fours));            // compared here: masks kept from step to step do not fit the scalar registers
        if (quad * 8 + half * 4 == fours) {
          *reinterpret_cast<float4v*>(to + (bi * 32 + of32) * a_row + mp * 2) = v - __builtin_convertvector(__builtin_convertvector(v, half4), float4v);
        }
      }
    };
    if (share_k) {
      // four waves take the block that has two operands to read, two each of the others
      const uint32_t sharing = blocks == 1 ? kWaves : (wave < 4 ? 4 : 2), share = blocks == 1 ? wave : (wave < 4 ? wave : wave & 1);
      const uint32_t bi = blocks == 1 || wave / 2 == 2 ? 0 : 1, bj = blocks == 1 || wave < 6 ? 0 : 1;
      const float16v d = block_product(from, row_bytes, bi, bj, slices * share / sharing, slices * (share + 1) / sharing);
#pragma unroll
      for (int quad = 0; quad < 4; ++quad) *reinterpret_cast<float4v*>(shares + ((wave * 4 + quad) * 64 + lane) * 4) = four_of(d, quad);
      __syncthreads();
      for (uint32_t t = wave; t < pairs * 4; t += kWaves) {
        const uint32_t block = t / 4, quad = t % 4;                  // blocks (1, 0), (0, 0), (1, 1), or (0, 0) alone
        const uint32_t first = blocks == 1 ? 0 : (block == 0 ? 0 : 2 + block * 2), count = blocks == 1 ? kWaves : (block == 0 ? 4 : 2);
        float4v sum = *reinterpret_cast<const float4v*>(shares + ((first * 4 + quad) * 64 + lane) * 4);
        for (uint32_t other = 1; other < count; ++other) sum += *reinterpret_cast<const float4v*>(shares + (((first + other) * 4 + quad) * 64 + lane) * 4);
        const uint32_t ri = blocks == 1 || block == 1 ? 0 : 1, rj = block == 2 ? 1 : 0;
        write(ri, rj, quad, result(ri, rj, quad, sum));
      }
    } else {
      for (uint32_t t = wave; t < pairs; t += kWaves) {
        uint32_t bi, bj;
        below(t, bi, bj);
        const float16v d = block_product(from, row_bytes, bi, bj, 0, slices);
        float4v v[4];                 // all of them, since a read does not overtake a write
#pragma unroll
        for (int quad = 0; quad < 4; ++quad) v[quad] = result(bi, bj, quad, four_of(d, quad));
#pragma unroll
        for (int quad = 0; quad < 4; ++quad) write(bi, bj, quad, v[quad]);
      }
    }
    __syncthreads();
  };

  for (int step = 0; step < steps.count; ++step) {
    // X_0 is `missing` times what the LDS holds, A its square times
    const float missing = PLANES == 1 && step == 0 ? near : 1.f;
    const float constant = steps.k[3 * step] * ns_unit_p(PLANES) * missing;
    const float linear = steps.k[3 * step + 1] * (ns_unit_p(PLANES) / ns_unit_a(PLANES)) * (missing * missing * missing);
    const float square = steps.k[3 * step + 2] * (ns_unit_p(PLANES) / (ns_unit_a(PLANES) * ns_unit_a(PLANES))) *
                         (missing * missing * missing * missing * missing);
    symmetric(x, x_row, np / 16, gram, blocks <= 2, [&](uint32_t, uint32_t, uint32_t, float4v d) { return d * kUnitGram; });
    symmetric(gram, a_row, mp / 16, poly, false, [&](uint32_t bi, uint32_t bj, uint32_t quad, float4v d) {
      const uint32_t row = bj * 32 + quad * 8 + half * 4, col = bi * 32 + of32;
      const char* at = gram + col * a_row + spot(bj * 32) + (quad * 8 + half * 4) * 2;
      float4v a = __builtin_convertvector(*reinterpret_cast<const half4*>(at), float4v);
      if constexpr (PLANES == 2) a += __builtin_convertvector(*reinterpret_cast<const half4*>(at + 64), float4v);
      float on_diagonal = constant;
      if constexpr (PLANES == 1) {      // A with its diagonal's rests R: A^2 + A R + R A, and A + R
        const float of_column = rest(gram, col);
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) d[e] += a[e] * (rest(gram, row + e) + of_column);
        on_diagonal += linear * of_column;
      }
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) d[e] = square * d[e] + linear * a[e] + (row + e == col ? on_diagonal : 0.f);
      return d;
    });
    // B = mp / 32 blocks of rows
    auto apply = [&](auto count) {
      constexpr int B = decltype(count)::value, S = 2 * B;
      constexpr bool kKept = B * S * PLANES <= 16;         // P stays in registers for all columns
      Fragment q[kKept ? B : 1][S];
      if constexpr (kKept) {
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
          for (int k = 0; k < S; ++k) q[b][k] = plain(poly + b * 32 * a_row, a_row, k);
      }
      for (uint32_t j0 = wave * 32; j0 < np; j0 += kWaves * 32) {
        Fragment f[S];
#pragma unroll
        for (int k = 0; k < S; ++k) {
          const char* at = x + (k * 16 + half * 8 + ((lane >> 2) & 3)) * x_row + spot(j0) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
          for (int p = 0; p < PLANES; ++p) {
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(at + p * 64));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(at + p * 64 + 4 * x_row));
            const half4 l = __builtin_bit_cast(half4, lo), h = __builtin_bit_cast(half4, hi);
            f[k].p[p] = __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
          }
        }
        constexpr int kRows = B < 2 ? B : 2;                // blocks of rows side by side
#pragma unroll
        for (int b0 = 0; b0 < B; b0 += kRows) {
          float16v d[kRows];
#pragma unroll
          for (int b = 0; b < kRows; ++b) d[b] = nothing();
          half4 before[kRows][4];             // what X is, and of P's diagonal the rests
          float left[kRows];
          if constexpr (PLANES == 1) {
#pragma unroll
            for (int b = 0; b < kRows; ++b) {
              if (b0 + b >= B) continue;
              left[b] = rest(poly, (b0 + b) * 32 + of32);
#pragma unroll
              for (int quad = 0; quad < 4; ++quad)
                before[b][quad] = *reinterpret_cast<const half4*>(x + ((b0 + b) * 32 + of32) * x_row + spot(j0) + (quad * 8 + half * 4) * 2);
            }
          }
#pragma unroll
          for (int k = 0; k < S; ++k)
#pragma unroll
            for (int b = 0; b < kRows; ++b)
              if (b0 + b < B) d[b] = multiply(f[k], kKept ? q[kKept ? b0 + b : 0][k] : plain(poly + (b0 + b) * 32 * a_row, a_row, k), d[b]);
#pragma unroll
          for (int b = 0; b < kRows; ++b)
            if (b0 + b < B) {
              char* const row = x + ((b0 + b) * 32 + of32) * x_row;
#pragma unroll
              for (int quad = 0; quad < 4; ++quad) {
                float4v v = four_of(d[b], quad);
                if constexpr (PLANES == 1) v += __builtin_convertvector(before[b][quad], float4v) * left[b];
                write_four(row, j0, quad, v * (1.f / ns_unit_p(PLANES)));
              }
            }
        }
      }
    };
    if (blocks == 1) apply(Number<1>{});
    else if (blocks == 2) apply(Number<2>{});
    else if (blocks == 3) apply(Number<3>{});
    else apply(Number<4>{});
    __syncthreads();
  }

  auto finish = [&](auto way) {
    constexpr int V = decltype(way)::value != 0 ? 4 : 1;
    typedef Out out4 __attribute__((ext_vector_type(4)));
    const float by = arrays.lr * item.scale;
    Walk walk = walk_of(way);
#pragma unroll 1
    for (uint32_t done = 0; done < walk.all; done += kAhead * kThreads) {
      Spot c[kAhead];
      Numbers<Out, V> old[kAhead][8 / V];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        c[k] = next_chunk(way, walk);
        if (arrays.update) {
#pragma unroll
          for (int e = 0; e < 8; e += V)
            old[k][e / V].load(static_cast<const Out*>(arrays.out) + c[k].at + (real(way, c[k], e) ? offset_of(way, e) : 0));
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const half8 high = __builtin_bit_cast(half8, get(way, c[k], 0));
        half8 low;
        if constexpr (PLANES == 2) low = __builtin_bit_cast(half8, get(way, c[k], 1));
        Out v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float value = static_cast<float>(high[e]);
          if constexpr (PLANES == 2) value += static_cast<float>(low[e]);
          value *= 1.f / ns_unit_x(PLANES);
          if (arrays.update) value = old[k][e / V].v[e % V] * arrays.keep - by * value;
          if constexpr (sizeof(Out) == 2) v[e] = narrow(value); else v[e] = value;
        }
        Out* const out = static_cast<Out*>(arrays.out) + c[k].at;
#pragma unroll
        for (int e = 0; e < 8; e += V) {
          if (!real(way, c[k], e)) continue;
          if constexpr (V == 4) *reinterpret_cast<out4*>(out + offset_of(way, e)) = out4{v[e], v[e + 1], v[e + 2], v[e + 3]};
          else out[offset_of(way, e)] = v[e];
        }
      }
    }
  };
  if (row_vectors) finish(Number<1>{});
  else if (tall_vectors) finish(Number<2>{});
  else finish(Number<0>{});
}

// ---------------------------------------------------------------------------
// Momentum, and the sum of squares of what is orthogonalised
// ---------------------------------------------------------------------------

// One workgroup sums one chunk of an item: numbers part * size .. of the matrix in row-major order, V at a time where
// rows are whole vectors, and four (V = 1: eight) of a thread's on their way together.  Squares are summed in binary64: gradients
// are small enough for their squares to leave binary32's range.  Bound by memory: 170M numbers, float, 12 bytes each, 381 us,
// 5.3 TB/s (a copy reaches 5.9).
template <bool BF16, bool MOMENTUM, int V>
__device__ __forceinline__ double sum_chunk(const NsArrays& arrays, const NsClass& cls, const NsItem& item, uint32_t part) {
  constexpr int kAtOnce = V == 4 ? 4 : 8;
  typedef typename Stored<BF16>::type In;
  const uint32_t cols = cls.tall ? cls.m : cls.n;
  const uint64_t total = uint64_t(cls.m) * cls.n;
  const uint64_t size = ((total + cls.per_item - 1) / cls.per_item + V - 1) / V * V;
  const uint64_t begin = part * size, end = begin + size < total ? begin + size : total;
  uint64_t e = begin + threadIdx.x * V;
  uint64_t row = e / cols, col = e - row * cols;
  const uint32_t step_rows = 256 * V / cols, step_cols = 256 * V - step_rows * cols;
  double sum = 0.;
  while (e < end) {
    int64_t at[kAtOnce];
    Numbers<In, V> g[kAtOnce];
    Numbers<float, V> moved[kAtOnce];
    const uint64_t first = e;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      at[k] = item.offset + (e < end ? static_cast<int64_t>(row) * item.row_stride + static_cast<int64_t>(col) : 0);
      g[k].load(static_cast<const In*>(arrays.in) + at[k]);
      if constexpr (MOMENTUM) moved[k].load(arrays.momentum + at[k]);
      e += 256 * V;
      row += step_rows;
      col += step_cols;
      if (col >= cols) { col -= cols; ++row; }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const bool there = first + k * 256 * V < end;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float u = g[k].v[i];
        if constexpr (MOMENTUM) {
          moved[k].v[i] = arrays.mu * moved[k].v[i] + u;
          u = direction(u, moved[k].v[i], arrays.mu, arrays.nesterov != 0);
        }
        sum += there ? static_cast<double>(u) * u : 0.;
      }
      if constexpr (MOMENTUM)
        if (there) moved[k].store(arrays.momentum + at[k]);
    }
  }
  return sum;
}

// Whether four neighbouring numbers of a row are one vector, wherever they begin at a multiple of four.
__device__ __forceinline__ bool whole_vectors(const NsItem& item, uint32_t cols) {
  return (static_cast<uint64_t>(item.offset) | static_cast<uint64_t>(item.row_stride) | cols) % 4 == 0;
}

template <bool BF16, bool MOMENTUM>
__global__ __launch_bounds__(256) void ns_sums(NsArgs args, NsArrays arrays) {
  const Place place = locate(args, blockIdx.x);
  const NsItem item = item_at(args, place.cls.first_item + place.item);
  double sum = whole_vectors(item, place.cls.tall ? place.cls.m : place.cls.n)
                   ? sum_chunk<BF16, MOMENTUM, 4>(arrays, place.cls, item, place.part)
                   : sum_chunk<BF16, MOMENTUM, 1>(arrays, place.cls, item, place.part);
  __shared__ double part[4];
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_down(sum, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0)
    args.sums[uint64_t(place.cls.first_sum + place.item) * kNsChunks + place.part] = part[0] + part[1] + part[2] + part[3];
}

// ---------------------------------------------------------------------------
// X_0
// ---------------------------------------------------------------------------

// workgroups of an item in ns_sums; the same on the host
__host__ __device__ inline uint32_t chunks_of(uint64_t elements) {
  const uint64_t c = (elements + kNsChunkElems - 1) / kNsChunkElems;
  return c < 1 ? 1 : (c > kNsChunks ? kNsChunks : static_cast<uint32_t>(c));
}

// A workgroup writes a 64 x 64 tile of X_0, zeros where it is padded; tall matrices are turned in the LDS.  Each adds up the
// item's partial sums itself, which costs less than a launch for it.  Bound by memory: the momentum (and gradient) is read again,
// since a matrix's norm is known only after all of it: 170M numbers, 12 bytes each, 418 us, 4.9 TB/s.
template <bool BF16, bool MOMENTUM, int PLANES>
__global__ __launch_bounds__(256) void ns_start(NsArgs args, NsArrays arrays) {
  __shared__ __align__(16) float tile[64][68];
  __shared__ double part[4];
  typedef typename Stored<BF16>::type In;
  const Place place = locate(args, blockIdx.x);
  const NsClass& cls = place.cls;
  const NsItem item = item_at(args, cls.first_item + place.item);
  const uint32_t chunks = chunks_of(uint64_t(cls.m) * cls.n);
  double sum = threadIdx.x < chunks ? args.sums[uint64_t(cls.first_sum + place.item) * kNsChunks + threadIdx.x] : 0.;

  const uint32_t across = cls.np / 64;
  const uint32_t i0 = place.part / across * 64, j0 = place.part % across * 64;     // of X
  const bool tall = cls.tall != 0;
  const uint32_t rows = tall ? cls.n : cls.m, cols = tall ? cls.m : cls.n;
  const uint32_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;                         // of the matrix
  auto fetch = [&](auto vectors) {
    constexpr int V = vectors ? 4 : 1, N = 16 / V;
    const uint32_t c = threadIdx.x % (64 / V) * V, r_first = threadIdx.x / (64 / V);
    Numbers<In, V> g[N];
    Numbers<float, V> moved[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t r = r_first + k * (4 * V);
      const int64_t at = item.offset + (r0 + r < rows && c0 + c < cols ? static_cast<int64_t>(r0 + r) * item.row_stride + c0 + c : 0);
      if (!MOMENTUM || arrays.nesterov) g[k].load(static_cast<const In*>(arrays.in) + at);
      if constexpr (MOMENTUM) moved[k].load(arrays.momentum + at);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t r = r_first + k * (4 * V);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float u;
        if constexpr (MOMENTUM) u = arrays.nesterov ? direction(g[k].v[i], moved[k].v[i], arrays.mu, true) : moved[k].v[i];
        else u = g[k].v[i];
        if (r0 + r >= rows || c0 + c >= cols) u = 0.f;
        if (tall) tile[c + i][r] = u; else tile[r][c + i] = u;
      }
    }
  };
  if (whole_vectors(item, cols)) fetch(Yes{}); else fetch(No{});
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_down(sum, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  const double norm = sqrt(part[0] + part[1] + part[2] + part[3]) + static_cast<double>(arrays.eps);
  // The factor as a number near 1 and a power of two, which float has room for whatever the norm.  A matrix of zeros stays one.
  int power = 0;
  const float near = norm == 0. ? 0.f : static_cast<float>(frexp(static_cast<double>(ns_unit_x(PLANES)) / norm, &power));
  char* x = args.workspace + cls.base + place.item * cls.item_bytes;
  const uint64_t ld = uint64_t(cls.np) * 2 * PLANES;
  // eight numbers of a row a thread: two rounds
  for (uint32_t v = threadIdx.x; v < 64 * 8; v += 256) {
    const uint32_t r = v >> 3, c = (v & 7) * 8;
    half8 high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = ldexpf(tile[r][c + e] * near, power);
      high[e] = static_cast<_Float16>(f);
      low[e] = static_cast<_Float16>(f - static_cast<float>(high[e]));
    }
    const uint32_t j = j0 + c;
    char* at = x + (i0 + r) * ld + (PLANES == 1 ? j * 2 : (j / 32) * 128 + (j % 32) * 2);
    *reinterpret_cast<half8*>(at) = high;
    if constexpr (PLANES == 2) *reinterpret_cast<half8*>(at + 64) = low;
  }
}

// ---------------------------------------------------------------------------
// The products
// ---------------------------------------------------------------------------

// Workgroups are dealt to the 8 XCDs in turn; each XCD takes runs of `run` consecutive tiles, which share rows and
// columns in its L2: 32 of 256, one round of its CUs, 64 of the smaller ones, of which two share a CU.
__device__ __forceinline__ uint32_t tile_of_block(uint32_t block, uint32_t blocks, uint32_t run) {
  const uint32_t whole = blocks / (8 * run) * (8 * run);
  if (block >= whole) return block;
  const uint32_t xcd = block & 7u, slot = block >> 3, k = slot / run;
  return (k * 8 + xcd) * run + (slot - k * run);
}

// D[r][c] = sum over k of F[r][k] S[c][k], a T x T tile of it.  For A and P F and S are rows of X or A; for P X
// the second operand is rows of P and the first is columns of X, whose rows lie in the LDS as in memory and are
// turned by the LDS's transposing reads.  With pairs a row holds 32 high halves, their 32 low halves, the next 32 high
// ones and so on, so that a stage of 128 bytes of every row is 64 numbers, or 32 pairs.
//
// A wave owns a (T / WR) x (T / WC) part in 32 x 32 blocks.  The operands come to the LDS by loads that bypass the
// registers, two stages deep (tiles of 64, which are taken where there are few, four: two of them share a CU; with eight
// stages and a CU to itself P X of two 768 x 768 matrices took 10.0 us, so 7.0).  Fragments are read one slice of 16 k ahead
// of the products that use them, across the stage's end too: the barrier in front of the last slice's products tells that
// the next stage has come and that this one's buffer is free.
//
// What bounds it: in tiles of 256 the clock, which falls to 1.63 to 1.75 of 2.4 GHz under these products, and the stages' way to
// the LDS: the matrix cores are busy 68 % of that clock's cycles in P X of 4096 x 4096 to 4096 x 16384, 60 % at 2048, 48 to 54 %
// in the symmetric products.  (Stages of half the depth, four to five of them, were 2 to 10 % slower.)  P X at 4096 1165
// TFLOP/s, at 2048 1043, X X^T 916 and 838, A^2 923 and 794, symmetric ones counted by half; a large library product 1220 to
// 1480.  In pairs (768 x 768 to 768 x 3072, tiles of 128) 905, 808 and 627, three products a number counted, with the matrix cores
// busy 53, 56 and 40 % at 1.66 to 1.8 GHz: two stages of 32 KiB bring too little work for each of their waits.  A symmetric
// product ends with both its images, from registers the one and through the LDS the other, the last P X with the update of theta
// in the same way (2048 wide, bf16: 2205 us beside 1581 of the other P X).
//
// Rows of 128 bytes: 16-byte chunk q of row r lies at q ^ (r >> 1 & 7), so that the 16 lanes that read at once meet
// 16 different quarters of the 64 banks.  Rows of X in the transposed operand: chunk q of row k at q ^ (k & 3) << 2
// (shorter rows: q ^ (k >> 1 & 1) << 2), since four lanes of a group of 16 read each of four rows.
template <int T, int WR, int WC, int KIND, int PLANES, typename Out>
__global__ __launch_bounds__(WR * WC * 64) void ns_product(NsArgs args, NsArrays arrays, int32_t step, float ca, float cb, float cc, uint32_t run) {
  constexpr bool kApplies = KIND == kNsApply || KIND == kNsLast, kSplits = KIND == kNsGram && T == kNsSplitTile;
  constexpr int kWaves = WR * WC, kThreads = kWaves * 64;
  constexpr int kDepth = 64 / PLANES;                       // k of a stage
  constexpr int kSlices = kDepth / 16;
  constexpr int kOperand = T * 128;                         // bytes of one operand's stage
  constexpr int kStage = 2 * kOperand;
  constexpr int kStages = T == 64 ? 4 : 2;
  constexpr int MB = T / WR / 32, NB = T / WC / 32;         // a wave's blocks
  constexpr int kLoads = T / 8 / kWaves;                    // of 1 KiB, of a wave, operand and stage
  constexpr int kTurned = T * 2 * PLANES;                   // bytes of a row of the transposed operand
  constexpr int kTurnedRows = 1024 / kTurned > 0 ? 1024 / kTurned : 1;   // rows of one load
  constexpr int kHalf = T / 2;
  constexpr int kImageRow = T * 2 * PLANES + 16;            // staged results, bytes of a row
  constexpr int kImage = kHalf * kImageRow;
  constexpr int kFloatRow = (T + 4) * 4, kFloatTallRow = (kHalf + 4) * 4;
  constexpr int kFloats = kHalf * kFloatRow > T * kFloatTallRow ? kHalf * kFloatRow : T * kFloatTallRow;
  constexpr int kResult = KIND == kNsLast ? kFloats : kImage;
  constexpr bool kRests = PLANES == 1 && KIND != kNsGram;   // what is left of a diagonal is read
  constexpr int kRestAt = kStages * kStage > kResult ? kStages * kStage : (kResult + 1023) / 1024 * 1024;
  constexpr int kLds = kRestAt + (kRests ? (kApplies ? 1 : 2) * 1024 : 0);
  static_assert(kTurned <= 1024 && kLoads >= 1 && kLds <= 160 * 1024 && (kStages & (kStages - 1)) == 0, "tile");
  __shared__ __align__(1024) char lds[kLds];

  const Place place = locate(args, tile_of_block(blockIdx.x, gridDim.x, run));
  const NsClass& cls = place.cls;
  const uint32_t mp = cls.mp, np = cls.np;
  const uint64_t x_bytes = uint64_t(mp) * np * 2 * PLANES, a_bytes = uint64_t(mp) * mp * 2 * PLANES;
  char* const buffers = args.workspace + cls.base + place.item * cls.item_bytes;
  char* const x = buffers + (step & 1 ? x_bytes : 0);
  char* const x_next = buffers + (step & 1 ? 0 : x_bytes);
  char* const gram = buffers + 2 * x_bytes;
  char* const poly = gram + a_bytes;
  float* const gram_rest = reinterpret_cast<float*>(poly + a_bytes);
  float* const poly_rest = gram_rest + mp;

  // Tile (r0, c0) of the result, and where it is found in the operands.
  uint32_t r0, c0;
  if constexpr (kApplies) {
    // columns of X by four tiles of rows of P
    const uint32_t tall_tiles = mp / T, wide_tiles = np / T, band = 4 * wide_tiles;
    const uint32_t g = place.part / band, in = place.part - g * band;
    const uint32_t high = tall_tiles - g * 4 < 4 ? tall_tiles - g * 4 : 4;
    r0 = in / high * T;
    c0 = (g * 4 + in % high) * T;
  } else {
    uint32_t row = static_cast<uint32_t>((sqrtf(8.f * place.part + 1.f) - 1.f) * 0.5f);
    if ((row + 1) * (row + 2) / 2 <= place.part) ++row;
    if (row * (row + 1) / 2 > place.part) --row;
    row = __builtin_amdgcn_readfirstlane(row);
    c0 = row * T;
    r0 = (place.part - row * (row + 1) / 2) * T;            // r0 <= c0
  }

  const uint32_t thread = threadIdx.x, lane = thread & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const uint32_t wr = wave / WC, wc = wave % WC;

  const char* const first = kApplies ? x : (KIND == kNsGram ? x : gram);
  const char* const second = kApplies ? poly : (KIND == kNsGram ? x : gram);
  const uint32_t first_ld = (KIND == kNsSquare ? mp : np) * 2 * PLANES, second_ld = (KIND == kNsGram ? np : mp) * 2 * PLANES;
  const uint32_t first_bytes = static_cast<uint32_t>(KIND == kNsSquare ? a_bytes : x_bytes);
  const uint32_t second_bytes = static_cast<uint32_t>(KIND == kNsGram ? x_bytes : a_bytes);
  const uint4v first_buffer = buffer_words(first, first_bytes), second_buffer = buffer_words(second, second_bytes);
  uint32_t stages = ((KIND == kNsGram ? cls.n : cls.m) + kDepth - 1) / kDepth, first_stage = 0;
  if constexpr (kSplits) {
    if (blockIdx.y >= cls.splits) return;
    first_stage = static_cast<uint32_t>(uint64_t(stages) * blockIdx.y / cls.splits);
    stages = static_cast<uint32_t>(uint64_t(stages) * (blockIdx.y + 1) / cls.splits) - first_stage;
  }

  // Where a lane's 16 bytes of a load come from.
  uint32_t plain_first[2], plain_second[2], turned[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t chunk = (lane & 7) ^ (((i << 2) | (lane >> 4)) & 7);
    plain_first[i] = (lane >> 3) * first_ld + chunk * 16 + first_stage * 128;
    plain_second[i] = (lane >> 3) * second_ld + chunk * 16 + first_stage * 128;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t in_row = lane * 16 % kTurned, row = lane * 16 / kTurned;
    const uint32_t k = i * kTurnedRows + row;
    const uint32_t turn = kTurned >= 256 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
    turned[i] = row * first_ld + ((in_row >> 4) ^ turn) * 16;
  }
  const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_memory char*)lds));
  auto ask = [&](uint32_t stage) {
    const uint32_t to = lds_at + (stage % kStages) * kStage;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t load = wave * kLoads + i;
      if constexpr (kApplies)
        load_to_lds(first_buffer, turned[i & 3], (stage * kDepth + load * kTurnedRows) * first_ld + r0 * 2 * PLANES, to + load * 1024);
      else
        load_to_lds(first_buffer, plain_first[(kLoads > 1 ? i : load) & 1], (r0 + load * 8) * first_ld + stage * 128, to + load * 1024);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t load = wave * kLoads + i;
      load_to_lds(second_buffer, plain_second[(kLoads > 1 ? i : load) & 1], (c0 + load * 8) * second_ld + stage * 128, to + kOperand + load * 1024);
    }
  };

  // Where a lane's fragments lie in a stage.
  const uint32_t fr = lane & 31, fk = lane >> 5;
  const uint32_t plain_r = (wr * (T / WR) + fr) * 128, plain_c = kOperand + (wc * (T / WC) + fr) * 128;
  uint32_t turned_at[4];
  {
    const uint32_t k = (lane >> 5) * 8 + ((lane >> 2) & 3), byte = (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    const uint32_t turn = kTurned >= 256 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t of_block = wr * (T / WR) * 2 * PLANES + i * 64 + byte;        // 64 bytes: 32 columns of one plane
      turned_at[i] = k * kTurned + (((of_block >> 4) ^ turn) << 4) + (of_block & 15);
    }
  }
  struct Fragments { half8 r[PLANES][MB], c[PLANES][NB]; };
  auto read = [&](uint32_t stage, int slice, Fragments& f) {
    const char* from = lds + (stage % kStages) * kStage;
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
      const uint32_t q = ((p * 4 + slice * 2 + fk) ^ ((fr >> 1) & 7)) * 16;
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        if constexpr (kApplies) {
          const int b = i * PLANES + p;                      // 64 bytes each
          const uint32_t at = turned_at[b & 3] + (b >> 2) * 256 + slice * 16 * kTurned;
          const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(from + at));
          const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(from + at + 4 * kTurned));
          const half4 l = __builtin_bit_cast(half4, lo), h = __builtin_bit_cast(half4, hi);
          f.r[p][i] = __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
          f.r[p][i] = *reinterpret_cast<const half8*>(from + plain_r + i * 4096 + q);
        }
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) f.c[p][j] = *reinterpret_cast<const half8*>(from + plain_c + j * 4096 + q);
    }
  };
  float16v acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  auto multiply = [&](const Fragments& f) {
    if constexpr (PLANES == 2) {
      // the small products first
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.r[1][i], f.c[0][j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.r[0][i], f.c[1][j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.r[0][i], f.c[0][j], acc[i][j], 0, 0, 0);
  };

  // What is left of the diagonal, of the tile's columns and, for A^2, its rows: in front of all else, so that it has come with it.
  if constexpr (kRests) {
    const float* const rests = kApplies ? poly_rest : gram_rest;
    if (wave == 0) load_to_lds(buffer_words(rests + c0, T * 4), lane * 16, 0, lds_at + kRestAt);
    if (!kApplies && wave == 1) load_to_lds(buffer_words(rests + r0, T * 4), lane * 16, 0, lds_at + kRestAt + 1024);
  }
  if (stages >= kStages) {
#pragma unroll
    for (int i = 0; i < kStages; ++i) ask(i);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * 2 * kLoads) : "memory");
  } else {
    for (uint32_t i = 0; i < stages; ++i) ask(i);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __builtin_amdgcn_s_barrier();
  Fragments even, odd;
  read(0, 0, even);
  // P with its diagonal's rests R is P X + R X: R, whose numbers binary16 has room for, goes through the products as a block of
  // its own where the stages hold the rows of X that are the tile's columns, 64 of them each.  (From memory, at the end, R X made P X
  // of 2048 x 8192 11 % longer, this 2.5.)
  constexpr bool kDiagonal = kRests && kApplies;
  const uint32_t diagonal = c0 / kDepth, diagonal_end = diagonal + T / kDepth;
  _Float16 left[NB];
  if constexpr (kDiagonal) {
#pragma unroll
    for (int j = 0; j < NB; ++j) left[j] = static_cast<_Float16>(*reinterpret_cast<const float*>(lds + kRestAt + (wc * (T / WC) + j * 32 + fr) * 4));
  }
  auto multiply_rests = [&](const Fragments& f, uint32_t piece, int slice) {
    static_assert(!kDiagonal || T / WC == 64 || (T == 64 && T / WC == 32), "a wave's columns are a stage's, or half of one's");
    if (T / WC == 64 ? piece != wc : static_cast<uint32_t>(slice >> 1) != wc) return;
    const int j = T / WC == 64 ? slice >> 1 : 0;
    const uint32_t mine = fr - (slice & 1) * 16 - fk * 8;        // where the lane's row has its column's number, if it has
    half8 d;
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) d[e] = e == mine ? left[j] : static_cast<_Float16>(0.f);
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.r[0][i], d, acc[i][j], 0, 0, 0);
  };
  // The stages behind the last one that is asked for by themselves, so that nothing in the loop is conditional.
  auto stage = [&](uint32_t s, auto ask_more, auto read_next, auto with_rests) {
#pragma unroll
    for (int slice = 0; slice < kSlices; ++slice) {
      Fragments& now = slice & 1 ? odd : even;
      Fragments& next = slice & 1 ? even : odd;
      if (slice + 1 < kSlices) {
        read(s, slice + 1, next);
      } else {
        // the next stage has come, those behind it may be on their way
        if constexpr (ask_more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * 2 * kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        if constexpr (read_next) read(s + 1, 0, next);
        if constexpr (ask_more) ask(s + kStages);
      }
      multiply(now);
      if constexpr (kDiagonal && with_rests)
        if (s >= diagonal && s < diagonal_end) multiply_rests(now, s - diagonal, slice);
      // the products of a slice stay behind its reads, which the compiler would put in front of the next barrier
      if constexpr (T == 256 && PLANES == 1) __builtin_amdgcn_sched_barrier(0);
    }
  };
  uint32_t s = 0;
  if constexpr (kDiagonal) {
    for (; s + kStages < stages && s < diagonal; ++s) stage(s, Yes{}, Yes{}, No{});
    for (; s + kStages < stages && s < diagonal_end; ++s) stage(s, Yes{}, Yes{}, Yes{});
  }
  for (; s + kStages < stages; ++s) stage(s, Yes{}, Yes{}, No{});
  for (; s + 1 < stages; ++s) stage(s, No{}, Yes{}, Yes{});
  stage(s, No{}, No{}, Yes{});

  if constexpr (kSplits) {
    if (cls.splits > 1) {       // a part, as the registers hold it
      float4v* part = reinterpret_cast<float4v*>(x_next + (uint64_t(blockIdx.y) * cls.per_item + place.part) * kNsSplitBytes);
#pragma unroll
      for (int quad = 0; quad < 4; ++quad)
        part[(wave * 4 + quad) * 64 + lane] = float4v{acc[0][0][quad * 4], acc[0][0][quad * 4 + 1], acc[0][0][quad * 4 + 2], acc[0][0][quad * 4 + 3]};
      return;
    }
  }

  // A wave's results go through the LDS, half of the tile's columns at a time, and from there in whole lines.
  // Block (i, j), element e of a lane: r = 32 i + 8 (e / 4) + 4 fk + e % 4, c = 32 j + fr.
  const uint32_t r_of = wr * (T / WR) + 4 * fk, c_of = (wc % (WC / 2)) * (T / WC) + fr;
  const uint32_t c_first = c0 + wc * (T / WC) + fr;
  if constexpr (KIND != kNsLast) {
    char* const to = KIND == kNsGram ? gram : (KIND == kNsSquare ? poly : x_next);
    const uint64_t to_ld = uint64_t(KIND == kNsApply ? np : mp) * 2 * PLANES;
    if constexpr (KIND == kNsSquare) {
      const float constant = ca * ns_unit_p(PLANES), linear = cb * (ns_unit_p(PLANES) / ns_unit_a(PLANES));
      const float square = cc * (ns_unit_p(PLANES) / (ns_unit_a(PLANES) * ns_unit_a(PLANES)));
      if constexpr (PLANES == 1) {
        // A's tile comes to the LDS, where nobody reads stages any more: rows of its transpose, which is itself, 16-byte chunk q of
        // row c at q ^ c.  With its diagonal's rests R it is A + R, and its square A^2 + A R + R A.
        constexpr int kRow = T * 2, kRows = 1024 / kRow;
        static_assert(T * kRow <= kStages * kStage, "tile of A");
#pragma unroll
        for (int i = 0; i < T / kRows / kWaves; ++i) {
          const uint32_t load = wave * (T / kRows / kWaves) + i, row = lane * 16 / kRow;
          const uint32_t chunk = (lane * 16 % kRow / 16) ^ ((load * kRows + row) & (kRow / 16 - 1));
          load_to_lds(first_buffer, row * first_ld + chunk * 16, (c0 + load * kRows) * first_ld + r0 * 2, lds_at + load * 1024);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        const float* const of_columns = reinterpret_cast<const float*>(lds + kRestAt);
        float of_column[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) of_column[j] = of_columns[wc * (T / WC) + j * 32 + fr];
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const uint32_t r = r_of + i * 32 + e * 2;
            const float4v of_row = *reinterpret_cast<const float4v*>(of_columns + 256 + r);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              const uint32_t c = wc * (T / WC) + j * 32 + fr;
              const float4v a = __builtin_convertvector(*reinterpret_cast<const half4*>(lds + c * kRow + (((r >> 3) ^ (c & (kRow / 16 - 1))) << 4) + fk * 8), float4v);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float v = acc[i][j][e + k] + a[k] * (of_row[k] + of_column[j]);
                acc[i][j][e + k] = square * v + linear * a[k];
              }
            }
          }
      } else {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const uint32_t r = r0 + r_of + i * 32 + e * 2, c = c_first + j * 32;
              // A is symmetric: its columns are read as rows, whose neighbouring numbers neighbouring lanes take
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const char* from = gram + (r + k) * to_ld + (c / 32) * 128 + (c % 32) * 2;
                float v = static_cast<float>(*reinterpret_cast<const _Float16*>(from));
                v += static_cast<float>(*reinterpret_cast<const _Float16*>(from + 64));
                acc[i][j][e + k] = square * acc[i][j][e + k] + linear * v + (r + k == c ? constant : 0.f);
              }
            }
      }
    }
    constexpr float kUnit = KIND == kNsGram ? ns_unit_a(PLANES) / (ns_unit_x(PLANES) * ns_unit_x(PLANES))
                                            : (KIND == kNsSquare ? 1.f : 1.f / ns_unit_p(PLANES));
    if constexpr (!kApplies && PLANES == 1) {
      // The diagonal: of a block on it, the lanes whose row is among their four hold one number each. A^2's is not whole yet, and
      // of both goes what a binary16 leaves to memory.
      if (r0 == c0) {
        const int mine = (fr >> 2 & 1) == fk ? static_cast<int>((fr >> 3) * 4 + (fr & 3)) : -1;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            if (wr * (T / WR) + i * 32 != wc * (T / WC) + j * 32) continue;
            const uint32_t c = wc * (T / WC) + j * 32 + fr;
            float more = 0.f, v = 0.f;
            if constexpr (KIND == kNsSquare)
              more = ca * ns_unit_p(PLANES) + cb * (ns_unit_p(PLANES) / ns_unit_a(PLANES)) * *reinterpret_cast<const float*>(lds + kRestAt + c * 4);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if constexpr (KIND == kNsSquare) acc[i][j][e] += e == mine ? more : 0.f;
              v = e == mine ? acc[i][j][e] * kUnit : v;
            }
            if (mine >= 0) (KIND == kNsGram ? gram_rest : poly_rest)[c0 + c] = v - static_cast<float>(static_cast<_Float16>(v));
          }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __syncthreads();
      if (wc / (WC / 2) == h) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const uint32_t r = r_of + i * 32 + e * 2;
              char* at = lds + (c_of + j * 32) * kImageRow + (PLANES == 1 ? r * 2 : (r / 32) * 128 + (r % 32) * 2);
              float4v v;
#pragma unroll
              for (int k = 0; k < 4; ++k) v[k] = acc[i][j][e + k] * kUnit;
              const half4 high = __builtin_convertvector(v, half4);
              *reinterpret_cast<half4*>(at) = high;
              if constexpr (PLANES == 2) *reinterpret_cast<half4*>(at + 64) = __builtin_convertvector(v - __builtin_convertvector(high, float4v), half4);
            }
      }
      __syncthreads();
      // rows of the result's transpose, as they lie
      constexpr int kChunks = T * 2 * PLANES / 16;
      for (uint32_t v = thread; v < kHalf * kChunks; v += kThreads) {
        const uint32_t row = v / kChunks, chunk = v % kChunks;
        const uint4v data = *reinterpret_cast<const uint4v*>(lds + row * kImageRow + chunk * 16);
        *reinterpret_cast<uint4v*>(to + uint64_t(c0 + h * kHalf + row) * to_ld + r0 * 2 * PLANES + chunk * 16) = data;
      }
      if constexpr (!kApplies) {
        // and the result itself, through the transposing reads: a wave takes 16 rows of 32 columns
        if (r0 != c0)
          for (uint32_t v = wave; v < (T / 16) * (kHalf / 32); v += kWaves) {
            const uint32_t rb = v / (kHalf / 32) * 16, cb32 = v % (kHalf / 32) * 32;
            const uint32_t c = cb32 + (lane >> 4) * 8 + ((lane >> 2) & 3);
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
              const uint32_t at = c * kImageRow + (PLANES == 1 ? rb * 2 : (rb / 32) * 128 + (rb % 32) * 2 + p * 64) + (lane & 3) * 8;
              const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(lds + at));
              const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(lds + at + 4 * kImageRow));
              const uint32_t row = r0 + rb + (lane & 15), col = c0 + h * kHalf + cb32 + (lane >> 4) * 8;
              char* out = to + row * to_ld + (PLANES == 1 ? col * 2 : (col / 32) * 128 + (col % 32) * 2 + p * 64);
              typedef short short8v __attribute__((ext_vector_type(8)));
              *reinterpret_cast<short8v*>(out) = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            }
          }
      }
    }
  } else {
    // r counts X's columns (the long side), c its rows.  A tall matrix has r as its row.
    const NsItem item = item_at(args, cls.first_item + place.item);
    const bool tall = cls.tall != 0;
    Out* const out = static_cast<Out*>(arrays.out) + item.offset;
    const bool vectors = ((reinterpret_cast<uintptr_t>(out) / sizeof(Out)) | static_cast<uint64_t>(item.row_stride)) % 4 == 0;
    const float by = arrays.lr * item.scale;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __syncthreads();
      if (wc / (WC / 2) == h) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const uint32_t r = r_of + i * 32 + e * 2, c = c_of + j * 32;
              float4v v;
#pragma unroll
              for (int k = 0; k < 4; ++k) v[k] = acc[i][j][e + k] * (1.f / (ns_unit_x(PLANES) * ns_unit_p(PLANES)));
              if (!tall) {
                *reinterpret_cast<float4v*>(lds + c * kFloatRow + r * 4) = v;
              } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) *reinterpret_cast<float*>(lds + (r + k) * kFloatTallRow + c * 4) = v[k];
              }
            }
      }
      __syncthreads();
      const uint32_t wide = tall ? kHalf : T, high = tall ? T : kHalf, lds_row = tall ? kFloatTallRow : kFloatRow;
      const uint32_t row0 = tall ? r0 : c0 + h * kHalf, col0 = tall ? c0 + h * kHalf : r0;
      const uint32_t rows = tall ? cls.n : cls.m, cols = tall ? cls.m : cls.n;
      // Eight vectors (numbers, where they are none) of a thread at a time, what was there asked for before the first is written.
      auto write = [&](auto four) {
        constexpr int V = four ? 4 : 1;
        for (uint32_t v0 = thread; v0 < high * (wide / V); v0 += 8 * kThreads) {
          Numbers<Out, V> old[8];
          Out* at[8];
          uint32_t r[8], c[8];
          int there[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t v = v0 + k * kThreads;
            r[k] = v / (wide / V);
            c[k] = v % (wide / V) * V;
            there[k] = v < high * (wide / V) && row0 + r[k] < rows ? static_cast<int>(cols) - static_cast<int>(col0 + c[k]) : 0;
            at[k] = out + (there[k] > 0 ? static_cast<int64_t>(row0 + r[k]) * item.row_stride + col0 + c[k] : 0);
            if (there[k] >= V && arrays.update) old[k].load(at[k]);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (there[k] <= 0) continue;
            const float* from = reinterpret_cast<const float*>(lds + r[k] * lds_row + c[k] * 4);
            if (there[k] >= V) {
              Numbers<Out, V> value;
#pragma unroll
              for (int i = 0; i < V; ++i) value.v[i] = arrays.update ? old[k].v[i] * arrays.keep - by * from[i] : from[i];
              value.store(at[k]);
            } else {
              for (int i = 0; i < there[k]; ++i) put_result(arrays, at[k] + i, by, from[i]);
            }
          }
        }
      };
      if (vectors) write(Yes{}); else write(No{});
    }
  }
}

// A from the parts that ns_product leaves of its tiles, in their order.  A workgroup adds a quarter of a tile: what one wave held.
// Bound by its launch and the reads' way: 3 to 5 us, of up to 64 parts.
template <int PLANES>
__global__ __launch_bounds__(256) void ns_join(NsArgs args, int32_t step) {
  const Place place = locate(args, blockIdx.x);
  const NsClass& cls = place.cls;
  if (cls.splits < 2) return;
  const uint64_t x_bytes = uint64_t(cls.mp) * cls.np * 2 * PLANES;
  char* const buffers = args.workspace + cls.base + place.item * cls.item_bytes;
  const char* const parts = buffers + (step & 1 ? 0 : x_bytes) + uint64_t(place.part) * kNsSplitBytes;
  char* const gram = buffers + 2 * x_bytes;
  uint32_t row = 0;
  while ((row + 1) * (row + 2) / 2 <= place.part) ++row;
  const uint32_t c0 = row * kNsSplitTile, r0 = (place.part - row * (row + 1) / 2) * kNsSplitTile;
  const uint32_t lane = threadIdx.x & 63, quad = threadIdx.x >> 6, wave = blockIdx.y;
  const uint64_t from = ((wave * 4 + quad) * 64 + lane) * sizeof(float4v), each = uint64_t(cls.per_item) * kNsSplitBytes;
  float4v sum = {0.f, 0.f, 0.f, 0.f};
  constexpr uint32_t kAhead = 8;
  uint32_t s = 0;
  for (; s + kAhead <= cls.splits; s += kAhead) {
    float4v v[kAhead];
#pragma unroll
    for (uint32_t k = 0; k < kAhead; ++k) v[k] = *reinterpret_cast<const float4v*>(parts + (s + k) * each + from);
#pragma unroll
    for (uint32_t k = 0; k < kAhead; ++k) sum += v[k];
  }
  for (; s < cls.splits; ++s) sum += *reinterpret_cast<const float4v*>(parts + s * each + from);
  sum *= ns_unit_a(PLANES) / (ns_unit_x(PLANES) * ns_unit_x(PLANES));
  const uint32_t r = r0 + wave / 2 * 32 + quad * 8 + (lane >> 5) * 4, c = c0 + wave % 2 * 32 + (lane & 31);
  const uint64_t ld = uint64_t(cls.mp) * 2 * PLANES;
  auto spot = [](uint32_t i) { return PLANES == 1 ? i * 2 : (i / 32) * 128 + (i % 32) * 2; };
  const half4 high = __builtin_convertvector(sum, half4);
  const float4v left = sum - __builtin_convertvector(high, float4v);
  const half4 low = __builtin_convertvector(left, half4);
  if constexpr (PLANES == 1) {
    float* const rests = reinterpret_cast<float*>(gram + 2 * ld * cls.mp);
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
      if (r + k == c) rests[c] = left[k];
  }
  *reinterpret_cast<half4*>(gram + c * ld + spot(r)) = high;
  if constexpr (PLANES == 2) *reinterpret_cast<half4*>(gram + c * ld + spot(r) + 64) = low;
  if (r0 != c0) {
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      *reinterpret_cast<_Float16*>(gram + (r + k) * ld + spot(c)) = high[k];
      if constexpr (PLANES == 2) *reinterpret_cast<_Float16*>(gram + (r + k) * ld + spot(c) + 64) = low[k];
    }
  }
}

template <int T, int WR, int WC, int PLANES>
int launch_product(const NsArgs& args, const NsArrays& arrays, int kind, int step, float a, float b, float c, uint32_t run,
                   uint32_t workgroups, void* stream) {
  constexpr uint32_t kThreads = WR * WC * 64;
  switch (kind) {
    case kNsGram: {
      const uint32_t splits = T == kNsSplitTile ? args.splits : 1;
      const int st = enqueue_with(0, ns_product<T, WR, WC, kNsGram, PLANES, float>, dim3(workgroups, splits), kThreads, stream, args, arrays, step, a, b, c, run);
      return st != 0 || splits < 2 ? st : enqueue_with(0, ns_join<PLANES>, dim3(workgroups, 4), 256, stream, args, step);
    }
    case kNsSquare: return enqueue(ns_product<T, WR, WC, kNsSquare, PLANES, float>, workgroups, kThreads, stream, args, arrays, step, a, b, c, run);
    case kNsApply: return enqueue(ns_product<T, WR, WC, kNsApply, PLANES, float>, workgroups, kThreads, stream, args, arrays, step, a, b, c, run);
    default:
      return arrays.out_bf16 ? enqueue(ns_product<T, WR, WC, kNsLast, PLANES, uint16_t>, workgroups, kThreads, stream, args, arrays, step, a, b, c, run)
                             : enqueue(ns_product<T, WR, WC, kNsLast, PLANES, float>, workgroups, kThreads, stream, args, arrays, step, a, b, c, run);
  }
}

}  // namespace

int launch_ns_small(const NsArgs& args, const NsArrays& arrays, const NsSteps& steps, int planes, uint32_t workgroups,
                    uint32_t lds_bytes, void* stream) {
  auto pick = [&](auto momentum, auto bf16, auto out) {
    typedef decltype(out) Out;
    return enqueue_with(lds_bytes, planes == 1 ? ns_small<1, bf16, momentum, Out> : ns_small<2, bf16, momentum, Out>, dim3(workgroups),
                        kNsSmallThreads, stream, args, arrays, steps);
  };
  auto with_out = [&](auto momentum, auto bf16) {
    return arrays.out_bf16 ? pick(momentum, bf16, uint16_t{}) : pick(momentum, bf16, float{});
  };
  if (arrays.momentum != nullptr) return arrays.in_bf16 ? with_out(Yes{}, Yes{}) : with_out(Yes{}, No{});
  return arrays.in_bf16 ? with_out(No{}, Yes{}) : with_out(No{}, No{});
}

int launch_ns_sums(const NsArgs& args, const NsArrays& arrays, uint32_t workgroups, void* stream) {
  if (arrays.momentum != nullptr)
    return arrays.in_bf16 ? enqueue(ns_sums<true, true>, workgroups, 256, stream, args, arrays)
                          : enqueue(ns_sums<false, true>, workgroups, 256, stream, args, arrays);
  return arrays.in_bf16 ? enqueue(ns_sums<true, false>, workgroups, 256, stream, args, arrays)
                        : enqueue(ns_sums<false, false>, workgroups, 256, stream, args, arrays);
}

int launch_ns_start(const NsArgs& args, const NsArrays& arrays, int planes, uint32_t workgroups, void* stream) {
  auto pick = [&](auto one, auto two) { return enqueue(planes == 1 ? one : two, workgroups, 256, stream, args, arrays); };
  if (arrays.momentum != nullptr)
    return arrays.in_bf16 ? pick(ns_start<true, true, 1>, ns_start<true, true, 2>) : pick(ns_start<false, true, 1>, ns_start<false, true, 2>);
  return arrays.in_bf16 ? pick(ns_start<true, false, 1>, ns_start<true, false, 2>) : pick(ns_start<false, false, 1>, ns_start<false, false, 2>);
}

int launch_ns_product(const NsArgs& args, const NsArrays& arrays, int kind, int tile, int planes, int step,
                      float a, float b, float c, uint32_t workgroups, void* stream) {
  if (tile == 256)
    return planes == 1 ? launch_product<256, 2, 4, 1>(args, arrays, kind, step, a, b, c, 32, workgroups, stream)
                       : launch_product<256, 2, 4, 2>(args, arrays, kind, step, a, b, c, 32, workgroups, stream);
  if (tile == 128)
    return planes == 1 ? launch_product<128, 2, 2, 1>(args, arrays, kind, step, a, b, c, 64, workgroups, stream)
                       : launch_product<128, 2, 2, 2>(args, arrays, kind, step, a, b, c, 64, workgroups, stream);
  return planes == 1 ? launch_product<64, 2, 2, 1>(args, arrays, kind, step, a, b, c, 64, workgroups, stream)
                     : launch_product<64, 2, 2, 2>(args, arrays, kind, step, a, b, c, 64, workgroups, stream);
}

}  // namespace noloco
