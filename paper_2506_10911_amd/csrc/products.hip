// Products sum over k of A(m, k) B(n, k) with bias, activation and residual in their end (kernels and their launchers):
// what matrices do forward (z = x M + bias, out = act(z) + residual) and backward (dx = dz M^T + add, M's gradient x^T dz).
// Operands lie with their numbers along k or along m (n) next to each other; the matrix cores take 16-bit ones.
//
// Large products (product_direct) load bf16 operands past the registers to the LDS as they lie.  Others are packed first, to
// rows that begin at multiples of 16 bytes:
//   bf16 result, one float operand     that one rounded to bf16, which costs as much as the result's own rounding (0.0023 of the result's norm
//                                      together, 0.0017 with the operand in two parts; but these are twice the products: dx of 8 x 2048 x
//                                      768 x 2304 and its matrix's gradient 237 us in place of 179, of 2 x 4096 x 4096 x 16384 4098 of 2014)
//   bf16 result, two float operands    both rounded to binary16 (11 bits), each times a power of two of its worker
//   float result, float operands       a float one as a pair of binary16 (22 bits), a bf16 one as one, times powers of two; the
//                                      products of two pairs but that of their low halves
// What binary16 leaves of a number is 2^-39 of the operand's largest or less.  Where a piece of a row is so small that this is more than
// 2^-22 of the piece's largest number (another row may hold anything, as padding does) the worker's operands are packed to bf16 parts
// instead, whose range is binary32's: two for a bf16 result (16 bits), three for a float one (24), and the products of parts that
// reach 2^-16 of the largest: 4 x 2048 x 2048 x 2048 float 400 us in place of 241, with a bf16 result 226 in place of 120.
// Small products (product_small), which packing would make longer, take any operands from memory to the registers and a float one
// apart into bf16: two of them, 16 bits, for a bf16 result; three, which together are the number, for a float one, and the products of
// parts that reach 2^-16 of the largest.
#include <type_traits>

#include "activations.h"
#include "device_numbers.h"
#include "model_internal.h"

namespace noloco {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint16_t ushort8 __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

#define lds_memory __attribute__((address_space(3)))

// What the end of a product adds to N neighbouring numbers of a row: the residual, or what is there.
template <int N> __device__ __forceinline__ void load_more(const ProductArgs& a, int64_t w, uint32_t m, uint32_t n, float* more) {
  if (a.more != nullptr || a.accumulate)
    load_numbers<N>(a.accumulate ? a.out : a.more, w * a.out_stride + m * a.out_ld + n, a.out_bf16, more);
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
  activate<N>(a.activation, v);
  if (a.more != nullptr || a.accumulate) {
    float more[N];
    load_more<N>(a, w, m, n, more);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += more[i];
  }
  store_numbers<N>(a.out, at, a.out_bf16, v);
}

// Do N neighbouring numbers (four or eight) of everything that the end of a product touches lie at a multiple of their vectors' size
// (16 bytes, four bf16 8)?
template <int N> __device__ __forceinline__ bool ends_in(const ProductArgs& a) {
  auto fits = [](const void* p, int32_t bf16, int64_t steps) {
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % (bf16 ? 2 * N : 16) == 0 && (steps & (bf16 ? N - 1 : 3)) == 0);
  };
  const int64_t steps = a.out_stride | a.out_ld;
  return fits(a.out, a.out_bf16, steps) && fits(a.more, a.out_bf16, steps) && fits(a.before, a.out_bf16, steps) &&
         fits(a.bias, a.bias_bf16, a.bias_stride);
}

// ---------------------------------------------------------------------------
// Small products
// ---------------------------------------------------------------------------

// Eight neighbouring numbers at any address of their type's alignment, in whole loads.
template <typename E> struct Eight {
  typedef E vector __attribute__((ext_vector_type(16 / sizeof(E)), aligned(sizeof(E))));
  E v[8];
  __device__ __forceinline__ void along(const E* p) {
    constexpr int N = 16 / sizeof(E);
#pragma unroll
    for (int i = 0; i < 8; i += N) {
      const vector x = *reinterpret_cast<const vector*>(p + i);
#pragma unroll
      for (int k = 0; k < N; ++k) v[i + k] = x[k];
    }
  }
  __device__ __forceinline__ void across(const E* p, int64_t apart, int there) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < there ? p[i * apart] : E(0);
  }
  // Part `part` of PARTS of the numbers.
  template <int PARTS> __device__ __forceinline__ bf16x8 part(int part) const {
    ushort8 out;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(E) == 2) {
        out[i] = v[i];
      } else {
        // cut, not rounded, but for the last: each rest is exact, and a third has at most eight bits
        float x = v[i];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (k < part) x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        out[i] = part == PARTS - 1 ? narrow(x) : static_cast<uint16_t>(__float_as_uint(x) >> 16);
      }
    }
    return __builtin_bit_cast(bf16x8, out);
  }
};

constexpr int kSmallRow = 36;                // floats of a row of a wave's sums in the LDS
constexpr int kSmallSums = 32 * kSmallRow;

// 32 x 32 of the result by a workgroup, whose waves take blocks of 64 k in turn and add up their sums in the LDS (and
// by several, where k is long and tiles are few).  Operands come
// from memory to the registers as the matrix cores take them, without a barrier: a wave's loads for 64 k are on their way together.
// What is read of an operand is read by every tile that needs it, which the caches bear in small products: 4 x 256 x 96 x 192 float
// 5.1 us, which is a launch's (through the LDS, a stage of 32 k after the other, 17.6); 1024 x 1024 x 1024 bf16 17, 126 TFLOP/s.
template <typename TA, typename TB, bool ALONG_A, bool ALONG_B, int PA, int PB>
__global__ __launch_bounds__(1024) void product_small(ProductArgs a, float* parts) {
  extern __shared__ __align__(16) float sums[];
  constexpr int kSlices = 4;
  const uint32_t lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tiles_m = (a.m + 31) / 32, m0 = blockIdx.x % tiles_m * 32, n0 = blockIdx.x / tiles_m * 32;
  const int64_t w = blockIdx.y;
  // rows behind the last one are the last one: what comes of them is not stored
  const uint32_t of32 = lane & 31, half = lane >> 5, m = min(m0 + of32, a.m - 1), n = min(n0 + of32, a.n - 1);
  const TA* const pa = static_cast<const TA*>(a.a.p) + w * a.a.worker_stride + (ALONG_A ? m * a.a.ld : static_cast<int64_t>(m));
  const TB* const pb = static_cast<const TB*>(a.b.p) + w * a.b.worker_stride + (ALONG_B ? n * a.b.ld : static_cast<int64_t>(n));
  float16v acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  auto block = [&](uint32_t k0, auto whole) {
    Eight<TA> fa[kSlices];
    Eight<TB> fb[kSlices];
    auto load = [&](auto& f, const auto* p, int64_t ld, auto along, uint32_t k) {
      if constexpr (whole) {
        if (along) f.along(p + k); else f.across(p + k * ld, ld, 8);
      } else {
        const int there = static_cast<int>(a.k) - static_cast<int>(k);
        if (along && there >= 8) f.along(p + k); else if (along) f.across(p + k, 1, there); else f.across(p + k * ld, ld, there);
      }
    };
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
      if (!whole && k0 + s * 16 >= a.k) break;
      const uint32_t k = k0 + s * 16 + half * 8;
      load(fa[s], pa, a.a.ld, std::integral_constant<bool, ALONG_A>{}, k);
      load(fb[s], pb, a.b.ld, std::integral_constant<bool, ALONG_B>{}, k);
    }
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
      if (!whole && k0 + s * 16 >= a.k) break;
      // the small products first
#pragma unroll
      for (int both = PA > 2 || PB > 2 ? 2 : 1; both >= 0; --both)
#pragma unroll
        for (int p = 0; p <= both; ++p) {
          if (p >= PA || both - p >= PB) continue;
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s].template part<PB>(both - p), fa[s].template part<PA>(p), acc, 0, 0, 0);
        }
    }
  };
  for (uint32_t k0 = (blockIdx.z * waves + wave) * 64; k0 < a.k; k0 += gridDim.z * waves * 64) {
    if (k0 + 64 <= a.k) block(k0, Yes{}); else block(k0, No{});
  }
  // element e of a lane: m = lane % 32, n = 8 (e / 4) + 4 (lane / 32) + e % 4
#pragma unroll
  for (int e = 0; e < 16; e += 4)
    *reinterpret_cast<float4v*>(sums + wave * kSmallSums + of32 * kSmallRow + e * 2 + half * 4) = float4v{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  __syncthreads();
  const bool fours = ends_in<4>(a);
  for (uint32_t v4 = threadIdx.x; v4 < 256; v4 += blockDim.x) {
    const uint32_t row = v4 >> 3, col = (v4 & 7) * 4;
    if (m0 + row >= a.m || n0 + col >= a.n) continue;
    float4v sum = *reinterpret_cast<const float4v*>(sums + row * kSmallRow + col);
    for (uint32_t i = 1; i < waves; ++i) sum += *reinterpret_cast<const float4v*>(sums + i * kSmallSums + row * kSmallRow + col);
    if (parts != nullptr) {
      *reinterpret_cast<float4v*>(parts + ((blockIdx.z * static_cast<uint64_t>(a.W) + w) * a.m + m0 + row) * ((a.n + 7) / 8 * 8) + n0 + col) = sum;
      continue;
    }
    float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    if (n0 + col + 4 <= a.n && fours) {
      finish<4>(a, w, m0 + row, n0 + col, v);
    } else {
#pragma unroll
      for (uint32_t c = 0; c < 4; ++c)
        if (n0 + col + c < a.n) finish<1>(a, w, m0 + row, n0 + col + c, v + c);
    }
  }
}

// ---------------------------------------------------------------------------
// Large products
// ---------------------------------------------------------------------------

// 16 bytes a lane from a buffer to the LDS, at `to` + 16 times the lane, past the registers; zeros for what lies behind the buffer's
// last byte.  The compiler does not count these loads: who reads what they bring waits for vmcnt itself.  m0 is a register that the
// compiler keeps nothing in and that a clobber list may not name; its own instructions that read it, each behind a write of
// its own, are none in these kernels.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v))); }
__device__ __forceinline__ uint4v buffer_words(uint64_t at, uint32_t bytes) {
  return uint4v{uniform(static_cast<uint32_t>(at)), uniform(static_cast<uint32_t>(at >> 32) & 0xffffu), uniform(bytes), 0x00020000u};
}
__device__ __forceinline__ void load_to_lds(uint4v buffer, uint32_t lane_offset, uint32_t to) {
  to = uniform(to);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" :: "v"(lane_offset), "s"(buffer), "s"(to) : "memory");
}

// Workgroups are dealt to the 8 XCDs in turn; each XCD takes runs of `run` consecutive tiles, which share rows and columns in
// its L2: 32 of 256 x 256, one round of its CUs, 64 of the smaller ones, of which two share a CU.
__device__ __forceinline__ uint32_t tile_of_block(uint32_t block, uint32_t blocks, uint32_t run) {
  const uint32_t whole = blocks / (8 * run) * (8 * run);
  if (block >= whole) return block;
  const uint32_t xcd = block & 7u, slot = block >> 3, k = slot / run;
  return (k * 8 + xcd) * run + (slot - k * run);
}

constexpr uint32_t kBehind = 0xfffffff0u;       // an offset behind every buffer

// How one operand's stages of 64 k come to the LDS and are read from it: T numbers along m (or n), by WAVES waves.
//   ALONG  rows of 128 bytes, one number of m each: 16-byte chunk q of row r lies at q ^ (r >> 1 & 7), so that the 16 lanes that read
//          at once meet 16 different quarters of the 64 banks
//   else   rows of 2 T bytes, one k each: chunk q of row k at q ^ (k & 3) << 2 (128-byte rows: q ^ (k >> 1 & 1) << 2), since four lanes of
//          a group of 16 read each of four rows; turned by the LDS's transposing reads
template <int T, int WAVES, bool ALONG> struct Stages {
  static constexpr int kBytes = T * 128, kLoads = T / 8 / WAVES, kRow = ALONG ? 128 : T * 2, kRows = 1024 / kRow;
  static_assert(kLoads >= 1 && kRow <= 1024, "tile");
  uint64_t base;             // of the tile's first number, k = 0, part 0
  uint64_t k_bytes, part_bytes;      // from one stage of 64 k, and from one part, to the next
  uint32_t ld_bytes, rows;   // ALONG: rows of the tile that there are; else: numbers of a row from the tile's first on
  uint32_t offset[kLoads];   // of the lane's 16 bytes of each load
  uint32_t chunk[2];         // ALONG: which eight k they are, of even and odd loads
  __device__ __forceinline__ void open(const void* p, int64_t worker, int64_t ld, int64_t part, uint32_t first, uint32_t size, uint32_t lane, uint32_t wave) {
    base = reinterpret_cast<uint64_t>(p) + 2 * static_cast<uint64_t>(worker + (ALONG ? first * ld : static_cast<int64_t>(first)));
    ld_bytes = static_cast<uint32_t>(2 * ld);
    k_bytes = ALONG ? 128 : 64ull * ld_bytes;
    part_bytes = 2 * part;
    rows = ALONG ? (size - first < T ? size - first : T) : size - first;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t load = wave * kLoads + i;
      if constexpr (ALONG) {
        const uint32_t q = (lane & 7) ^ (((load & 1) << 2 | lane >> 4) & 7);
        chunk[i & 1] = q;
        offset[i] = (load * 8 + (lane >> 3)) * ld_bytes + q * 16;
      } else {
        const uint32_t in_row = lane * 16 % kRow, k = load * kRows + lane * 16 / kRow;
        const uint32_t turn = kRow >= 256 ? (k & 3) << 2 : (kRow == 128 ? (k >> 1 & 1) << 2 : 0);
        offset[i] = k * ld_bytes + ((in_row >> 4) ^ turn) * 16;
      }
    }
  }
  // Asks for the stage that begins at k = 64 `stage`, of which `k_left` there are.
  __device__ __forceinline__ void ask(uint32_t part, uint32_t stage, uint32_t k_left, uint32_t to, uint32_t wave) const {
    const uint64_t at = base + part * part_bytes + stage * k_bytes;
    const uint32_t deep = k_left < 64 ? k_left : 64;
    // up to the end of the last vector that holds a number: what is not there whole comes as zeros
    const uint32_t last = ((ALONG ? k_left : rows) + 7) / 8 * 16, bytes = ((ALONG ? rows : deep) - 1) * ld_bytes + last;
    const uint4v buffer = buffer_words(at, bytes < kBehind ? bytes : kBehind);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      uint32_t from = offset[i];
      if constexpr (ALONG) {
        if (k_left < 64) from = chunk[i & 1] * 8 < k_left ? from : kBehind;
      }
      load_to_lds(buffer, from, to + (wave * kLoads + i) * 1024);
    }
  }
  // Where a lane's fragments of blocks of 32 numbers, `first` and on, lie in a stage.
  template <int BLOCKS> struct Reader {
    uint32_t at[ALONG ? 1 : BLOCKS], row;
    __device__ __forceinline__ void open(uint32_t first, uint32_t lane) {
      if constexpr (ALONG) {
        row = first + (lane & 31);
        at[0] = row * 128;
      } else {
        const uint32_t k = (lane >> 5) * 8 + (lane >> 2 & 3);
        const uint32_t turn = kRow >= 256 ? (k & 3) << 2 : (kRow == 128 ? (k >> 1 & 1) << 2 : 0);
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          const uint32_t byte = (first + i * 32) * 2 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
          at[i] = k * kRow + (((byte >> 4) ^ turn) << 4) + (byte & 15);
        }
      }
    }
    __device__ __forceinline__ short8v read(const char* stage, int block, int slice, uint32_t lane) const {
      if constexpr (ALONG) {
        const uint32_t q = ((slice * 2 + (lane >> 5)) ^ ((lane & 31) >> 1 & 7)) * 16;
        return *reinterpret_cast<const short8v*>(stage + at[0] + block * 32 * 128 + q);
      } else {
        const char* const from = stage + at[block] + slice * 16 * kRow;
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(from));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_memory short4v*)(from + 4 * kRow));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    }
  };
};

template <bool F16> __device__ __forceinline__ float16v multiply(short8v a, short8v b, float16v d) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), d, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), d, 0, 0, 0);
}

// TM x TN of the result by WM x WN waves, each (TM / WM) x (TN / WN) in blocks of 32 x 32.  Operands come to the LDS past the registers,
// STAGES stages of 64 k deep.  Fragments are read one slice of 16 k ahead of the products that use them, across the stage's end too:
// the barrier in front of the last slice's products tells that the next stage has come and that this one's buffer is free.
//
// Tiles of 256 x 256 (eight waves, a CU to themselves) 1070 to 1280 TFLOP/s where they fill the chip several times (8192 x 8192 x
// 8192 859 us; a large library product 1400 to 1460), of 128 x 128 (four, two workgroups a CU) 1040.  The matrix cores are busy 60 % of
// the cycles at 1.75 to 1.87 of 2.4 GHz, the LDS 25 %: a wave waits for its stage and the barrier for 30 to 41 % of its cycles, which nothing else
// on the CU covers.  (Reads held in front of the slice's products by force, and four stages for a workgroup with a CU to itself, changed
// nothing.)  The end of a tile is not hidden either: 8 x 4096 x 2048 x 8192 takes 1027 us, with the activation and what stands before
// it 1175.  32 x 256 reads a matrix for a few tokens as it streams, four stages deep: 2 x 16384 x 4096 44 us, 6.1 TB/s.
template <int TM, int TN, int WM, int WN, bool ALONG_A, bool ALONG_B, bool F16, int STAGES>
__global__ __launch_bounds__(WM * WN * 64) void product_direct(ProductArgs a, DirectArgs d) {
  constexpr int kWaves = WM * WN, kThreads = kWaves * 64, MB = TM / WM / 32, NB = TN / WN / 32, kSlices = 4;
  typedef Stages<TM, kWaves, ALONG_A> A;
  typedef Stages<TN, kWaves, ALONG_B> B;
  constexpr int kStage = A::kBytes + B::kBytes, kLoads = A::kLoads + B::kLoads;
  constexpr int kImageRow = TN * 4 + 16, kImageRows = WM * 32, kImage = kImageRow * kImageRows;
  constexpr int kLds = STAGES * kStage > kImage ? STAGES * kStage : kImage;
  static_assert(kLds <= 160 * 1024 && (STAGES & (STAGES - 1)) == 0 && STAGES * kLoads < 64, "stages");
  __shared__ __align__(1024) char lds[kLds];
  const uint32_t thread = threadIdx.x, lane = thread & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const uint32_t wm = wave / WN, wn = wave % WN;

  // four tiles of m by all of n
  const uint32_t tiles = d.tiles_m * d.tiles_n, tile = tile_of_block(blockIdx.x, gridDim.x, d.run);
  const uint32_t w = tile / tiles, of_worker = tile - w * tiles, band = 4 * d.tiles_n, group = of_worker / band, in = of_worker - group * band;
  const uint32_t high = d.tiles_m - group * 4 < 4 ? d.tiles_m - group * 4 : 4;
  const uint32_t m0 = (group * 4 + in % high) * TM, n0 = in / high * TN;

  // is the worker in bf16 parts?  Asked for before the operands' places are made
  const int32_t parts_flag = F16 ? d.exponents[4 * w + 2] : 0;
  A of_a;
  B of_b;
  of_a.open(d.a, w * d.a_worker, d.a_ld, d.a_part, m0, a.m, lane, wave);
  of_b.open(d.b, w * d.b_worker, d.b_ld, d.b_part, n0, a.n, lane, wave);
  const bool in_parts = F16 && uniform(static_cast<uint32_t>(parts_flag)) != 0;
  const uint32_t a_parts = in_parts ? d.a_parts[1] : d.a_parts[0], b_parts = in_parts ? d.b_parts[1] : d.b_parts[0];
  const uint32_t deep = (a.k + 63) / 64, all = deep * (in_parts ? d.segments[1] : d.segments[0]);
  const uint32_t s0 = static_cast<uint32_t>(static_cast<uint64_t>(all) * blockIdx.y / d.splits);
  const uint32_t stages = static_cast<uint32_t>(static_cast<uint64_t>(all) * (blockIdx.y + 1) / d.splits) - s0;
  uint32_t segment = s0 / deep, stage_k = s0 - segment * deep, asked = 0;
  const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_memory char*)lds));
  auto ask = [&] {
    const uint32_t to = lds_at + (asked & (STAGES - 1)) * kStage, k_left = a.k - stage_k * 64;
    of_a.ask(a_parts >> segment * 2 & 3, stage_k, k_left, to, wave);
    of_b.ask(b_parts >> segment * 2 & 3, stage_k, k_left, to + A::kBytes, wave);
    ++asked;
    if (++stage_k == deep) {
      stage_k = 0;
      ++segment;
    }
  };
  typename A::template Reader<MB> read_a;
  typename B::template Reader<NB> read_b;
  read_a.open(wm * (TM / WM), lane);
  read_b.open(wn * (TN / WN), lane);
  struct Fragments { short8v a[MB], b[NB]; };
  auto read = [&](uint32_t stage, int slice, Fragments& f) {
    const char* const from = lds + (stage & (STAGES - 1)) * kStage;
#pragma unroll
    for (int i = 0; i < MB; ++i) f.a[i] = read_a.read(from, i, slice, lane);
#pragma unroll
    for (int j = 0; j < NB; ++j) f.b[j] = read_b.read(from + A::kBytes, j, slice, lane);
  };
  float16v acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  if (stages >= STAGES) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) ask();
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((STAGES - 1) * kLoads) : "memory");
  } else {
    for (uint32_t i = 0; i < stages; ++i) ask();
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  }
  Fragments even, odd;
  read(0, 0, even);
  // The stages behind the last one that is asked for by themselves, so that nothing in the loop is conditional.
  auto stage = [&](uint32_t s, auto half, auto ask_more, auto read_next) {
#pragma unroll
    for (int slice = 0; slice < kSlices; ++slice) {
      Fragments& now = slice & 1 ? odd : even;
      Fragments& next = slice & 1 ? even : odd;
      if (slice + 1 < kSlices) {
        read(s, slice + 1, next);
      } else {
        // the next stage has come, those behind it may be on their way; wait and barrier in one, so that no read comes between them
        if constexpr (ask_more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if constexpr (read_next) read(s + 1, 0, next);
        if constexpr (ask_more) ask();
      }
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = multiply<decltype(half)::value>(now.b[j], now.a[i], acc[i][j]);
      // the products of a slice stay behind its reads, which the compiler would put in front of the next barrier
      if constexpr (TM == 256) __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto all_stages = [&](auto half) {
    uint32_t s = 0;
    for (; s + STAGES < stages; ++s) stage(s, half, Yes{}, Yes{});
    for (; s + 1 < stages; ++s) stage(s, half, No{}, Yes{});
    stage(s, half, No{}, No{});
  };
  if (F16 && !in_parts) all_stages(std::bool_constant<F16>{}); else all_stages(std::false_type{});

  if (F16 && !in_parts) {
    const int by = -(d.exponents[4 * w] + d.exponents[4 * w + 1]);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = ldexpf(acc[i][j][e], by);
  }

  // Results go through the LDS, 32 rows of every wave at a time, and from there in whole lines.  Block (i, j), element e of a lane:
  // m = 32 i + lane % 32, n = 32 j + 8 (e / 4) + 4 (lane / 32) + e % 4.
  const bool eights = ends_in<8>(a), fours = ends_in<4>(a);
  const bool adds = d.parts == nullptr && eights && a.activation == NOLOCO_ACT_NONE && a.before == nullptr && a.bias == nullptr && a.n % 8 == 0 &&
                    (a.more != nullptr || a.accumulate);
  const uint32_t of32 = lane & 31, half = lane >> 5;
  constexpr int kVectors = kImageRows * (TN / 8) / kThreads;      // of eight numbers that a thread writes at a time
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    auto row_of = [&](uint32_t row) { return m0 + row / 32 * (TM / WM) + i * 32 + row % 32; };
    // Where something is added and nothing else is done it is asked for before the barriers, all of it at once (one by one, each
    // behind the last one's store, 8 products of 768 x 2048 x 2304 added to float gradients took 84 us).
    float more[kVectors][8];
    if (adds) {
#pragma unroll
      for (int u = 0; u < kVectors; ++u) {
        const uint32_t v = thread + u * kThreads, m = row_of(v / (TN / 8)), n = n0 + v % (TN / 8) * 8;
        if (m < a.m && n + 8 <= a.n) load_more<8>(a, w, m, n, more[u]);
      }
    }
    __syncthreads();
    char* const mine = lds + (wm * 32 + of32) * kImageRow + (wn * (TN / WN) + half * 4) * 4;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<float4v*>(mine + j * 128 + e * 8) = float4v{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
    __syncthreads();
    if (adds) {
#pragma unroll
      for (int u = 0; u < kVectors; ++u) {
        const uint32_t v = thread + u * kThreads, row = v / (TN / 8), col = v % (TN / 8) * 8, m = row_of(row), n = n0 + col;
        if (m >= a.m || n >= a.n) continue;
        const float4v* const from = reinterpret_cast<const float4v*>(lds + row * kImageRow + col * 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) more[u][e] += from[e / 4][e % 4];
        store_numbers<8>(a.out, w * a.out_stride + m * a.out_ld + n, a.out_bf16, more[u]);
      }
    } else if (d.parts != nullptr || fours) {
      for (uint32_t v = thread; v < kImageRows * (TN / 8); v += kThreads) {
        const uint32_t row = v / (TN / 8), col = v % (TN / 8) * 8, m = row_of(row), n = n0 + col;
        if (m >= a.m || n >= a.n) continue;
        const float4v* const from = reinterpret_cast<const float4v*>(lds + row * kImageRow + col * 4);
        const float4v lo = from[0], hi = from[1];
        if (d.parts != nullptr) {
          float4v* const to = reinterpret_cast<float4v*>(d.parts + ((static_cast<uint64_t>(blockIdx.y) * a.W + w) * a.m + m) * d.parts_ld + n);
          to[0] = lo;
          to[1] = hi;
          continue;
        }
        float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (eights && n + 8 <= a.n) {
          finish<8>(a, w, m, n, x);
        } else {
#pragma unroll
          for (int h = 0; h < 8; h += 4) {
            if (n + h + 4 <= a.n) {
              finish<4>(a, w, m, n + h, x + h);
            } else {
#pragma unroll
              for (int e = h; e < h + 4; ++e)
                if (n + e < a.n) finish<1>(a, w, m, n + e, x + e);
            }
          }
        }
      }
    } else {
      for (uint32_t v = thread; v < kImageRows * TN; v += kThreads) {
        const uint32_t row = v / TN, col = v % TN, m = row_of(row), n = n0 + col;
        if (m >= a.m || n >= a.n) continue;
        float x = *reinterpret_cast<const float*>(lds + row * kImageRow + col * 4);
        finish<1>(a, w, m, n, &x);
      }
    }
  }
}

// Results of fewer vectors of eight are joined a number to a thread, others a vector. Few numbers want many waves, as their loads wait for each
// other: whole products 3 x 119 x 7665 x 405 31.0 us against 33.8 in vectors, 100 x 5000 x 1001 22.4 and 25.1, 512 x 8192 x 2048 (131072
// vectors) 36.8 and 37.3. Many want wide loads: 1024 x 8192 x 4096 (524288) 85.5 us against 81.4 in vectors.
constexpr uint64_t kJoinVectors = 1 << 18;

// The parts of a product whose k is shared out, in their order, and its end: a thread takes N neighbouring numbers.
template <int N> __global__ __launch_bounds__(256) void product_join(ProductArgs a, DirectArgs d) {
  const uint32_t wide = (a.n + N - 1) / N;
  const uint64_t v = static_cast<uint64_t>(blockIdx.x) * blockDim.x + threadIdx.x, rows = static_cast<uint64_t>(a.W) * a.m;
  if (v >= rows * wide) return;
  const uint64_t row = v / wide, w = row / a.m;
  const uint32_t n = static_cast<uint32_t>(v - row * wide) * N, m = static_cast<uint32_t>(row - w * a.m);
  float x[N] = {};
  const float* const from = d.parts + row * d.parts_ld + n;
#pragma unroll 4
  for (uint32_t s = 0; s < d.splits; ++s) {
    float part[N];
    Stored<float, N>::load(from + s * rows * d.parts_ld, part);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] += part[e];
  }
  if constexpr (N == 1) {
    finish<1>(a, w, m, n, x);
  } else if (n + N <= a.n && ends_in<N>(a)) {
    finish<N>(a, w, m, n, x);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (n + e < a.n) finish<1>(a, w, m, n + e, x + e);
  }
}

// ---------------------------------------------------------------------------
// Operands as large products take them
// ---------------------------------------------------------------------------

// Eight numbers of a row from column `col` on as floats; zeros behind its end.
__device__ __forceinline__ void load_eight(const PackOperand& o, int64_t row_at, uint32_t col, float* x) {
  auto load = [&](auto element) {
    typedef decltype(element) E;
    const E* const p = static_cast<const E*>(o.p) + row_at + col;
    Eight<E> eight;
    if (col + 8 <= o.wide) eight.along(p); else eight.across(p, 1, static_cast<int>(o.wide - col));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(E) == 2) x[e] = widen(eight.v[e]); else x[e] = eight.v[e];
    }
  };
  if (o.bf16) load(uint16_t{}); else load(float{});
}

// The largest size among eight numbers, as the bits of a float: sizes are in the order of their bits, above all of them infinities and NaN, which
// count as zeros.
template <typename E> __device__ __forceinline__ uint32_t largest_of(const Eight<E>& eight) {
  constexpr uint32_t kInfinite = 0x7f800000u;
  uint32_t most = 0;
  if constexpr (sizeof(E) == 2) {
    ushort8 sizes;
#pragma unroll
    for (int e = 0; e < 8; ++e) sizes[e] = eight.v[e] & 0x7fff;
    const auto four = __builtin_elementwise_max(sizes.lo, sizes.hi);
    const auto two = __builtin_elementwise_max(four.lo, four.hi);
    most = static_cast<uint32_t>(max(two[0], two[1])) << 16;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(eight.v[e]) & 0x7fffffffu);
  }
  if (most >= kInfinite) {
    most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t size = (sizeof(E) == 2 ? static_cast<uint32_t>(eight.v[e]) << 16 : __builtin_bit_cast(uint32_t, static_cast<float>(eight.v[e]))) & 0x7fffffffu;
      most = size < kInfinite ? max(most, size) : most;
    }
  }
  return most;
}
template <int CONTROL> __device__ __forceinline__ uint32_t larger(uint32_t v) {
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CONTROL, 15, 15, true)));
}
__device__ __forceinline__ uint32_t lane_bits(uint32_t v, int lane) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), lane)); }
// Over the wave, in scalar registers from the sixteens on.
__device__ __forceinline__ uint32_t wave_largest_bits(uint32_t v) {
  v = larger<0x140>(larger<0x141>(larger<0x4E>(larger<0xB1>(v))));
  return max(max(lane_bits(v, 0), lane_bits(v, 16)), max(lane_bits(v, 32), lane_bits(v, 48)));
}

// The largest finite number of what one of kPackParts workgroups takes of an operand, and the least of its pieces' largest but those of zeros
// alone: a wave takes a piece, a vector of eight a lane, or several short rows.  Who has no piece or vector of its own takes the last one again,
// and a row's last vector and last piece begin within the ones before them (a number by itself may well be small), so that loads depend on
// nothing; four of them are on their way together.  Bound by instructions, of which small operands' waves have few to share: the two of 8
// products, 1038 x 332 and 1842 x 332 float, take 7 us (with loads under conditions and sizes compared as floats 15).
__global__ __launch_bounds__(256) void product_largest(PackArgs p) {
  constexpr uint32_t kAhead = 4;
  static_assert(kPackPiece == 64 * 8, "a vector of a lane");
  const PackOperand& o = p.operand[blockIdx.z];
  const int64_t w = blockIdx.y;
  const uint32_t vectors = (o.wide + 7) / 8, wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  uint32_t most = 0, least = ~0u;              // least: less one, so that zeros are the largest
  auto find = [&](auto element) {
    typedef decltype(element) E;
    const E* const from = static_cast<const E*>(o.p) + w * o.worker_stride;
    const uint32_t last = o.wide - 8;
    if (vectors > 32) {
      const uint32_t pieces = (vectors + 63) / 64, all = o.rows * pieces, begin = vectors - min(vectors, 64u);
      for (uint32_t first = blockIdx.x * 4 + wave; first < all; first += kAhead * kPackParts * 4) {
        Eight<E> eight[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
          const uint32_t piece = min(first + i * kPackParts * 4, all - 1), row = pieces == 1 ? piece : uniform(piece / pieces);
          eight[i].along(from + row * o.ld + min((min((piece - row * pieces) * 64, begin) + lane) * 8, last));
        }
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
          const uint32_t here = wave_largest_bits(largest_of(eight[i]));
          most = max(most, here);
          least = min(least, here - 1);
        }
      }
      return;
    }
    uint32_t lanes = 1;
    while (lanes < vectors) lanes *= 2;
    const uint32_t at_once = 256 / lanes, col = min((lane & (lanes - 1)) * 8, last);
    for (uint32_t first = blockIdx.x * at_once; first < o.rows; first += kAhead * kPackParts * at_once) {
      Eight<E> eight[kAhead];
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) {
        const E* const at = from + min(first + i * kPackParts * at_once + threadIdx.x / lanes, o.rows - 1) * o.ld;
        if (o.wide >= 8) eight[i].along(at + col); else eight[i].across(at, 1, static_cast<int>(o.wide));
      }
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) {
        uint32_t here = largest_of(eight[i]);
        if (lanes > 1) here = larger<0xB1>(here);
        if (lanes > 2) here = larger<0x4E>(here);
        if (lanes > 4) here = larger<0x141>(here);
        if (lanes > 8) here = larger<0x140>(here);
        if (lanes > 16) here = max(here, static_cast<uint32_t>(__shfl_xor(static_cast<int>(here), 16)));
        most = max(most, here);
        least = min(least, here - 1);
      }
    }
    most = wave_largest_bits(most);
    least = ~wave_largest_bits(~least);
  };
  if (o.bf16) find(uint16_t{}); else find(float{});
  __shared__ uint32_t waves[2][4];
  if (lane == 0) {
    waves[0][wave] = most;
    waves[1][wave] = least;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float* const to = p.largest + (w * 2 + blockIdx.z) * 2 * kPackParts + blockIdx.x;
    to[0] = __uint_as_float(max(max(waves[0][0], waves[0][1]), max(waves[0][2], waves[0][3])));
    least = min(min(waves[1][0], waves[1][1]), min(waves[1][2], waves[1][3]));
    to[kPackParts] = least == ~0u ? __builtin_inff() : __uint_as_float(least + 1);
  }
}

// Rows of `wide` numbers to rows of a multiple of eight, zeros behind their ends: bf16, or one or two binary16 of the numbers times a power
// of two that takes the largest of the worker's operand to between 2^14 and 2^15, or `parts` bf16 where that leaves too little of a row.
__global__ __launch_bounds__(256) void product_pack(PackArgs p) {
  const PackOperand& o = p.operand[blockIdx.z];
  if (o.out == nullptr) return;
  const int64_t w = blockIdx.y;
  int by = 0;
  bool halves = p.f16;
  if (p.f16) {
    static_assert(kPackParts == 256, "four of a lane");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t* const from = reinterpret_cast<const uint32_t*>(p.largest) + (w * 2 + i) * 2 * kPackParts + (threadIdx.x & 63) * 4;
      const uint4v four = *reinterpret_cast<const uint4v*>(from), rows = *reinterpret_cast<const uint4v*>(from + kPackParts);
      // floats of at least zero, in the order of their bits
      const float most = __uint_as_float(wave_largest_bits(max(max(four[0], four[1]), max(four[2], four[3]))));
      const float least = __uint_as_float(~wave_largest_bits(~min(min(rows[0], rows[1]), min(rows[2], rows[3]))));
      halves = halves && !(least < most * kPackRange);
      if (i == blockIdx.z && most > 0.f) {
        int power;
        (void)frexpf(most, &power);      // most = 0.5 to 1 times 2^power
        by = 15 - power;
      }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      p.exponents[w * 4 + blockIdx.z] = by;
      if (blockIdx.z == 0) p.exponents[w * 4 + 2] = halves ? 0 : 1;
    }
  }
  const uint32_t vectors = (o.wide + 7) / 8, all = o.rows * vectors;
  uint16_t* const out = static_cast<uint16_t*>(o.out) + w * (all * 8ll);
  for (uint32_t v = blockIdx.x * 256 + threadIdx.x; v < all; v += gridDim.x * 256) {
    const uint32_t row = v / vectors;
    float x[8];
    load_eight(o, w * o.worker_stride + row * o.ld, (v - row * vectors) * 8, x);
    auto store = [&](int part, const ushort8& eight) { *reinterpret_cast<ushort8*>(out + part * (p.W * (all * 8ll)) + v * 8ll) = eight; };
    ushort8 first, second;
    if (halves) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = ldexpf(x[e], by);
        const _Float16 high = static_cast<_Float16>(y);
        first[e] = __builtin_bit_cast(uint16_t, high);
        second[e] = __builtin_bit_cast(uint16_t, static_cast<_Float16>(y - static_cast<float>(high)));
      }
      store(0, first);
      if (o.parts == 3) store(1, second);
    } else {
      for (int part = 0; part < o.parts; ++part) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // cut where the nearest bf16 is infinity, which a zero would make NaN: what is left is exact either way
          first[e] = narrow(x[e]);
          if ((first[e] & 0x7fff) == 0x7f80) first[e] = static_cast<uint16_t>(__float_as_uint(x[e]) >> 16);
          x[e] -= widen(first[e]);
        }
        store(part, first);
      }
    }
  }
}

}  // namespace

namespace {

int launch_small(const ProductArgs& args, uint32_t splits, float* parts, void* stream) {
  // blocks of 64 k that a wave takes: one, where a workgroup has as many waves
  const uint32_t blocks = (args.k + 63) / 64, waves = blocks <= 2 ? std::max(blocks, 1u) : (blocks <= 4 ? 4 : (blocks <= 8 ? 8 : 16));
  const dim3 grid((args.m + 31) / 32 * ((args.n + 31) / 32), args.W, splits);
  auto with_layout = [&](auto ta, auto tb, auto pa, auto pb) {
    typedef decltype(ta) TA;
    typedef decltype(tb) TB;
    constexpr int PA = decltype(pa)::value, PB = decltype(pb)::value;
    if (args.a.along_k) {
      return args.b.along_k ? enqueue(product_small<TA, TB, true, true, PA, PB>, grid, waves * 64, waves * kSmallSums * 4, stream, args, parts)
                            : enqueue(product_small<TA, TB, true, false, PA, PB>, grid, waves * 64, waves * kSmallSums * 4, stream, args, parts);
    }
    return enqueue(product_small<TA, TB, false, false, PA, PB>, grid, waves * 64, waves * kSmallSums * 4, stream, args, parts);
  };
  const uint16_t half = 0;
  const float whole = 0.f;
  const Number<1> one;
  const Number<2> two;
  const Number<3> three;
  if (args.a.bf16) {
    if (args.b.bf16) return with_layout(half, half, one, one);
    return args.out_bf16 ? with_layout(half, whole, one, two) : with_layout(half, whole, one, three);
  }
  if (args.b.bf16) return args.out_bf16 ? with_layout(whole, half, two, one) : with_layout(whole, half, three, one);
  return args.out_bf16 ? with_layout(whole, whole, two, two) : with_layout(whole, whole, three, three);
}

}  // namespace

int launch_product(const ProductArgs& args, const ProductPlan& plan, char* room, void* stream) {
  if (args.m == 0 || args.n == 0) return 0;
  DirectArgs d{};
  d.splits = plan.splits;
  d.parts = plan.splits > 1 ? reinterpret_cast<float*>(room + plan.parts_at) : nullptr;
  d.parts_ld = (args.n + 7) / 8 * 8;
  auto join = [&](int st) {
    if (st != 0 || d.splits == 1) return st;
    const uint64_t rows = static_cast<uint64_t>(args.W) * args.m, vectors = rows * ((args.n + 7) / 8);
    if (vectors < kJoinVectors) return enqueue(product_join<1>, dim3(static_cast<uint32_t>((rows * args.n + 63) / 64)), 64, 0, stream, args, d);
    return enqueue(product_join<8>, dim3(static_cast<uint32_t>((vectors + 255) / 256)), 256, 0, stream, args, d);
  };
  if (plan.tile == 0) return join(launch_small(args, plan.splits, d.parts, stream));
  PackArgs pack{};
  pack.f16 = plan.f16;
  pack.W = args.W;
  pack.largest = reinterpret_cast<float*>(room + plan.largest_at);
  pack.exponents = reinterpret_cast<int32_t*>(room + plan.exponents_at);
  uint64_t most = 0;
  for (int i = 0; i < 2; ++i) {
    const Operand& o = i == 0 ? args.a : args.b;
    const uint32_t size = i == 0 ? args.m : args.n;
    const void* p = o.p;
    int64_t worker = o.worker_stride, ld = o.ld, part = 0;
    if (plan.packed[i]) {
      PackOperand& to = pack.operand[i];
      to = {o.p, room + plan.packed_at[i], o.worker_stride, o.ld, o.along_k ? size : args.k, o.along_k ? args.k : size, o.bf16, plan.parts[i]};
      p = to.out;
      ld = (to.wide + 7ll) / 8 * 8;
      worker = to.rows * ld;
      part = worker * args.W;
      most = std::max<uint64_t>(most, to.rows * static_cast<uint64_t>(ld) / 8);
    }
    (i == 0 ? d.a : d.b) = p;
    (i == 0 ? d.a_worker : d.b_worker) = worker;
    (i == 0 ? d.a_ld : d.b_ld) = ld;
    (i == 0 ? d.a_part : d.b_part) = part;
  }
  if (most > 0) {
    int st = 0;
    if (plan.f16) st = enqueue(product_largest, dim3(kPackParts, args.W, 2), 256, 0, stream, pack);
    if (st == 0) st = enqueue(product_pack, dim3(static_cast<uint32_t>(std::min<uint64_t>((most + 255) / 256, 4096)), args.W, 2), 256, 0, stream, pack);
    if (st != 0) return st;
  }
  // the small products first: of the low halves, of the high ones; of bf16 parts, by what they reach
  auto segment = [&](int way, uint32_t part_a, uint32_t part_b) {
    d.a_parts[way] |= part_a << 2 * d.segments[way];
    d.b_parts[way] |= part_b << 2 * d.segments[way]++;
  };
  if (plan.parts[0] == 3) segment(0, 1, 0);
  if (plan.parts[1] == 3) segment(0, 0, 1);
  segment(0, 0, 0);
  if (plan.f16) {
    for (int both = std::max(plan.parts[0], plan.parts[1]) - 1; both >= 0; --both)
      for (int of_a = 0; of_a <= both; ++of_a)
        if (of_a < plan.parts[0] && both - of_a < plan.parts[1]) segment(1, of_a, both - of_a);
  }
  d.exponents = pack.exponents;
  auto tiles = [&](uint32_t tm, uint32_t tn, uint32_t run) {
    d.tiles_m = (args.m + tm - 1) / tm;
    d.tiles_n = (args.n + tn - 1) / tn;
    d.run = run;
    return dim3(d.tiles_m * d.tiles_n * args.W, d.splits);
  };
  const bool aa = args.a.along_k, ab = args.b.along_k;
  int st;
#define NOLOCO_PRODUCT(TM, TN, WM, WN, STAGES, AA, AB) \
  (plan.f16 ? enqueue(product_direct<TM, TN, WM, WN, AA, AB, true, STAGES>, grid, WM * WN * 64, 0, stream, args, d) \
            : enqueue(product_direct<TM, TN, WM, WN, AA, AB, false, STAGES>, grid, WM * WN * 64, 0, stream, args, d))
  if (plan.tile == 256) {
    const dim3 grid = tiles(256, 256, 32);
    st = !aa ? NOLOCO_PRODUCT(256, 256, 2, 4, 2, false, false) : (ab ? NOLOCO_PRODUCT(256, 256, 2, 4, 2, true, true) : NOLOCO_PRODUCT(256, 256, 2, 4, 2, true, false));
  } else if (plan.tile == 128) {
    const dim3 grid = tiles(128, 128, 64);
    st = !aa ? NOLOCO_PRODUCT(128, 128, 2, 2, 2, false, false) : (ab ? NOLOCO_PRODUCT(128, 128, 2, 2, 2, true, true) : NOLOCO_PRODUCT(128, 128, 2, 2, 2, true, false));
  } else {
    const dim3 grid = tiles(32, 256, 64);
    st = ab ? NOLOCO_PRODUCT(32, 256, 1, 4, 4, true, true) : NOLOCO_PRODUCT(32, 256, 1, 4, 4, true, false);
  }
#undef NOLOCO_PRODUCT
  return join(st);
}

}  // namespace noloco
