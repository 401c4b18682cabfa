// Embedding lookup and its gradient (kernels and their launchers).
//
//   lookup     out[w][t] = scale * table_w[tokens[w][t]]
//   gradient   grad_w[v] = (accumulate ? grad_w[v] : 0) + scale * sum of dout[w][t] over the t with tokens[w][t] = v
//
// Both are bound by memory.  The gradient's rows are found by sorting (token, position) pairs: lists of 2048 are sorted in
// the LDS, and sixteen lists at a time are joined by ranks (a pair's place is its place in its own list plus the number
// of smaller pairs in each other list).  No atomics anywhere: a row's sum is taken in the order of positions, in chunks
// of 32 sorted pairs whose sums are joined in order.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "inner_internal.h"

namespace noloco {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint16_t ushort4v __attribute__((ext_vector_type(4)));

template <typename T> struct same { typedef T type; };
template <typename... KArgs>
int enqueue(void (*kernel)(KArgs...), dim3 grid, uint32_t block, void* stream, typename same<KArgs>::type... args) {
  void* argv[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), argv, 0, static_cast<hipStream_t>(stream));
}

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ uint16_t narrow(float v) {   // to bf16, nearest, ties to even; NaN stays NaN
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
  return static_cast<uint16_t>((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// N neighbouring numbers of type E (float, or bf16 as stored) as floats.
template <typename E, int N> struct Numbers {
  float v[N];
  __device__ __forceinline__ void load(const E* p) {
    if constexpr (N == 4 && sizeof(E) == 4) {
      const float4v x = *reinterpret_cast<const float4v*>(p);
      for (int i = 0; i < 4; ++i) v[i] = x[i];
    } else if constexpr (N == 4) {
      const ushort4v x = *reinterpret_cast<const ushort4v*>(p);
      for (int i = 0; i < 4; ++i) v[i] = widen(x[i]);
    } else if constexpr (sizeof(E) == 4) {
      v[0] = *p;
    } else {
      v[0] = widen(*p);
    }
  }
  __device__ __forceinline__ void store(E* p) const {
    if constexpr (N == 4 && sizeof(E) == 4) {
      *reinterpret_cast<float4v*>(p) = float4v{v[0], v[1], v[2], v[3]};
    } else if constexpr (N == 4) {
      *reinterpret_cast<ushort4v*>(p) = ushort4v{narrow(v[0]), narrow(v[1]), narrow(v[2]), narrow(v[3])};
    } else if constexpr (sizeof(E) == 4) {
      *p = v[0];
    } else {
      *p = narrow(v[0]);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
  }
};

// A token's row, or vocab for one that has none.
__device__ __forceinline__ uint32_t token_at(const EmbedArgs& a, int64_t i) {
  const int64_t token = a.tokens_i64 ? static_cast<const int64_t*>(a.tokens)[i] : static_cast<const int32_t*>(a.tokens)[i];
  return token >= 0 && token < static_cast<int64_t>(a.vocab) ? static_cast<uint32_t>(token) : a.vocab;
}

// One wave a token.
template <typename Table, typename Row, int N>
__global__ __launch_bounds__(256) void embed_lookup(EmbedArgs a) {
  const int64_t all = static_cast<int64_t>(a.W) * a.num_tokens;
  const uint32_t lane = threadIdx.x & 63;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); i < all; i += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t w = i / a.num_tokens;
    const uint32_t token = token_at(a, i);
    const Table* from = static_cast<const Table*>(a.table) + w * a.stride + static_cast<int64_t>(token) * a.width;
    Row* to = static_cast<Row*>(a.rows) + i * a.width;
    for (uint32_t c = lane * N; c < a.width; c += 64 * N) {
      Numbers<Table, N> x;
      x.zero();
      if (token < a.vocab) {
        x.load(from + c);
#pragma unroll
        for (int k = 0; k < N; ++k) x.v[k] *= a.scale;
      }
      Numbers<Row, N> y;
#pragma unroll
      for (int k = 0; k < N; ++k) y.v[k] = x.v[k];
      y.store(to + c);
    }
  }
}

// ---------------------------------------------------------------------------
// Sorting
// ---------------------------------------------------------------------------

// A workgroup sorts 2048 positions of one worker in its LDS: a bitonic network over (token, position).
__global__ __launch_bounds__(1024) void embed_sort(EmbedArgs a, uint64_t* out) {
  __shared__ uint64_t key[kSortChunk];
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortChunk, row = static_cast<int64_t>(blockIdx.y) * a.num_tokens;
  const uint32_t t = threadIdx.x;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t p = first + t + h * 1024;
    key[t + h * 1024] = p < a.num_tokens ? static_cast<uint64_t>(token_at(a, row + p)) << 32 | static_cast<uint32_t>(p) : ~0ull;
  }
  for (uint32_t size = 2; size <= kSortChunk; size *= 2) {
    for (uint32_t gap = size / 2; gap > 0; gap /= 2) {
      __syncthreads();
      const uint32_t i = (t & ~(gap - 1)) * 2 + (t & (gap - 1)), j = i + gap;
      const uint64_t x = key[i], y = key[j];
      if ((x > y) == ((i & size) == 0)) {
        key[i] = y;
        key[j] = x;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (first + t + h * 1024 < a.num_tokens) out[row + first + t + h * 1024] = key[t + h * 1024];
}

// Joins up to 16 sorted lists of `length` pairs each: a pair's place is the number of smaller ones in all of them.
// Pairs differ, since positions do.
__global__ __launch_bounds__(256) void embed_merge(const uint64_t* from, uint64_t* to, int64_t num_tokens, int64_t length) {
  const int64_t p = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (p >= num_tokens) return;
  const uint64_t* list = from + static_cast<int64_t>(blockIdx.y) * num_tokens;
  const int64_t mine = p / length, begin = mine / kMergeWays * kMergeWays;
  const uint64_t key = list[p];
  int64_t lo[kMergeWays], hi[kMergeWays];
#pragma unroll
  for (int k = 0; k < kMergeWays; ++k) {
    const int64_t a = (begin + k) * length, b = a + length;
    lo[k] = a < num_tokens ? a : num_tokens;
    hi[k] = b < num_tokens ? b : num_tokens;
  }
  // sixteen searches side by side
  for (int64_t span = length; span > 0; span >>= 1) {
#pragma unroll
    for (int k = 0; k < kMergeWays; ++k) {
      if (lo[k] < hi[k]) {
        const int64_t mid = lo[k] + ((hi[k] - lo[k]) >> 1);
        if (list[mid] < key) lo[k] = mid + 1; else hi[k] = mid;
      }
    }
  }
  int64_t place = begin * length;
#pragma unroll
  for (int k = 0; k < kMergeWays; ++k) {
    const int64_t a = (begin + k) * length;
    place += lo[k] - (a < num_tokens ? a : num_tokens);
  }
  to[static_cast<int64_t>(blockIdx.y) * num_tokens + place] = key;
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------

template <typename Table, int N>
__device__ __forceinline__ void finish_row(const EmbedArgs& a, int64_t w, uint32_t token, uint32_t c, const float* sum) {
  Table* at = static_cast<Table*>(a.table) + w * a.stride + static_cast<int64_t>(token) * a.width + c;
  Numbers<Table, N> x;
  if (a.accumulate) x.load(at); else x.zero();
#pragma unroll
  for (int k = 0; k < N; ++k) x.v[k] += a.scale * sum[k];
  x.store(at);
}

// A workgroup takes 32 sorted pairs and 256 * N columns.  A token whose pairs all lie in the chunk is finished here;
// the sum of one that the chunk before began goes to slot 0 of the chunk's partial rows, of one that goes on in
// the next chunk to slot 1 (one that does both: slot 0).
template <typename Table, typename Row, int N>
__global__ __launch_bounds__(256) void embed_sums(EmbedArgs a, const uint64_t* sorted, uint32_t chunks) {
  __shared__ uint64_t key[kSumChunk + 2];       // with the pairs before and after
  const int64_t w = blockIdx.y, T = a.num_tokens;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSumChunk;
  const uint64_t* list = sorted + w * T;
  if (threadIdx.x < kSumChunk + 2) {
    const int64_t p = first + threadIdx.x - 1;
    key[threadIdx.x] = p >= 0 && p < T ? list[p] : ~0ull;
  }
  __syncthreads();
  const uint32_t c = (blockIdx.z * 256 + threadIdx.x) * N;
  if (c >= a.width) return;
  const Row* rows = static_cast<const Row*>(a.rows) + w * T * a.width + c;
  float* partial = a.partial + ((w * chunks + blockIdx.x) * 2) * static_cast<int64_t>(a.width) + c;
  float sum[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = 0.f;
  const uint32_t before = static_cast<uint32_t>(key[0] >> 32);
  bool from_before = false;
  constexpr int kAhead = 8;
  for (int b = 0; b < kSumChunk; b += kAhead) {
    Numbers<Row, N> x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint64_t at = key[1 + b + k];
      if (static_cast<uint32_t>(at >> 32) < a.vocab) x[k].load(rows + static_cast<int64_t>(static_cast<uint32_t>(at)) * a.width);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t token = static_cast<uint32_t>(key[1 + b + k] >> 32), next = static_cast<uint32_t>(key[2 + b + k] >> 32);
      if (token < a.vocab) {
        if (b + k == 0) from_before = first > 0 && before == token;
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += x[k].v[i];
        const bool last_here = b + k == kSumChunk - 1;
        if (next != token || last_here) {
          const bool goes_on = next == token;
          if (from_before || goes_on) {
            Numbers<float, N> y;
#pragma unroll
            for (int i = 0; i < N; ++i) y.v[i] = sum[i];
            y.store(partial + (from_before ? 0 : a.width));
          } else {
            finish_row<Table, N>(a, w, token, c, sum);
          }
          from_before = false;
#pragma unroll
          for (int i = 0; i < N; ++i) sum[i] = 0.f;
        }
      }
    }
  }
}

// Joins the partial sums of the token that begins in a chunk and goes on beyond it.
template <typename Table, int N>
__global__ __launch_bounds__(256) void embed_join(EmbedArgs a, const uint64_t* sorted, uint32_t chunks) {
  const int64_t w = blockIdx.y, T = a.num_tokens;
  const uint64_t* list = sorted + w * T;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSumChunk, next = first + kSumChunk;
  if (next >= T) return;
  const uint32_t token = static_cast<uint32_t>(list[next - 1] >> 32);
  if (token >= a.vocab || static_cast<uint32_t>(list[next] >> 32) != token) return;                // nothing goes on
  if (first > 0 && static_cast<uint32_t>(list[first] >> 32) == token && static_cast<uint32_t>(list[first - 1] >> 32) == token) return;   // began earlier
  // where it ends
  int64_t lo = next, hi = T;
  while (lo < hi) {
    const int64_t mid = lo + ((hi - lo) >> 1);
    if (static_cast<uint32_t>(list[mid] >> 32) <= token) lo = mid + 1; else hi = mid;
  }
  const int64_t last = (lo - 1) / kSumChunk;
  const uint32_t c = (blockIdx.z * 256 + threadIdx.x) * N;
  if (c >= a.width) return;
  const float* partial = a.partial + (w * chunks * 2) * static_cast<int64_t>(a.width) + c;
  Numbers<float, N> sum;
  sum.load(partial + (static_cast<int64_t>(blockIdx.x) * 2 + 1) * a.width);
#pragma unroll 8
  for (int64_t k = static_cast<int64_t>(blockIdx.x) + 1; k <= last; ++k) {
    Numbers<float, N> x;
    x.load(partial + k * 2 * a.width);
#pragma unroll
    for (int i = 0; i < N; ++i) sum.v[i] += x.v[i];
  }
  finish_row<Table, N>(a, w, token, c, sum.v);
}

// Zeros in the rows of tokens that do not come up; a workgroup takes 64 rows of the table.
template <typename Table, int N>
__global__ __launch_bounds__(256) void embed_zero(EmbedArgs a, const uint64_t* sorted) {
  __shared__ int64_t edge[65];
  const int64_t w = blockIdx.y, T = a.num_tokens;
  const uint64_t* list = sorted + w * T;
  const uint32_t v0 = blockIdx.x * 64;
  if (threadIdx.x < 65) {
    const uint64_t key = static_cast<uint64_t>(v0 + threadIdx.x) << 32;
    int64_t lo = 0, hi = T;
    while (lo < hi) {
      const int64_t mid = lo + ((hi - lo) >> 1);
      if (list[mid] < key) lo = mid + 1; else hi = mid;
    }
    edge[threadIdx.x] = lo;
  }
  __syncthreads();
  Numbers<Table, N> none;
  none.zero();
  for (uint32_t r = threadIdx.x >> 6; r < 64 && v0 + r < a.vocab; r += 4) {
    if (edge[r] != edge[r + 1]) continue;
    Table* at = static_cast<Table*>(a.table) + w * a.stride + static_cast<int64_t>(v0 + r) * a.width;
    for (uint32_t c = (threadIdx.x & 63) * N; c < a.width; c += 64 * N) none.store(at + c);
  }
}

template <typename Table, typename Row, int N> int lookup(const EmbedArgs& a, void* stream) {
  const int64_t all = static_cast<int64_t>(a.W) * a.num_tokens, groups = (all + 3) / 4;
  return enqueue(embed_lookup<Table, Row, N>, dim3(static_cast<uint32_t>(groups < (1 << 22) ? groups : 1 << 22)), 256, stream, a);
}

template <typename Table, typename Row, int N> int gradient(const EmbedArgs& a, void* stream) {
  const int64_t T = a.num_tokens;
  const uint32_t W = static_cast<uint32_t>(a.W);
  int at = 0;
  if (T > 0) {
    const uint32_t lists = static_cast<uint32_t>((T + kSortChunk - 1) / kSortChunk);
    int st = enqueue(embed_sort, dim3(lists, W), 1024, stream, a, a.sorted[0]);
    if (st != 0) return st;
    for (int64_t length = kSortChunk; length < T; length *= kMergeWays) {
      st = enqueue(embed_merge, dim3(static_cast<uint32_t>((T + 255) / 256), W), 256, stream, a.sorted[at], a.sorted[at ^ 1], T, length);
      if (st != 0) return st;
      at ^= 1;
    }
  }
  const uint64_t* sorted = a.sorted[at];
  if (!a.accumulate) {
    const int st = enqueue(embed_zero<Table, N>, dim3((a.vocab + 63) / 64, W), 256, stream, a, sorted);
    if (st != 0) return st;
  }
  if (T == 0) return 0;
  const uint32_t chunks = static_cast<uint32_t>((T + kSumChunk - 1) / kSumChunk);
  const dim3 grid(chunks, W, (a.width + 256 * N - 1) / (256 * N));
  const int st = enqueue(embed_sums<Table, Row, N>, grid, 256, stream, a, sorted, chunks);
  return st != 0 ? st : enqueue(embed_join<Table, N>, grid, 256, stream, a, sorted, chunks);
}

}  // namespace

int launch_embed_lookup(const EmbedArgs& a, void* stream) {
  if (a.vectors)
    return a.table_bf16 ? (a.rows_bf16 ? lookup<uint16_t, uint16_t, 4>(a, stream) : lookup<uint16_t, float, 4>(a, stream))
                        : (a.rows_bf16 ? lookup<float, uint16_t, 4>(a, stream) : lookup<float, float, 4>(a, stream));
  return a.table_bf16 ? (a.rows_bf16 ? lookup<uint16_t, uint16_t, 1>(a, stream) : lookup<uint16_t, float, 1>(a, stream))
                      : (a.rows_bf16 ? lookup<float, uint16_t, 1>(a, stream) : lookup<float, float, 1>(a, stream));
}

int launch_embed_gradient(const EmbedArgs& a, void* stream) {
  if (a.vectors)
    return a.table_bf16 ? (a.rows_bf16 ? gradient<uint16_t, uint16_t, 4>(a, stream) : gradient<uint16_t, float, 4>(a, stream))
                        : (a.rows_bf16 ? gradient<float, uint16_t, 4>(a, stream) : gradient<float, float, 4>(a, stream));
  return a.table_bf16 ? (a.rows_bf16 ? gradient<uint16_t, uint16_t, 1>(a, stream) : gradient<uint16_t, float, 1>(a, stream))
                      : (a.rows_bf16 ? gradient<float, uint16_t, 1>(a, stream) : gradient<float, float, 1>(a, stream));
}

}  // namespace noloco
