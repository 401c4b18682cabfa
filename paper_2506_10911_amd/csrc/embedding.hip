// Embedding lookup and its gradient (kernels and their launchers).
//
//   lookup     out[w][t] = scale * table_w[tokens[w][t]]
//   gradient   grad_w[v] = (accumulate ? grad_w[v] : 0) + scale * sum of dout[w][t] over the t with tokens[w][t] = v
//
// Both are bound by memory.  The gradient's rows are found by sorting (token, position) pairs: lists of 2048 are sorted by a
// workgroup each, and sixteen lists at a time are joined by ranks (a pair's place is its place in its own list plus the number
// of smaller pairs in each other list).  No atomics anywhere: a row's sum is taken in the order of positions, in chunks
// of 32 sorted pairs whose sums are joined in order.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "inner_internal.h"

namespace noloco {
namespace {

template <typename T> struct same { typedef T type; };
template <typename... KArgs>
int enqueue(void (*kernel)(KArgs...), dim3 grid, uint32_t block, uint32_t lds, void* stream, typename same<KArgs>::type... args) {
  void* argv[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), argv, lds, static_cast<hipStream_t>(stream));
}

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ uint16_t narrow(float v) {   // to bf16, nearest, ties to even; NaN stays NaN
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// N neighbouring numbers of type E (float, or bf16 as stored) as floats, in vectors of four, or eight bf16.
template <typename E, int N> struct Numbers {
  static constexpr int kVector = N == 1 ? 1 : (sizeof(E) == 2 && N % 8 == 0 ? 8 : 4);
  typedef E vector __attribute__((ext_vector_type(kVector)));
  float v[N];
  __device__ __forceinline__ void load(const E* p) {
#pragma unroll
    for (int i = 0; i < N; i += kVector) {
      E raw[kVector];
      if constexpr (kVector == 1) {
        raw[0] = *p;
      } else {
        const vector x = *reinterpret_cast<const vector*>(p + i);
#pragma unroll
        for (int k = 0; k < kVector; ++k) raw[k] = x[k];
      }
#pragma unroll
      for (int k = 0; k < kVector; ++k) {
        if constexpr (sizeof(E) == 2) v[i + k] = widen(raw[k]); else v[i + k] = raw[k];
      }
    }
  }
  __device__ __forceinline__ void store(E* p) const {
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
        *reinterpret_cast<vector*>(p + i) = x;
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
  }
};

template <int N> struct Number { static constexpr int value = N; };

// A token's row, or vocab for one that has none.
__device__ __forceinline__ uint32_t token_at(const EmbedArgs& a, int64_t i) {
  const int64_t token = a.tokens_i64 ? static_cast<const int64_t*>(a.tokens)[i] : static_cast<const int32_t*>(a.tokens)[i];
  return token >= 0 && token < static_cast<int64_t>(a.vocab) ? static_cast<uint32_t>(token) : a.vocab;
}

// A wave takes four tokens at a time, whose rows are asked for together (one at a time 46 us where four take 43).  Bound by memory:
// 8 x 8192 rows of 768, float to bf16, 40 us; what is written and the different rows that are read are 190 MB, 4.8 TB/s.
template <typename Table, typename Row, int N>
__global__ __launch_bounds__(256) void embed_lookup(EmbedArgs a) {
  constexpr int kTokens = 4;
  const int64_t all = static_cast<int64_t>(a.W) * a.num_tokens;
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  static_assert(kLookupTokens == 4 * kTokens, "tokens of a workgroup");
  const int64_t first = ((static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 4 + wave) * kTokens;
  if (first >= all) return;
  const uint32_t mine = first + lane < all && lane < kTokens ? token_at(a, first + lane) : a.vocab;
  const Table* from[kTokens];
  bool there[kTokens];
#pragma unroll
  for (int k = 0; k < kTokens; ++k) {
    const uint32_t token = __builtin_amdgcn_readlane(mine, k);
    const int64_t w = static_cast<uint64_t>(first + k) / static_cast<uint64_t>(a.num_tokens);
    there[k] = token < a.vocab;
    from[k] = static_cast<const Table*>(a.table) + (there[k] ? w * a.stride + static_cast<int64_t>(token) * a.width : 0);
  }
  Row* const to = static_cast<Row*>(a.rows) + first * a.width;
  for (uint32_t c = lane * N; c < a.width; c += 64 * N) {
    Numbers<Table, N> x[kTokens];
#pragma unroll
    for (int k = 0; k < kTokens; ++k) x[k].load(from[k] + c);
#pragma unroll
    for (int k = 0; k < kTokens; ++k) {
      if (first + k >= all) break;
      Numbers<Row, N> y;
#pragma unroll
      for (int i = 0; i < N; ++i) y.v[i] = there[k] ? x[k].v[i] * a.scale : 0.f;
      y.store(to + k * static_cast<int64_t>(a.width) + c);
    }
  }
}

// ---------------------------------------------------------------------------
// Sorting
// ---------------------------------------------------------------------------

// The key of the lane whose number differs by GAP.
template <int GAP> __device__ __forceinline__ uint32_t across(uint32_t v) {
  auto moved = [](uint32_t x, auto control) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(control)::value, 15, 15, false));
  };
  if constexpr (GAP == 1) return moved(v, Number<0xB1>{});                              // quads 1 0 3 2
  else if constexpr (GAP == 2) return moved(v, Number<0x4E>{});                         // quads 2 3 0 1
  else if constexpr (GAP == 4) return moved(moved(v, Number<0x141>{}), Number<0x1B>{}); // eights mirrored, then quads
  else if constexpr (GAP == 8) return moved(v, Number<0x128>{});                        // sixteens turned by 8
  else return __shfl_xor(v, GAP);
}
template <int GAP> __device__ __forceinline__ uint64_t across(uint64_t v) {
  return static_cast<uint64_t>(across<GAP>(static_cast<uint32_t>(v >> 32))) << 32 | across<GAP>(static_cast<uint32_t>(v));
}

// A workgroup sorts up to 2048 positions of one worker: a bitonic network over (token, position in the list), keys of 32 bits
// where tokens leave eleven for the position.  A thread holds places 128 wave + lane and 64 more, so that only places at
// least 128 apart meet in the LDS, ten of the network's 66 stages; the others are a few instructions each (all stages in the
// LDS took 16 us).  Bound by the network's chain: 8 x 8192 positions 10.8 us, with keys of 64 bits 17; a few microseconds fewer
// where there are less.
template <typename Key>
__global__ __launch_bounds__(kSortChunk / 2) void embed_sort(EmbedArgs a) {
  constexpr uint32_t kPlaceBits = 11;
  static_assert(kSortChunk == 1 << kPlaceBits, "places");
  __shared__ Key shared[kSortChunk];
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortChunk, row = static_cast<int64_t>(blockIdx.y) * a.num_tokens;
  const uint32_t lane = threadIdx.x & 63, places = 2 * blockDim.x;
  const uint32_t place[2] = {(threadIdx.x >> 6) * 128 + lane, (threadIdx.x >> 6) * 128 + lane + 64};
  Key key[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    key[h] = first + place[h] < a.num_tokens ? static_cast<Key>(token_at(a, row + first + place[h])) << kPlaceBits | place[h] : ~static_cast<Key>(0);
  auto keep = [](Key mine, Key other, bool smaller) { return (mine < other) == smaller ? mine : other; };
  auto lanes = [&](auto gap, uint32_t size) {
    constexpr uint32_t kGap = decltype(gap)::value;
    if (size <= kGap) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) key[h] = keep(key[h], across<static_cast<int>(kGap)>(key[h]), ((place[h] & size) == 0) == ((lane & kGap) == 0));
  };
  for (uint32_t size = 2; size <= places; size *= 2) {
    for (uint32_t gap = size / 2; gap >= 128; gap /= 2) {
      __syncthreads();
#pragma unroll
      for (int h = 0; h < 2; ++h) shared[place[h]] = key[h];
      __syncthreads();
#pragma unroll
      for (int h = 0; h < 2; ++h) key[h] = keep(key[h], shared[place[h] ^ gap], ((place[h] & size) == 0) == ((place[h] & gap) == 0));
    }
    if (size >= 128) {
      const bool up = (place[0] & size) == 0;
      const Key x = key[0], y = key[1];
      key[0] = keep(x, y, up);
      key[1] = keep(y, x, !up);
    }
    lanes(Number<32>{}, size);
    lanes(Number<16>{}, size);
    lanes(Number<8>{}, size);
    lanes(Number<4>{}, size);
    lanes(Number<2>{}, size);
    lanes(Number<1>{}, size);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (first + place[h] < a.num_tokens) {
      a.token[0][row + first + place[h]] = static_cast<uint32_t>(key[h] >> kPlaceBits);
      a.position[0][row + first + place[h]] = static_cast<uint32_t>(first) + static_cast<uint32_t>(key[h] & (kSortChunk - 1));
    }
}

// Joins up to 16 sorted lists of `length` tokens each, which are of consecutive positions: a token's place is its place in
// its own list, the number of tokens not above it in each list before and of those below it in each list behind.
template <typename Tokens>
__device__ __forceinline__ int64_t merged_place(Tokens list, int64_t count, int64_t length, int64_t p, uint32_t token) {
  const int64_t mine = p / length;
  int64_t lo[kMergeWays], hi[kMergeWays];
#pragma unroll
  for (int k = 0; k < kMergeWays; ++k) {
    const int64_t a = k * length, b = a + length;
    lo[k] = a < count ? a : count;
    hi[k] = k == mine ? lo[k] : (b < count ? b : count);
  }
  // sixteen searches side by side
  for (int64_t span = length; span > 0; span >>= 1) {
#pragma unroll
    for (int k = 0; k < kMergeWays; ++k) {
      if (lo[k] < hi[k]) {
        const int64_t mid = lo[k] + ((hi[k] - lo[k]) >> 1);
        const uint32_t other = list[mid];
        if (other < token || (other == token && k < mine)) lo[k] = mid + 1; else hi[k] = mid;
      }
    }
  }
  int64_t place = p - mine * length;
#pragma unroll
  for (int k = 0; k < kMergeWays; ++k)
    if (k != mine) place += lo[k] - (k * length < count ? k * length : count);
  return place;
}

// Lists that fit the LDS together.  The tokens of a wave lie between its first and its last one, and so do their places in
// every other list: thirty-two lanes find these, and each lane searches between them only.  Bound by the searches' LDS reads:
// 8 x 8192 positions 8.7 us, 2 x 32768 26.
__global__ __launch_bounds__(1024) void embed_merge_lds(const uint32_t* token_in, const uint32_t* position_in, uint32_t* token_out,
                                                        uint32_t* position_out, int64_t num_tokens) {
  extern __shared__ uint32_t tokens[];
  const int64_t row = static_cast<int64_t>(blockIdx.y) * num_tokens;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 1024, group = at / kMergeChunk * kMergeChunk;
  const uint32_t count = static_cast<uint32_t>(num_tokens - group < kMergeChunk ? num_tokens - group : kMergeChunk);
  for (uint32_t i = threadIdx.x; i < count; i += 1024) tokens[i] = token_in[row + group + i];
  __syncthreads();
  const uint32_t lane = threadIdx.x & 63, wave_at = static_cast<uint32_t>(at - group) + (threadIdx.x & ~63u);
  if (wave_at >= count) return;
  const uint32_t p = wave_at + lane < count ? wave_at + lane : count - 1;
  const uint32_t mine = p / kSortChunk, token = tokens[p], lists = (count + kSortChunk - 1) / kSortChunk;
  // lane k: how many in list k come before the wave's first token; lane 16 + k: before its last one
  uint32_t edge;
  {
    const uint32_t k = lane & 15, limit = lane < 16 ? tokens[wave_at] : tokens[wave_at + 63 < count ? wave_at + 63 : count - 1];
    uint32_t lo = min(k * kSortChunk, count), hi = min(lo + kSortChunk, count);
    while (lo < hi) {
      const uint32_t mid = (lo + hi) >> 1, other = tokens[mid];
      if (other < limit || (other == limit && k < mine)) lo = mid + 1; else hi = mid;
    }
    edge = lo;
  }
  uint32_t place = p % kSortChunk;
  for (uint32_t first = 0; first < lists; first += 4) {
    uint32_t lo[4], hi[4], most = 0;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      lo[k] = __builtin_amdgcn_readlane(edge, first + k);
      hi[k] = first + k == mine ? lo[k] : __builtin_amdgcn_readlane(edge, 16 + first + k);
      most = max(most, hi[k] - lo[k]);
    }
    for (; most > 0; most >>= 1) {
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        if (lo[k] < hi[k]) {
          const uint32_t mid = (lo[k] + hi[k]) >> 1, other = tokens[mid];
          if (other < token || (other == token && first + k < mine)) lo[k] = mid + 1; else hi[k] = mid;
        }
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
      if (first + k != mine) place += lo[k] - min((first + k) * kSortChunk, count);
  }
  if (wave_at + lane < count) {
    token_out[row + group + place] = token;
    position_out[row + group + place] = position_in[row + group + p];
  }
}

// Longer ones, which do not fit: every search goes to memory.  2 x 200000 positions, the second of two joins, 52 us.
__global__ __launch_bounds__(256) void embed_merge(const uint32_t* token_in, const uint32_t* position_in, uint32_t* token_out,
                                                   uint32_t* position_out, int64_t num_tokens, int64_t length) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (at >= num_tokens) return;
  const int64_t row = static_cast<int64_t>(blockIdx.y) * num_tokens, group = at / (length * kMergeWays) * (length * kMergeWays);
  const int64_t count = num_tokens - group < length * kMergeWays ? num_tokens - group : length * kMergeWays;
  const uint32_t token = token_in[row + at];
  const int64_t place = merged_place(token_in + row + group, count, length, at - group, token);
  token_out[row + group + place] = token;
  position_out[row + group + place] = position_in[row + at];
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------

// Lists that no kernel of the launch writes are read through the scalar cache: their entries steer whole workgroups.
#define scalar_memory __attribute__((address_space(4)))

// One row of the table: what was there, if it is added to, and the sum times the scale.
template <typename Table, int N>
__device__ __forceinline__ void finish_row(const EmbedArgs& a, Table* at, const Numbers<Table, N>& old, const float* sum) {
  Numbers<Table, N> x;
#pragma unroll
  for (int k = 0; k < N; ++k) x.v[k] = (a.accumulate ? old.v[k] : 0.f) + a.scale * sum[k];
  x.store(at);
}

// A workgroup takes 32 sorted positions and 256 * N columns.  A token whose positions all lie in the chunk is finished here;
// the sum of one that the chunk before began goes to slot 0 of the chunk's partial rows, of one that goes on in
// the next chunk to slot 1 (one that does both: slot 0).  Workgroups beyond the chunks write zeros to 64 rows of the table
// each, those of tokens that do not come up.  Which of them do is looked up in the sorted list, so that no memory is cleared
// and then written.  Bound by memory: 2 x 32768 rows of 4096, bf16, into a table of 50257 rows 277 us, 4.9 TB/s; 8 x 8192 rows of
// 768 added to what is there 55 us.  Chunks of 32: a token that comes up often is spread over many workgroups.
template <typename Table, typename Row, int N>
__global__ __launch_bounds__(256) void embed_sums(EmbedArgs a, const uint32_t* token_list, const uint32_t* position_list, uint32_t chunks) {
  const int64_t w = blockIdx.y, T = a.num_tokens;
  const scalar_memory uint32_t* tokens = (const scalar_memory uint32_t*)(token_list + w * T);
  const scalar_memory uint32_t* positions = (const scalar_memory uint32_t*)(position_list + w * T);
  Table* const table = static_cast<Table*>(a.table) + w * a.stride;
  if (blockIdx.x >= chunks) {
    if (blockIdx.z > 0) return;
    __shared__ int64_t edge[65];
    const uint32_t v0 = (blockIdx.x - chunks) * 64;
    if (threadIdx.x < 65) {
      const uint32_t* list = token_list + w * T;
      int64_t lo = 0, hi = T;
      while (lo < hi) {
        const int64_t mid = lo + ((hi - lo) >> 1);
        if (list[mid] < v0 + threadIdx.x) lo = mid + 1; else hi = mid;
      }
      edge[threadIdx.x] = lo;
    }
    __syncthreads();
    Numbers<Table, N> none;
    none.zero();
    for (uint32_t r = threadIdx.x >> 6; r < 64 && v0 + r < a.vocab; r += 4) {
      if (edge[r] != edge[r + 1]) continue;
      Table* at = table + static_cast<int64_t>(v0 + r) * a.width;
      for (uint32_t c = (threadIdx.x & 63) * N; c < a.width; c += 64 * N) none.store(at + c);
    }
    return;
  }
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSumChunk;
  const int count = static_cast<int>(T - first < kSumChunk ? T - first : kSumChunk);
  const uint32_t c = (blockIdx.z * 256 + threadIdx.x) * N;
  const bool mine = c < a.width;
  const uint32_t at = mine ? c : 0;               // threads beyond the row's end load its first numbers and store nothing
  const Row* rows = static_cast<const Row*>(a.rows) + w * T * a.width + at;
  float* partial = a.partial + ((w * chunks + blockIdx.x) * 2) * static_cast<int64_t>(a.width) + at;
  float sum[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = 0.f;
  bool from_before = first > 0 && tokens[first - 1] == tokens[first];
  constexpr int kAhead = 8;
  for (int b = 0; b < count; b += kAhead) {
    uint32_t token[kAhead + 1];
    Numbers<Row, N> x[kAhead];
    Numbers<Table, N> old[kAhead];
#pragma unroll
    for (int k = 0; k <= kAhead; ++k) token[k] = first + b + k < T ? tokens[first + b + k] : ~0u;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool there = token[k] < a.vocab;
      x[k].load(rows + (there ? static_cast<int64_t>(positions[first + b + k]) * a.width : 0));
      if (a.accumulate && there && token[k + 1] != token[k]) old[k].load(table + static_cast<int64_t>(token[k]) * a.width + at);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (token[k] >= a.vocab || b + k >= count) break;
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += x[k].v[i];
      const bool goes_on = token[k + 1] == token[k];
      if (!goes_on || b + k == kSumChunk - 1) {
        if (from_before || goes_on) {
          Numbers<float, N> y;
#pragma unroll
          for (int i = 0; i < N; ++i) y.v[i] = sum[i];
          if (mine) y.store(partial + (from_before ? 0 : a.width));
        } else if (mine) {
          finish_row<Table, N>(a, table + static_cast<int64_t>(token[k]) * a.width + at, old[k], sum);
        }
        from_before = false;
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.f;
      }
    }
  }
}

// Joins the partial sums of the token that begins in a chunk and goes on beyond it, in order, sixteen on their way at a time.
// The most frequent token is what it waits for: 8 x 8192 positions 6 us, 2 x 32768 rows of 4096 20.
template <typename Table, int N>
__global__ __launch_bounds__(256) void embed_join(EmbedArgs a, const uint32_t* token_list, uint32_t chunks) {
  const int64_t w = blockIdx.y, T = a.num_tokens;
  const scalar_memory uint32_t* tokens = (const scalar_memory uint32_t*)(token_list + w * T);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSumChunk, next = first + kSumChunk;
  if (next >= T) return;
  const uint32_t token = tokens[next - 1];
  if (token >= a.vocab || tokens[next] != token) return;                                         // nothing goes on
  if (first > 0 && tokens[first] == token && tokens[first - 1] == token) return;                 // began earlier
  // the last chunk that begins with it: a wave looks at 64 at a time
  const uint32_t lane = threadIdx.x & 63;
  int64_t last = blockIdx.x;
  while (true) {
    const int64_t chunk = last + 1 + lane;
    const uint64_t others = __ballot(!(chunk * kSumChunk < T && token_list[w * T + chunk * kSumChunk] == token));
    if (others != 0) {
      last += __builtin_ctzll(others);
      break;
    }
    last += 64;
  }
  const uint32_t c = (blockIdx.z * 256 + threadIdx.x) * N;
  if (c >= a.width) return;
  const float* partial = a.partial + (w * chunks * 2) * static_cast<int64_t>(a.width) + c;
  Table* const at = static_cast<Table*>(a.table) + w * a.stride + static_cast<int64_t>(token) * a.width + c;
  Numbers<Table, N> old;
  if (a.accumulate) old.load(at);
  Numbers<float, N> sum;
  sum.load(partial + (static_cast<int64_t>(blockIdx.x) * 2 + 1) * a.width);
  int64_t k = static_cast<int64_t>(blockIdx.x) + 1;
  constexpr int kAhead = 16;
  for (; k + kAhead - 1 <= last; k += kAhead) {
    Numbers<float, N> x[kAhead];
#pragma unroll
    for (int b = 0; b < kAhead; ++b) x[b].load(partial + (k + b) * 2 * a.width);
#pragma unroll
    for (int b = 0; b < kAhead; ++b)
#pragma unroll
      for (int i = 0; i < N; ++i) sum.v[i] += x[b].v[i];
  }
  for (; k <= last; ++k) {
    Numbers<float, N> x;
    x.load(partial + k * 2 * a.width);
#pragma unroll
    for (int i = 0; i < N; ++i) sum.v[i] += x.v[i];
  }
  finish_row<Table, N>(a, at, old, sum.v);
}

template <typename Table, typename Row, int N> int lookup(const EmbedArgs& a, void* stream) {
  const LookupGrid grid = lookup_grid(static_cast<int64_t>(a.W) * a.num_tokens);
  return enqueue(embed_lookup<Table, Row, N>, dim3(grid.x, grid.y), 256, 0, stream, a);
}

template <typename Table, typename Row, int N> int gradient(const EmbedArgs& a, void* stream) {
  const int64_t T = a.num_tokens;
  const uint32_t W = static_cast<uint32_t>(a.W);
  int at = 0;
  if (T > 0) {
    // a network of as many places as there are positions, and a wave of threads at least
    uint32_t threads = 64;
    while (threads < kSortChunk / 2 && 2 * threads < T) threads *= 2;
    int st = enqueue(a.vocab < (1u << 21) ? embed_sort<uint32_t> : embed_sort<uint64_t>,
                     dim3(static_cast<uint32_t>((T + kSortChunk - 1) / kSortChunk), W), threads, 0, stream, a);
    if (st != 0) return st;
    for (int64_t length = kSortChunk; length < T; length *= kMergeWays) {
      st = length == kSortChunk
               ? enqueue(embed_merge_lds, dim3(static_cast<uint32_t>((T + 1023) / 1024), W), 1024,
                         static_cast<uint32_t>((T < kMergeChunk ? T : kMergeChunk) * sizeof(uint32_t)), stream, a.token[at], a.position[at],
                         a.token[at ^ 1], a.position[at ^ 1], T)
               : enqueue(embed_merge, dim3(static_cast<uint32_t>((T + 255) / 256), W), 256, 0, stream, a.token[at], a.position[at],
                         a.token[at ^ 1], a.position[at ^ 1], T, length);
      if (st != 0) return st;
      at ^= 1;
    }
  }
  const uint32_t chunks = static_cast<uint32_t>((T + kSumChunk - 1) / kSumChunk), wide = (a.width + 256 * N - 1) / (256 * N);
  const uint32_t zeros = a.accumulate ? 0 : (a.vocab + 63) / 64;
  const int st = enqueue(embed_sums<Table, Row, N>, dim3(chunks + zeros, W, wide), 256, 0, stream, a, a.token[at], a.position[at], chunks);
  if (st != 0 || chunks < 2) return st;
  return enqueue(embed_join<Table, N>, dim3(chunks - 1, W, wide), 256, 0, stream, a, a.token[at], chunks);
}

}  // namespace

// Types, and how many columns a thread takes: eight where bf16 is read and all is aligned for it, four where it is for that.
template <template <typename, typename, int> class What> static int by_types(const EmbedArgs& a, bool eight, void* stream) {
  auto with = [&](auto table, auto row) {
    typedef decltype(table) Table;
    typedef decltype(row) Row;
    if (a.vectors == 8 && eight) return What<Table, Row, 8>::run(a, stream);
    if (a.vectors >= 4) return What<Table, Row, 4>::run(a, stream);
    return What<Table, Row, 1>::run(a, stream);
  };
  if (a.table_bf16) return a.rows_bf16 ? with(uint16_t{}, uint16_t{}) : with(uint16_t{}, float{});
  return a.rows_bf16 ? with(float{}, uint16_t{}) : with(float{}, float{});
}
template <typename Table, typename Row, int N> struct Lookup {
  static int run(const EmbedArgs& a, void* stream) { return lookup<Table, Row, N>(a, stream); }
};
template <typename Table, typename Row, int N> struct Gradient {
  static int run(const EmbedArgs& a, void* stream) { return gradient<Table, Row, N>(a, stream); }
};

int launch_embed_lookup(const EmbedArgs& a, void* stream) { return by_types<Lookup>(a, a.table_bf16 != 0, stream); }
int launch_embed_gradient(const EmbedArgs& a, void* stream) { return by_types<Gradient>(a, a.rows_bf16 != 0, stream); }

}  // namespace noloco
