// Log probabilities of tokens, entropy and the likeliest alternatives, and their gradient (kernels and their launchers).
//
//   n = log sum exp(l),  log_prob = l[token] - n,  entropy = -sum p log p with p = exp(l - n)
//   dl[v] = dlog_prob ([v = token] - p[v]) - dentropy p[v] (log p[v] + entropy)
//
// Bound by memory: logits are read once each way (8 x 1024 rows of 50257 bf16 151 us, 5.5 TB/s; their gradient, which is read and
// written past the caches, 308, 5.3 TB/s; through them 327).  A row is read in one pass with sums relative to a reference that
// follows the largest logit at a distance of at most 16 (exp of that times a row's length is far from binary32's range),
// so that a new largest one hardly ever costs a correction.  Where one logit has most of the probability the sum is 1 and a rest,
// and log(1 + rest) needs the rest's own digits: such a row is read a second time, from the caches, and only its rest is summed.
//
// Alternatives: each thread keeps its largest logit.  Sixty-four groups of threads have 64 largest ones, and the top-th of
// these is a bound that at least `top` logits reach and few others do; the threads that have such look for them once more.
// Order is that of a 64-bit key, the logit's bits in an order of integers above the inverted place: all keys differ.
#include "device_numbers.h"
#include "model_internal.h"

namespace noloco {
namespace {

constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFollow = 16.f;              // how far the largest logit may be above the reference
constexpr float kInfinity = __builtin_inff();

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

__device__ __forceinline__ uint64_t key_of(float v, uint32_t at) {
  v = v == v ? v + 0.f : -kInfinity;
  const uint32_t u = __float_as_uint(v);
  return static_cast<uint64_t>(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | ~at;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t u = static_cast<uint32_t>(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ int64_t token_of(const LogProbArgs& a, int64_t row) {
  const int64_t t = a.tokens_i64 ? static_cast<const int64_t*>(a.tokens)[row] : static_cast<const int32_t*>(a.tokens)[row];
  return t >= 0 && t < static_cast<int64_t>(a.vocab) ? t : -1;
}

// What a call returns of a row, from its largest logit, the rest and the spread.
struct RowEnd {
  float largest, log_total;        // log(1 + rest)
  __device__ __forceinline__ float log_prob(float logit) const { return largest == -kInfinity ? largest : (logit - largest) - log_total; }
};
__device__ __forceinline__ RowEnd finish_row(const LogProbArgs& a, int64_t row, int64_t token, float logit, float largest, float rest, float spread, bool writes) {
  RowEnd end{largest, log1pf(rest)};
  const bool nan = rest != rest, nothing = !nan && largest == -kInfinity;
  if (nan) end.largest = rest;
  if (writes) {
    a.log_probs[row] = token >= 0 ? end.log_prob(logit) : 0.f;
    if (a.norms != nullptr) a.norms[row] = end.largest + end.log_total;
    if (a.entropy != nullptr) a.entropy[row] = nothing ? 0.f : end.log_total + spread / (1.f + rest);
  }
  return end;
}

// L threads take a part of a row; where that is a wave, four waves take four rows.  SPREAD: the entropy is asked for.  256 threads and
// several rows on a CU rather than 1024 and two: a row's barriers then cost others nothing (319 us, so 151).  Few rows are cut
// into parts of 4096 logits and more: four rows of 50257 with eight alternatives 7 us, and 5 for the join.
template <typename E, int L, bool TOP, bool SPREAD>
__global__ __launch_bounds__(L < 256 ? 256 : L) void log_probs_part(LogProbArgs a) {
  constexpr int V = 16 / sizeof(E);          // logits of a load
  constexpr int kAhead = 4;                  // loads of a thread on their way
  constexpr uint32_t kThreads = L < 256 ? 256 : L, kRows = kThreads / L, kWaves = L / 64;
  // candidates: 32 threads' logits in vectors, and all single ones
  constexpr uint32_t kMost = (NOLOCO_MAX_TOP * (L == 64 ? 16 : 64)) + 64;
  __shared__ float shared[4][2 * kWaves];
  __shared__ uint64_t keys[TOP ? kRows : 1][TOP ? L : 1], found[TOP ? kRows : 1][TOP ? kMost : 1];
  __shared__ uint64_t groups[TOP ? kRows : 1][64];
  __shared__ uint32_t found_count[kRows];
  __shared__ uint64_t bound_of[kRows];
  const uint32_t sub = threadIdx.x / L, at = threadIdx.x % L, lane = threadIdx.x & 63;
  auto everyone = [] {
    if constexpr (L > 64) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  auto largest_of_all = [&](float v, float* room) {
    v = wave_largest(v);
    if constexpr (L > 64) {
      if (lane == 0) room[threadIdx.x >> 6] = v;
      __syncthreads();
#pragma unroll
      for (uint32_t i = 0; i < kWaves; ++i) v = fmaxf(v, room[i]);
    }
    return v;
  };

  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + sub; row < a.rows; row += static_cast<int64_t>(gridDim.x) * kRows) {
    const uint32_t begin = blockIdx.y * a.part, end = min(begin + a.part, a.vocab), count = end - begin;
    const E* const from = static_cast<const E*>(a.logits) + row * a.row_stride + begin;
    // up to the first whole vector by single logits, and behind the last
    const uint32_t head = min(static_cast<uint32_t>(-static_cast<int64_t>(reinterpret_cast<uintptr_t>(from) / sizeof(E)) & (V - 1)), count);
    const uint32_t vectors = (count - head) / V, tail = head + vectors * V;
    const E* const body = from + head;
    auto single = [&](uint32_t i) {          // the thread's logit before or behind the vectors
      float v;
      Stored<E, 1>::load(from + i, &v);
      return v;
    };
    const bool in_head = at < head, in_tail = at < count - tail;

    float reference = kLowest, sum = 0.f, spread = 0.f, mine = -kInfinity;
    uint32_t mine_at = 0;                    // 0: in the head, 1 + vector, 1 + vectors: in the tail
    auto take = [&](const float* v, auto n, uint32_t place) {
      constexpr int kN = decltype(n)::value;
      float most = v[0];
#pragma unroll
      for (int i = 1; i < kN; ++i) most = fmaxf(most, v[i]);
      if (__builtin_amdgcn_ballot_w64(most > reference + kFollow) != 0) {
        const float next = fmaxf(reference, most), by = exp_of(reference - next);
        if constexpr (SPREAD) spread = by > 0.f && sum > 0.f ? by * (spread + (next - reference) * sum) : 0.f;     // the distance may be infinite
        sum *= by;
        reference = next;
      }
      if constexpr (TOP) {
        mine_at = most > mine ? place : mine_at;
      }
      mine = fmaxf(mine, most);
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float d = v[i] - reference, e = exp_of(d);
        sum += e;
        if constexpr (SPREAD) spread -= e > 0.f ? e * d : 0.f;
      }
    };
    if (__builtin_amdgcn_ballot_w64(in_head) != 0) {
      const float v = in_head ? single(at) : -kInfinity;
      take(&v, Number<1>{}, 0);
    }
    for (uint32_t first = 0; first < vectors; first += kAhead * L) {
      float v[kAhead][V];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t i = first + k * L + at;
        if (i < vectors) {
          Stored<E, V>::load(body + i * V, v[k]);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) v[k][e] = -kInfinity;
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (first + k * L + (at & ~63u) < vectors) take(v[k], Number<V>{}, first + k * L + at + 1);
    }
    if (__builtin_amdgcn_ballot_w64(in_tail) != 0) {
      const float v = in_tail ? single(tail + at) : -kInfinity;
      take(&v, Number<1>{}, vectors + 1);
    }

    const float largest = largest_of_all(mine, shared[0]);
    const float by = reference > largest ? 1.f : exp_of(reference - largest);
    float sums[2] = {sum * by, by > 0.f && sum > 0.f ? by * (spread + fmaxf(largest - reference, 0.f) * sum) : 0.f};
    sum_all<L, 2>(sums, shared[1]);
    float rest = sums[0] - 1.f;
    spread = sums[1];
    if (largest == -kInfinity && rest == rest) rest = spread = 0.f;
    if (largest != -kInfinity && rest < 1.f) {
      float again[3] = {0.f, 0.f, 0.f};      // the sum of the others, how many are the largest, the spread
      auto add = [&](float l) {
        const float d = l - largest, e = exp_of(d);
        again[0] += d < 0.f ? e : 0.f;
        again[1] += d < 0.f ? 0.f : 1.f;
        again[2] -= e > 0.f ? e * d : 0.f;
      };
      if (in_head) add(single(at));
      for (uint32_t i = at; i < vectors; i += L) {
        float v[V];
        Stored<E, V>::load(body + i * V, v);
#pragma unroll
        for (int e = 0; e < V; ++e) add(v[e]);
      }
      if (in_tail) add(single(tail + at));
      sum_all<L, 2>(again, shared[2]);
      sum_all<L, 1>(again + 2, shared[3]);
      rest = again[0] + (again[1] - 1.f);
      spread = again[2];
    }
    RowEnd row_end{};
    if (a.num_parts == 1) {
      const int64_t token = token_of(a, row);
      float logit = 0.f;
      if (at == 0 && token >= 0) load_numbers<1>(a.logits, row * a.row_stride + token, a.logits_bf16, &logit);
      row_end = finish_row(a, row, token, logit, largest, rest, spread, at == 0);
    } else if (at == 0) {
      a.parts[row * a.num_parts + blockIdx.y] = LogPart{largest, rest, spread, 0.f};
    }

    if constexpr (TOP) {
      const uint32_t top = a.top;
      // the thread's largest logit's key: its place is the first of its vector that is as large
      uint64_t key = 0;
      if (in_head) key = key_of(single(at), begin + at);
      auto better = [&](float v, uint32_t i) {
        const uint64_t other = key_of(v, begin + i);
        key = other > key ? other : key;
      };
      if (mine_at >= 1 && mine_at <= vectors) {
        float v[V];
        Stored<E, V>::load(body + (mine_at - 1) * V, v);
#pragma unroll
        for (int e = 0; e < V; ++e) better(v[e], head + (mine_at - 1) * V + e);
      } else if (mine_at == 0 && at < vectors) {        // all of them -infinity or NaN: the first
        better(-kInfinity, head + at * V);
      }
      if (in_tail) better(single(tail + at), tail + at);
      keys[sub][at] = key;
      if (at == 0) found_count[sub] = 0;
      everyone();
      // the top-th of 64 groups' largest: a wave's lanes find how many are larger than theirs
      if (at < 64) {
        uint64_t group = keys[sub][lane];
#pragma unroll
        for (uint32_t i = 1; i < kWaves; ++i) group = max(group, keys[sub][i * 64 + lane]);
        groups[sub][lane] = group;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        uint32_t larger = 0;
#pragma unroll 16
        for (int j = 0; j < 64; ++j) larger += groups[sub][j] > group ? 1 : 0;
        if (lane == 0) bound_of[sub] = 1;
        if (larger == top - 1 && group != 0) bound_of[sub] = group;
      }
      everyone();
      auto collect = [&](uint64_t bound) {
        if (key >= bound && key != 0) {
          auto offer = [&](float v, uint32_t i) {
            const uint64_t k = key_of(v, begin + i);
            if (k < bound) return;
            const uint32_t place = atomicAdd(&found_count[sub], 1u);
            if (place < kMost) found[sub][place] = k;
          };
          if (in_head) offer(single(at), at);
          for (uint32_t i = at; i < vectors; i += L) {
            float v[V];
            Stored<E, V>::load(body + i * V, v);
#pragma unroll
            for (int e = 0; e < V; ++e) offer(v[e], head + i * V + e);
          }
          if (in_tail) offer(single(tail + at), tail + at);
        }
        everyone();
      };
      collect(bound_of[sub]);
      uint32_t candidates = found_count[sub];
      if (candidates > kMost) {
        // one group has too many: the top-th largest of all threads' keys leaves at most `top` threads
        everyone();
        if (at == 0) found_count[sub] = 0;
        uint32_t larger = 0;
        for (uint32_t j = 0; j < L; ++j) larger += keys[sub][j] > key ? 1 : 0;
        if (larger == top - 1) bound_of[sub] = key;
        everyone();
        collect(bound_of[sub]);
        candidates = found_count[sub];
      }
      for (uint32_t c = at; c < candidates; c += L) {
        const uint64_t k = found[sub][c];
        uint32_t larger = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < candidates; ++j) larger += found[sub][j] > k ? 1 : 0;
        if (larger >= top) continue;
        if (a.num_parts == 1) {
          a.top_tokens[row * top + larger] = static_cast<int32_t>(~static_cast<uint32_t>(k));
          a.top_log_probs[row * top + larger] = row_end.log_prob(logit_of(k));
        } else {
          a.keys[(row * a.num_parts + blockIdx.y) * top + larger] = k;
        }
      }
      for (uint32_t c = candidates + at; c < top; c += L) {
        if (a.num_parts == 1) {
          a.top_tokens[row * top + c] = -1;
          a.top_log_probs[row * top + c] = -kInfinity;
        } else {
          a.keys[(row * a.num_parts + blockIdx.y) * top + c] = 0;
        }
      }
    }
    if constexpr (L > 64) __syncthreads();
  }
}

// A row's parts together, a workgroup a row: the first part that has the largest logit gives its rest, the others all of their sum.
// Rows in parts have more logits than there are alternatives, so that each place is some key's.
constexpr uint32_t kJoinKeys = 1024;
__global__ __launch_bounds__(256) void log_probs_join(LogProbArgs a) {
  __shared__ uint64_t near[kJoinKeys];
  const uint32_t lane = threadIdx.x & 63;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    // every wave for itself up to the alternatives, whose keys come meanwhile
    const int64_t token = token_of(a, row);
    float logit = 0.f;
    if (token >= 0) load_numbers<1>(a.logits, row * a.row_stride + token, a.logits_bf16, &logit);
    const uint32_t top = a.top, all = a.num_parts * top;
    const uint64_t* const keys = a.keys + row * all;
    if (all <= kJoinKeys)
      for (uint32_t c = threadIdx.x; c < all; c += 256) near[c] = keys[c];
    const LogPart* const parts = a.parts + row * a.num_parts;
    float largest = -kInfinity;
    for (uint32_t i = lane; i < a.num_parts; i += 64) largest = fmaxf(largest, parts[i].largest);
    largest = wave_largest(largest);
    uint32_t owner = ~0u;
    for (uint32_t i = lane; i < a.num_parts; i += 64)
      if (parts[i].largest == largest) { owner = i; break; }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) owner = min(owner, static_cast<uint32_t>(__shfl_xor(static_cast<int>(owner), d)));
    float rest = 0.f, spread = 0.f;
    for (uint32_t i = lane; i < a.num_parts; i += 64) {
      const LogPart p = parts[i];
      if (p.largest == -kInfinity) {
        rest += p.rest;                      // zero, or the NaN that a part of nothing else left
        continue;
      }
      const float d = p.largest - largest, e = i == owner ? 1.f : exp_of(d);
      rest += i == owner ? p.rest : (1.f + p.rest) * e;
      spread += e > 0.f ? e * (p.spread - d * (1.f + p.rest)) : 0.f;
    }
    rest = wave_sum(rest);
    spread = wave_sum(spread);
    const RowEnd end = finish_row(a, row, token, logit, largest, rest, spread, threadIdx.x == 0);
    if (top == 0) continue;
    __syncthreads();
    // A key's place is the number of larger ones: counted while there are few, searched in the sorted lists where there are many.
    for (uint32_t c = threadIdx.x; c < all; c += 256) {
      const uint64_t k = keys[c];
      if (k == 0) continue;
      uint32_t larger = 0;
      if (all <= kJoinKeys) {
#pragma unroll 8
        for (uint32_t i = 0; i < all; ++i) larger += near[i] > k ? 1 : 0;
      } else {
        for (uint32_t i = 0; i < a.num_parts && larger < top; ++i) {
          uint32_t lo = 0, hi = top;
          while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (keys[i * top + mid] > k) lo = mid + 1; else hi = mid;
          }
          larger += lo;
        }
      }
      if (larger >= top) continue;
      a.top_tokens[row * top + larger] = static_cast<int32_t>(~static_cast<uint32_t>(k));
      a.top_log_probs[row * top + larger] = end.log_prob(logit_of(k));
    }
    __syncthreads();
  }
}

// A workgroup takes 8192 neighbouring logits of a row, eight of a thread at a time, from a multiple of eight on.
constexpr uint32_t kGradientPart = 8192;
template <typename E, typename Out, bool ENTROPY>
__global__ __launch_bounds__(256) void log_probs_gradient(LogProbArgs a) {
  constexpr int kAhead = kGradientPart / (256 * 8);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    // places count from the last multiple of eight at or before the row's first logit
    const int64_t begin = row * a.row_stride, base = begin / 8 * 8;
    const uint32_t first = static_cast<uint32_t>(begin - base), end = first + a.vocab;
    const int64_t found = token_of(a, row);
    const uint32_t token = found >= 0 ? first + static_cast<uint32_t>(found) : ~0u;
    const float norm = a.norms[row], by = found >= 0 ? a.dlog_probs[row] : 0.f;
    const float of_entropy = ENTROPY ? a.dentropy[row] : 0.f, entropy = ENTROPY ? a.entropy[row] : 0.f;
    const bool nothing = norm == -kInfinity || (found < 0 && !ENTROPY);
    const E* const from = static_cast<const E*>(a.logits) + base;
    Out* const to = static_cast<Out*>(a.dlogits) + base;
    auto slope = [&](float l) {
      const float d = l - norm, p = exp_of(d);
      float v = -by * p;
      if constexpr (ENTROPY) v -= p > 0.f || p != p ? of_entropy * p * (d + entropy) : 0.f;
      return v;
    };
    // 1 - p at the token, also where p is next to 1
    auto at_token = [&](float l) {
      const float d = l - norm, p = exp_of(d);
      float v = by * -expm1f(d);
      if constexpr (ENTROPY) v -= p > 0.f || p != p ? of_entropy * p * (d + entropy) : 0.f;
      return v;
    };
    const uint32_t start = blockIdx.y * kGradientPart + threadIdx.x * 8;
    float v[kAhead][8];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t at = start + k * 256 * 8;
      if (!nothing && at >= first && at + 8 <= end) Stored<E, 8>::load_once(from + at, v[k]);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t at = start + k * 256 * 8;
      if (at >= first && at + 8 <= end) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = nothing ? 0.f : slope(v[k][e]);
        if (!nothing && token - at < 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (token - at == e) x[e] = at_token(v[k][e]);
        }
        Stored<Out, 8>::store_once(to + at, x);
      } else if (at < end) {
        for (uint32_t i = at < first ? first : at; i < at + 8 && i < end; ++i) {
          float l = 0.f;
          if (!nothing) {
            Stored<E, 1>::load(from + i, &l);
            l = i == token ? at_token(l) : slope(l);
          }
          Stored<Out, 1>::store(to + i, &l);
        }
      }
    }
  }
}

constexpr int64_t kMostGroups = 1 << 20;         // workgroups of a launch along the rows

template <typename E, bool TOP, bool SPREAD> int launch_part(const LogProbArgs& a, void* stream) {
  auto with = [&](auto threads) {
    constexpr int L = decltype(threads)::value;
    constexpr int64_t kRows = L == 64 ? 4 : 1;
    const dim3 grid(static_cast<uint32_t>(std::min((a.rows + kRows - 1) / kRows, kMostGroups)), a.num_parts);
    return enqueue(log_probs_part<E, L, TOP, SPREAD>, grid, L < 256 ? 256 : L, 0, stream, a);
  };
  if (a.part <= 1024) return with(Number<64>{});
  // candidates are kept for 64 logits a thread; without them a workgroup of 256 threads has fewer sums to join
  return !TOP || a.part <= 16384 ? with(Number<256>{}) : with(Number<1024>{});
}

}  // namespace

int launch_log_probs(const LogProbArgs& args, void* stream) {
  const bool top = args.top > 0;
  auto with = [&](auto e) {
    typedef decltype(e) E;
    if (args.entropy != nullptr) return top ? launch_part<E, true, true>(args, stream) : launch_part<E, false, true>(args, stream);
    return top ? launch_part<E, true, false>(args, stream) : launch_part<E, false, false>(args, stream);
  };
  const int st = args.logits_bf16 ? with(uint16_t{}) : with(float{});
  if (st != 0 || args.num_parts == 1) return st;
  return enqueue(log_probs_join, dim3(static_cast<uint32_t>(std::min(args.rows, kMostGroups))), 256, 0, stream, args);
}

int launch_log_probs_gradient(const LogProbArgs& args, void* stream) {
  // a row that begins within a vector of eight may need a part more
  const dim3 grid(static_cast<uint32_t>(std::min(args.rows, kMostGroups)), (args.vocab + 7 + kGradientPart - 1) / kGradientPart);
  auto with = [&](auto e, auto out) {
    typedef decltype(e) E;
    typedef decltype(out) Out;
    return args.dentropy != nullptr ? enqueue(log_probs_gradient<E, Out, true>, grid, 256, 0, stream, args)
                                    : enqueue(log_probs_gradient<E, Out, false>, grid, 256, 0, stream, args);
  };
  if (args.logits_bf16) return args.dlogits_bf16 ? with(uint16_t{}, uint16_t{}) : with(uint16_t{}, float{});
  return args.dlogits_bf16 ? with(float{}, uint16_t{}) : with(float{}, float{});
}

}  // namespace noloco
