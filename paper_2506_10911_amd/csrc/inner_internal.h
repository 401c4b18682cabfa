// Types shared by the host side of the inner step's operators and their kernels (not part of the C ABI).
#pragma once

#include <cstdint>

#include "noloco.h"

namespace noloco {

// ---------------------------------------------------------------------------
// Orthogonalised updates of matrices
// ---------------------------------------------------------------------------

// Matrices of one shape that go through a launch together; a launch serves at most kNsClasses shapes.
constexpr int kNsClasses = 32;
constexpr int kNsChunks = 256;          // partial sums of squares of one matrix
constexpr int kNsChunkElems = 8192;     // elements that a workgroup sums, as long as kNsChunks of them are enough

// X, A and P are held times powers of two, so that binary16 has room for what they can be (A's eigenvalues up to kNsMostA,
// P's up to kNsMostP).  One binary16 a number: units in which X X^T comes out as A is held, and P X as X is.  Pairs: larger
// ones, or the low halves would be subnormal.
constexpr float ns_unit_x(int planes) { return planes == 1 ? 64.f : 8192.f; }
constexpr float ns_unit_a(int planes) { return planes == 1 ? 4096.f : 8192.f; }
constexpr float ns_unit_p(int planes) { return planes == 1 ? 1.f : 4096.f; }
constexpr double kNsMostA = 7.8, kNsMostP = 15.5;

// A worker's copy of a matrix.
struct NsItem {
  int64_t offset;       // first element in the array of all workers' rows
  int64_t row_stride;
  float scale;
  int32_t pad;
};

struct NsClass {
  uint64_t base;        // bytes from the workspace's start to the first item's buffers
  uint64_t item_bytes;  // from one item's buffers to the next one's
  uint32_t per_item;    // workgroups of one item in this launch
  uint32_t first_item;  // in the plan's table of items
  uint32_t first_sum;   // first item's place in the partial sums
  uint32_t m, n;        // the short and the long side
  uint32_t mp, np;      // and what they are padded to
  uint32_t tall;        // the matrix has more rows than columns: X is its transpose
  uint32_t splits;      // parts of the long side that X X^T is summed in, each by workgroups of its own
  uint32_t pad;
};

// In device memory: as kernel arguments these 2 KB cost every launch 0.8 us (toy matrices, 17 launches 112 / 99 us).
struct NsTable {
  uint32_t end[kNsClasses];     // workgroups of all classes up to and with this one; the rest 0xffffffff
  NsClass cls[kNsClasses];
};

struct NsArgs {
  const NsTable* table;
  const NsItem* items;
  char* workspace;
  double* sums;                 // [item][kNsChunks]
  uint32_t splits;              // the most of the launch's classes
  NsClass first;                // the table's first class, which is often the only one: its workgroups read no table
  uint32_t first_end;
};

// What an item's buffers hold, in bytes from their start: X and the next X [mp][np], A and P [mp][mp], each number
// one binary16 or a pair of them ("planes"), and behind single ones what they leave of A's diagonal and of P's, binary32 [mp]
// each.  While X X^T is summed in parts, these lie where the next X comes.
inline uint64_t ns_x_bytes(uint32_t mp, uint32_t np, int planes) { return uint64_t(mp) * np * 2 * planes; }
inline uint64_t ns_rest_bytes(uint32_t mp, int planes) { return planes == 1 ? uint64_t(mp) * 4 : 0; }
inline uint64_t ns_item_bytes(uint32_t mp, uint32_t np, int planes) {
  return 2 * (ns_x_bytes(mp, np, planes) + ns_x_bytes(mp, mp, planes) + ns_rest_bytes(mp, planes));
}

// A matrix whose X, A and P fit a CU's LDS goes through all steps in one workgroup: rows padded to 32, 16 bytes behind
// each of them.
constexpr int kNsSmallLds = 160 * 1024;
constexpr int kNsSmallThreads = 512;
constexpr int kNsSmallSums = 8 * 8;       // bytes in front of X
// Numbers of X's rows, in whole eights: a thread's 128, of pairs 80 (more do not fit the LDS).
constexpr uint64_t ns_small_numbers(int planes) { return (planes == 1 ? 128 : 80) * kNsSmallThreads; }
inline uint64_t ns_small_bytes(uint32_t m, uint32_t n, int planes) {
  const uint64_t mp = (uint64_t(m) + 31) / 32 * 32, np = (uint64_t(n) + 31) / 32 * 32;
  const uint64_t shares = mp <= 64 ? 8 * 1024 * sizeof(float) : 0;
  return kNsSmallSums + mp * (np * 2 * planes + 16) + 2 * mp * (mp * 2 * planes + 16) + shares;
}
constexpr int kNsSplitTile = 64, kNsSplitBytes = kNsSplitTile * kNsSplitTile * 4;      // a part of a tile of X X^T
struct NsSteps {
  int32_t count;
  float k[3 * NOLOCO_MAX_NEWTON_SCHULZ_STEPS];
};

enum NsKind { kNsGram = 0, kNsSquare = 1, kNsApply = 2, kNsLast = 3 };

// The arrays that hold the matrices (device, all workers' rows).
struct NsArrays {
  const void* in;        // x, or the gradient
  float* momentum;       // null: x is orthogonalised as it stands
  void* out;             // out, or theta
  int32_t in_bf16, out_bf16;
  float mu;
  int32_t nesterov;
  float keep;            // 1 - lr * weight_decay
  float lr;
  int32_t update;        // out <- keep * out - lr * scale * result instead of out <- result
  float eps;
};

int launch_ns_small(const NsArgs& args, const NsArrays& arrays, const NsSteps& steps, int planes, uint32_t workgroups,
                    uint32_t lds_bytes, void* stream);
int launch_ns_sums(const NsArgs& args, const NsArrays& arrays, uint32_t workgroups, void* stream);
int launch_ns_start(const NsArgs& args, const NsArrays& arrays, int planes, uint32_t workgroups, void* stream);
// Step `step` reads X number step & 1.
int launch_ns_product(const NsArgs& args, const NsArrays& arrays, int kind, int tile, int planes, int step,
                      float a, float b, float c, uint32_t workgroups, void* stream);

// ---------------------------------------------------------------------------
// Embedding lookup and its gradient
// ---------------------------------------------------------------------------

constexpr int kSortChunk = 2048;        // tokens that one workgroup sorts in its LDS
constexpr int kMergeWays = 16;          // sorted lists that one merge joins
constexpr int kMergeChunk = kSortChunk * kMergeWays;      // tokens that the first one holds in the LDS
constexpr int kSumChunk = 32;           // sorted positions that a workgroup sums

// The lookup's workgroups: 256 threads, sixteen tokens each, all of which may be more than 2^32 threads in one dimension.
constexpr int64_t kLookupTokens = 16;
struct LookupGrid { uint32_t x, y; };
inline LookupGrid lookup_grid(int64_t all) {
  const int64_t groups = (all + kLookupTokens - 1) / kLookupTokens, rows = (groups + (1 << 23) - 1) >> 23;
  return {static_cast<uint32_t>((groups + rows - 1) / rows), static_cast<uint32_t>(rows)};
}

struct EmbedArgs {
  void* table;            // first element of worker 0's table (or of its gradient)
  void* rows;             // out, or dout: [W][tokens][width]
  const void* tokens;     // [W][tokens]
  int64_t stride;         // between workers' tables
  int64_t num_tokens;
  uint32_t vocab, width;
  int32_t W;
  float scale;
  int32_t table_bf16, rows_bf16, tokens_i64, accumulate;
  int32_t vectors;        // columns that everything is aligned for at a time: 1, 4 or 8
  uint32_t* token[2];     // [W][tokens], sorted, and their positions
  uint32_t* position[2];
  float* partial;         // [W][chunks][2][width]
};

int launch_embed_lookup(const EmbedArgs& args, void* stream);
int launch_embed_gradient(const EmbedArgs& args, void* stream);

}  // namespace noloco
