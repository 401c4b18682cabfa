// Types shared by the host side of layer norm, matrices and log probabilities and their kernels (not part of the C ABI).
#pragma once

#include <algorithm>
#include <cstdint>

#include "noloco.h"

namespace noloco {

// ---------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------

constexpr int64_t kNormHeld = 16384;        // widest row that a workgroup holds in registers, 16 numbers a thread
constexpr int64_t kNormGradientHeld = 8192; // and in the gradient, with as many weights' sums
constexpr int64_t kNormRows = 4;            // rows that a workgroup works on at once, at most

// Workgroups of a worker: each takes every `groups`th set of rows and leaves one sum of the weights' gradients.  768 in all: the
// gradient's registers let three share a CU, and with 1024 the last of them ran alone (2 x 8192 rows of 4096 97 us, so 91).  Rows that
// no workgroup holds: 64, so that the sums of the widest take 512 MB at most, with a quarter of the chip at work.
inline uint32_t norm_groups(int64_t tokens, int64_t W, int64_t width) {
  const int64_t most = std::max<int64_t>(1, (width > kNormGradientHeld ? 64 : 768) / W);
  return static_cast<uint32_t>(std::max<int64_t>(1, std::min((tokens + kNormRows - 1) / kNormRows, most)));
}

struct NormArgs {
  const void* x;              // [W][tokens][width]
  const void* dout;
  const void* add;
  const void* theta;
  void* out;                  // or dx
  float* stats;               // [W][tokens][2]
  void* grad;
  float* partial;             // [W][groups][2][width]
  int64_t tokens, stride;     // stride: between workers' rows of theta and grad
  int64_t weight, bias;       // places in a row; bias -1: none
  uint32_t width, groups;
  int32_t W;
  float eps;
  int32_t x_bf16, dout_bf16, theta_bf16, out_bf16, grad_bf16, accumulate;
};

int launch_layer_norm(const NormArgs& args, void* stream);
int launch_layer_norm_gradient(const NormArgs& args, void* stream);

// ---------------------------------------------------------------------------
// Matrices
// ---------------------------------------------------------------------------

// One operand of a product sum over k of A(m, k) B(n, k): number (m, k) of worker w is `p` plus
// w * worker_stride + (along_k ? m * ld + k : k * ld + m).
struct Operand {
  const void* p;
  int64_t worker_stride, ld;
  int32_t along_k, bf16;
};

struct ProductArgs {
  Operand a, b;
  uint32_t m, n, k;
  int32_t W;
  void* out;                  // [m][n] of every worker, rows out_ld apart
  int64_t out_stride, out_ld;
  int32_t out_bf16, accumulate;
  // the end of a product: out = act(sum + bias) + more, before = sum + bias
  const void* bias;           // of n, or null
  int64_t bias_stride;
  int32_t bias_bf16, activation;
  const void* more;           // [m][n] as out, or null
  void* before;               // the same
};

constexpr double kSmallWork = double(1 << 28);  // multiplications of all workers up to which dz stays in binary32

// How a product goes out, by its sizes and types alone (but for the alignment of its operands).  Offsets are into the workspace.
struct ProductPlan {
  int32_t tile;               // 0: product_small, 256, 128, or 32 (32 x 256)
  int32_t f16;                // operands packed to binary16 times powers of two, or to bf16 parts where a worker's rows are too far apart
  int32_t packed[2], parts[2];        // parts: that there is room for, as many bf16 as the result needs of the operand
  uint32_t splits;            // parts that k is shared out in
  uint64_t packed_at[2], largest_at, exponents_at, parts_at, bytes;      // bytes: of the workspace
};

// `room`: bytes that there are; sums in parts take what packing leaves of it.
ProductPlan plan_product(const ProductArgs& args, uint64_t room);
// Most bytes that packing a product takes for each worker, whatever its types.
uint64_t pack_bytes(int64_t m, int64_t n, int64_t k);
// And for sums in parts, for all workers, whatever the types and for any fewer workers and smaller sizes; never more than kPartsRoom.
uint64_t parts_bytes(int64_t W, int64_t m, int64_t n, int64_t k);
constexpr uint64_t kPartsRoom = 64 << 20;

struct DirectArgs {
  const void *a, *b;          // 16-bit numbers, part 0 of worker 0
  int64_t a_worker, a_ld, a_part, b_worker, b_ld, b_part;
  // [0]: of bf16 operands as they lie, or of binary16; [1]: of workers in bf16 parts
  uint32_t a_parts[2], b_parts[2];    // two bits a segment: which part it takes
  uint32_t segments[2], splits;
  uint32_t tiles_m, tiles_n, run;
  const int32_t* exponents;   // [W][4]: of the two operands, and 1 where the worker is in bf16 parts
  float* parts;               // [splits][W][m][parts_ld], or null
  int64_t parts_ld;
};

constexpr int kPackParts = 256;
// Of an operand packed to binary16 the largest number of every 512 neighbours of a row, or of a whole shorter one, is at least 2^-17 of the
// worker's largest: then what binary16 leaves, 2^-39 of the latter, is 2^-22 of the piece's largest.
constexpr uint32_t kPackPiece = 512;
constexpr float kPackRange = 0x1p-17f;
struct PackOperand {
  const void* p;
  void* out;                  // [parts][W][rows][wide rounded up to eight]; null: not packed
  int64_t worker_stride, ld;
  uint32_t rows, wide;
  int32_t bf16, parts;
};
struct PackArgs {
  PackOperand operand[2];
  float* largest;             // [W][2][2][kPackParts]: largest numbers, and the least of the rows' largest
  int32_t* exponents;
  int32_t f16, W;
};

int launch_product(const ProductArgs& args, const ProductPlan& plan, char* room, void* stream);

struct SlopeArgs {
  const void* dout;           // [W][tokens][outputs]
  const void* before;         // null: dz is dout, and only the sums are made
  void* dz;
  float* partial;             // [W][groups][outputs]
  void* grad;                 // worker 0's first bias; null: no sums
  int64_t stride;             // between workers' rows of grad
  int64_t tokens;
  uint32_t outputs, groups;
  int32_t W, activation;
  int32_t dout_bf16, dz_bf16, grad_bf16, accumulate;
};

// Groups of tokens, each a workgroup's: 64 of 64 tokens and more; up to 256 tokens are one group, which leaves its sums in the
// gradient itself.
constexpr int64_t kSlopeRows = 64;
inline uint32_t slope_groups(int64_t tokens) {
  return tokens <= 4 * kSlopeRows ? 1 : static_cast<uint32_t>(std::min<int64_t>((tokens + kSlopeRows - 1) / kSlopeRows, 64));
}
int launch_slope(const SlopeArgs& args, void* stream);

// ---------------------------------------------------------------------------
// Log probabilities
// ---------------------------------------------------------------------------

constexpr int64_t kLogChunk = 65536;         // most logits of a row that one workgroup takes: 64 of a thread

// Parts that a row is cut into: as many as its length needs, and more where there are few rows.
inline uint32_t log_prob_parts(int64_t rows, int64_t vocab) {
  const int64_t least = (vocab + kLogChunk - 1) / kLogChunk;
  const int64_t wanted = rows > 0 ? 256 / rows : 1, room = (vocab + 4095) / 4096;
  return static_cast<uint32_t>(std::max(least, std::min(wanted, room)));
}

// What a workgroup knows of its part of a row: the largest logit, the sum of exp(l - largest) over all but one that is the
// largest, and the sum of exp(l - largest) (largest - l).
struct LogPart { float largest, rest, spread, pad; };

struct LogProbArgs {
  const void* logits;
  const void* tokens;
  float* log_probs;
  float* entropy;
  float* norms;
  int32_t* top_tokens;
  float* top_log_probs;
  const float* dlog_probs;
  const float* dentropy;
  void* dlogits;
  LogPart* parts;             // [rows][parts]
  uint64_t* keys;             // [rows][parts][top]
  int64_t rows, row_stride;   // rows: of all workers
  uint32_t vocab, num_parts, part;      // part: logits of one
  int32_t top;
  int32_t logits_bf16, tokens_i64, dlogits_bf16;
};

int launch_log_probs(const LogProbArgs& args, void* stream);
int launch_log_probs_gradient(const LogProbArgs& args, void* stream);

}  // namespace noloco
