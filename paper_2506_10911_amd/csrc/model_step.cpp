// C ABI of layer norm, matrices and log probabilities: argument checking, plans, and the split of a call into kernel
// launches.  All arithmetic is in layer_norm.hip, products.hip, linear.hip and log_probs.hip.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>
#include <memory>
#include <new>
#include <vector>

#include "model_internal.h"

namespace {

constexpr int64_t kDefaultWorkspace = 1ll << 30;
constexpr int64_t kMostWidth = 1 << 20, kMostNormTokens = 1 << 27, kMostRows = std::numeric_limits<int32_t>::max();
constexpr int64_t kMostSide = 1 << 22, kMostTokens = 1 << 24, kMostNumbers = 1 << 30, kMostVocab = 1 << 24;

bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

bool is_dtype(int32_t t) { return t == NOLOCO_F32 || t == NOLOCO_BF16; }
uint64_t bytes_of(int32_t dtype) { return dtype == NOLOCO_BF16 ? 2 : 4; }
bool is_flag(int32_t v) { return v == 0 || v == 1; }

// Arrays of a call, of which those that are written must lie apart from all others.
struct Range { const void* p; uint64_t bytes; };
bool apart(const Range& written, std::initializer_list<Range> others) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(written.p);
  for (const Range& r : others) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(r.p);
    if (written.p != nullptr && r.p != nullptr && written.bytes > 0 && r.bytes > 0 && a < b + r.bytes && b < a + written.bytes) return false;
  }
  return true;
}

noloco_status check_device(int of_plan) {
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) return NOLOCO_ERR_DEVICE;
  return device == of_plan ? NOLOCO_OK : NOLOCO_ERR_INVALID_ARG;
}

// A plan's one device allocation, on the GPU that was current when it was made.
struct Block {
  int device = -1;
  char* memory = nullptr;
  Block() = default;
  Block(const Block&) = delete;
  Block& operator=(const Block&) = delete;
  ~Block() {
    if (memory != nullptr) (void)hipFree(memory);
  }
  bool allocate(uint64_t bytes) {
    if (hipGetDevice(&device) == hipSuccess && hipMalloc(reinterpret_cast<void**>(&memory), bytes + 256) == hipSuccess) return true;
    memory = nullptr;
    return false;
  }
};

template <typename Plan> noloco_status destroy(Plan* plan) {
  if (plan == nullptr) return NOLOCO_OK;
  noloco_status st = NOLOCO_OK;
  if (plan->block.memory != nullptr && hipFree(plan->block.memory) != hipSuccess) st = NOLOCO_ERR_DEVICE;
  plan->block.memory = nullptr;
  delete plan;
  return st;
}

noloco_status check_rows(int32_t num, const void* list, int64_t worker_stride, int32_t W, int64_t max_tokens) {
  if (num < 0 || worker_stride < 0 || W < 1 || max_tokens < 0) return NOLOCO_ERR_INVALID_ARG;
  if (list == nullptr && num > 0) return NOLOCO_ERR_NULL;
  if (W > NOLOCO_MAX_WORKERS || worker_stride > std::numeric_limits<int64_t>::max() / 8 / W) return NOLOCO_ERR_UNSUPPORTED;
  return worker_stride % NOLOCO_STRIDE_ALIGN_ELEMS != 0 ? NOLOCO_ERR_ALIGNMENT : NOLOCO_OK;
}

uint64_t whole(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

struct noloco_layer_norm_plan {
  std::vector<noloco_norm> norms;
  int64_t stride = 0, max_tokens = 0;
  int32_t W = 0;
  Block block;
};

struct noloco_linear_plan {
  std::vector<noloco_linear_layer> layers;
  int64_t stride = 0, max_tokens = 0;
  int32_t W = 0;
  uint64_t room = 0;          // bytes of the workspace
  Block block;
};

struct noloco_log_prob_plan {
  int64_t vocab = 0, row_stride = 0, max_tokens = 0;
  int32_t W = 0, max_top = 0;
  uint64_t parts_bytes = 0;
  Block block;
};

// ---------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------

extern "C" noloco_status noloco_layer_norm_plan_create(const noloco_norm* norms, int32_t num_norms, int64_t worker_stride, int32_t W,
                                                       int64_t max_tokens, noloco_layer_norm_plan** out) {
  if (out == nullptr) return NOLOCO_ERR_NULL;
  *out = nullptr;
  const noloco_status st = check_rows(num_norms, norms, worker_stride, W, max_tokens);
  if (st != NOLOCO_OK) return st;
  if (max_tokens > kMostNormTokens || W * max_tokens > kMostRows) return NOLOCO_ERR_UNSUPPORTED;
  uint64_t partial = 0;
  for (int32_t i = 0; i < num_norms; ++i) {
    const noloco_norm& n = norms[i];
    if (n.weight < 0 || n.bias < -1 || n.width < 1) return NOLOCO_ERR_INVALID_ARG;
    if (n.width > kMostWidth) return NOLOCO_ERR_UNSUPPORTED;
    for (int64_t at : {n.weight, n.bias})
      if (at > worker_stride || (at >= 0 && n.width > worker_stride - at)) return NOLOCO_ERR_SEGMENT_OVERLAP;
    if (n.bias >= 0 && n.bias < n.weight + n.width && n.weight < n.bias + n.width) return NOLOCO_ERR_SEGMENT_OVERLAP;
    partial = std::max(partial, static_cast<uint64_t>(W) * noloco::norm_groups(max_tokens, W, n.width) * 2 * n.width * sizeof(float));
  }
  try {
    std::unique_ptr<noloco_layer_norm_plan> plan(new noloco_layer_norm_plan);
    plan->norms.assign(norms, norms + num_norms);
    plan->stride = worker_stride;
    plan->max_tokens = max_tokens;
    plan->W = W;
    if (!plan->block.allocate(partial)) return NOLOCO_ERR_DEVICE;
    *out = plan.release();
    return NOLOCO_OK;
  } catch (const std::bad_alloc&) {
    return NOLOCO_ERR_NO_MEMORY;
  } catch (...) {
    return NOLOCO_ERR_INVALID_ARG;
  }
}

extern "C" noloco_status noloco_layer_norm_plan_destroy(noloco_layer_norm_plan* plan) { return destroy(plan); }

namespace {

noloco_status norm_args(const noloco_layer_norm_plan* plan, int32_t norm, int64_t num_tokens, noloco::NormArgs* args) {
  if (norm < 0 || static_cast<size_t>(norm) >= plan->norms.size() || num_tokens < 0 || num_tokens > plan->max_tokens) return NOLOCO_ERR_INVALID_ARG;
  const noloco_norm& n = plan->norms[norm];
  *args = noloco::NormArgs{};
  args->tokens = num_tokens;
  args->stride = plan->stride;
  args->weight = n.weight;
  args->bias = n.bias;
  args->width = static_cast<uint32_t>(n.width);
  args->W = plan->W;
  args->groups = noloco::norm_groups(num_tokens, plan->W, n.width);
  args->partial = reinterpret_cast<float*>(plan->block.memory);
  return NOLOCO_OK;
}

}  // namespace

extern "C" noloco_status noloco_layer_norm(const noloco_layer_norm_plan* plan, int32_t norm, const void* x, int32_t x_dtype,
                                           const void* theta, int32_t theta_dtype, int64_t num_tokens, float eps, void* out,
                                           int32_t out_dtype, float* stats, void* hip_stream) {
  if (plan == nullptr || theta == nullptr) return NOLOCO_ERR_NULL;
  noloco::NormArgs args;
  const noloco_status st = norm_args(plan, norm, num_tokens, &args);
  if (st != NOLOCO_OK) return st;
  if (num_tokens > 0 && (x == nullptr || out == nullptr)) return NOLOCO_ERR_NULL;
  if (!is_dtype(x_dtype) || !is_dtype(theta_dtype) || !is_dtype(out_dtype) || !(eps >= 0.f) || !std::isfinite(eps)) return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(theta, NOLOCO_BASE_ALIGN_BYTES) || !aligned(x, 16) || !aligned(out, 16) || !aligned(stats, 16)) return NOLOCO_ERR_ALIGNMENT;
  const uint64_t rows = static_cast<uint64_t>(plan->W) * num_tokens, numbers = rows * args.width;
  const Range of_theta{theta, static_cast<uint64_t>(plan->W) * plan->stride * bytes_of(theta_dtype)}, of_x{x, numbers * bytes_of(x_dtype)};
  const Range of_out{out, numbers * bytes_of(out_dtype)}, of_stats{stats, rows * 8};
  if (!apart(of_out, {of_theta, of_x, of_stats}) || !apart(of_stats, {of_theta, of_x})) return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens == 0) return NOLOCO_OK;
  args.x = x;
  args.theta = theta;
  args.out = out;
  args.stats = stats;
  args.eps = eps;
  args.x_bf16 = x_dtype == NOLOCO_BF16;
  args.theta_bf16 = theta_dtype == NOLOCO_BF16;
  args.out_bf16 = out_dtype == NOLOCO_BF16;
  const noloco_status there = check_device(plan->block.device);
  if (there != NOLOCO_OK) return there;
  return noloco::launch_layer_norm(args, hip_stream) == 0 ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}

extern "C" noloco_status noloco_layer_norm_gradient(const noloco_layer_norm_plan* plan, int32_t norm, const void* dout, int32_t dout_dtype,
                                                    const void* x, int32_t x_dtype, const void* theta, int32_t theta_dtype,
                                                    const float* stats, int64_t num_tokens, const void* add, void* dx, int32_t dx_dtype,
                                                    void* grad, int32_t grad_dtype, int32_t accumulate, void* hip_stream) {
  if (plan == nullptr || theta == nullptr) return NOLOCO_ERR_NULL;
  noloco::NormArgs args;
  const noloco_status st = norm_args(plan, norm, num_tokens, &args);
  if (st != NOLOCO_OK) return st;
  if (num_tokens > 0 && (x == nullptr || dout == nullptr || stats == nullptr || dx == nullptr)) return NOLOCO_ERR_NULL;
  if (!is_dtype(dout_dtype) || !is_dtype(x_dtype) || !is_dtype(theta_dtype) || !is_dtype(dx_dtype) || !is_dtype(grad_dtype) || !is_flag(accumulate))
    return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(theta, NOLOCO_BASE_ALIGN_BYTES) || !aligned(grad, NOLOCO_BASE_ALIGN_BYTES) || !aligned(x, 16) || !aligned(dout, 16) ||
      !aligned(stats, 16) || !aligned(add, 16) || !aligned(dx, 16))
    return NOLOCO_ERR_ALIGNMENT;
  const uint64_t rows = static_cast<uint64_t>(plan->W) * num_tokens, numbers = rows * args.width, elements = static_cast<uint64_t>(plan->W) * plan->stride;
  const Range of_theta{theta, elements * bytes_of(theta_dtype)}, of_x{x, numbers * bytes_of(x_dtype)}, of_dout{dout, numbers * bytes_of(dout_dtype)};
  const Range of_stats{stats, rows * 8}, of_dx{dx, numbers * bytes_of(dx_dtype)}, of_grad{grad, elements * bytes_of(grad_dtype)};
  const Range of_add{add == dx ? nullptr : add, of_dx.bytes};
  if (!apart(of_dx, {of_theta, of_x, of_dout, of_stats, of_add, of_grad}) || !apart(of_grad, {of_theta, of_x, of_dout, of_stats, of_add}))
    return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens == 0 && (accumulate || grad == nullptr)) return NOLOCO_OK;
  args.x = x;
  args.dout = dout;
  args.add = add;
  args.theta = theta;
  args.out = dx;
  args.stats = const_cast<float*>(stats);
  args.grad = grad;
  args.x_bf16 = x_dtype == NOLOCO_BF16;
  args.dout_bf16 = dout_dtype == NOLOCO_BF16;
  args.theta_bf16 = theta_dtype == NOLOCO_BF16;
  args.out_bf16 = dx_dtype == NOLOCO_BF16;
  args.grad_bf16 = grad_dtype == NOLOCO_BF16;
  args.accumulate = accumulate;
  const noloco_status there = check_device(plan->block.device);
  if (there != NOLOCO_OK) return there;
  return noloco::launch_layer_norm_gradient(args, hip_stream) == 0 ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}

// ---------------------------------------------------------------------------
// Matrices
// ---------------------------------------------------------------------------

namespace noloco {

namespace {

constexpr uint64_t kMostGroups = 1u << 22;      // workgroups of a launch
constexpr int64_t kMostRow = 1 << 22;           // numbers from one row of an operand to the next: 256 of them have 32-bit offsets

// Does the operand lie as product_direct loads it?
bool lies_well(const Operand& o, uint32_t k) {
  return o.bf16 && aligned(o.p, 16) && o.ld <= kMostRow && ((o.ld | o.worker_stride) & 7) == 0 && (!o.along_k || k % 8 == 0);
}

uint64_t tiles_of(uint64_t v, uint64_t tile) { return (v + tile - 1) / tile; }

}  // namespace

uint64_t pack_bytes(int64_t m, int64_t n, int64_t k) {
  auto most = [k](int64_t size) { return static_cast<uint64_t>(std::max(size * ((k + 7) / 8 * 8), k * ((size + 7) / 8 * 8))) * 6; };
  return whole(most(m)) + whole(most(n)) + 2 * 2 * kPackParts * sizeof(float) + 1024;
}

uint64_t parts_bytes(int64_t W, int64_t m, int64_t n, int64_t k) {
  const uint64_t part = static_cast<uint64_t>(W) * m * (tiles_of(n, 8) * 8) * sizeof(float), rounds = tiles_of(k, 1024);
  // as plan_product shares k out: small products in up to 1024 workgroups' tiles, others eight stages each of up to three segments
  const uint64_t small = rounds > 2 ? std::min<uint64_t>(rounds, 32) : 0, direct = std::min<uint64_t>(tiles_of(k, 64) * 3 / 8, 32);
  return std::max(std::min<uint64_t>(small * part, 1024 * 32 * 32 * sizeof(float)), direct > 1 ? std::min(direct * part, kPartsRoom) : 0);
}

// Estimates of a product's time, us, from which its way is chosen.
//   small    tiles of 32 x 32 that read their operands from the caches at 8 TB/s together (5 where these are larger,
//            half where vectors lie across lines): 4 x 512 x
//            1024 x 1024 bf16 35 us, float 60; and rounds of 1024 k of a workgroup's sixteen waves, 2.5 us each
//   direct   stages of 64 k: in tiles of 128 0.85 us each with one workgroup on a CU (2048 x 2048 x 2048 33 us), 0.52 with two (2 of
//            them 39), of 256 1.1, and 1.6 where the chip is full (8 x 4096 x 2048 x 8192 1013 us, in tiles of 128 1237); 32 rows 0.4 us or
//            what reading the matrix takes; packing and joining by what they move, and 3 us a launch
// Both sides where they meet, small and direct: 64 x 4096 x 4096 bf16 31 and 16 us, float 36 and 65; one token through 4096 x 4096 16
// and 10, float 18 and 60; 2 x 128 x 1024 x 1024 7.3 and 12.3, float 9.6 and 29.5; 1024 x 1024 x 1024 float 30 and 32.  In bf16 the
// estimates take the slower one there, 20.6 and 18.4, and for 2 x 2456 x 6912 x 32, 26 and 20: the rate of the caches is cruder than it is.
ProductPlan plan_product(const ProductArgs& args, uint64_t room) {
  ProductPlan plan{};
  plan.parts[0] = plan.parts[1] = 1;
  plan.splits = 1;
  const uint64_t W = args.W, m = args.m, n = args.n, k = args.k;
  if (k == 0 || m == 0 || n == 0) return plan;
  const uint64_t part = W * m * (tiles_of(n, 8) * 8) * sizeof(float);
  auto parts_in = [&](uint64_t bytes) { return std::min(bytes, kPartsRoom) / part; };

  const uint64_t tiles32 = tiles_of(m, 32) * tiles_of(n, 32) * W, rounds = tiles_of(k, 1024);
  const int element = (args.a.bf16 ? 2 : 4) + (args.b.bf16 ? 2 : 4);
  ProductPlan small = plan;
  if (rounds > 2) small.splits = static_cast<uint32_t>(std::max<uint64_t>(1, std::min({rounds, 1024 / tiles32, parts_in(room), uint64_t(32)})));
  small.bytes = small.splits > 1 ? small.splits * part : 0;
  double rate = double(W) * k * (m + n) * element < 2e8 ? 8 : 5;
  if ((args.a.along_k && args.a.ld % 8 != 0) || (args.b.along_k && args.b.ld % 8 != 0)) rate /= 2;
  const double of_small = 4 + (small.splits > 1 ? 3 : 0) + std::max(2.5 * std::min(k / 1024., double(tiles_of(rounds, small.splits))), tiles32 * 2048e-6 * k * element / 64 / rate);

  const int floats = (args.a.bf16 ? 0 : 1) + (args.b.bf16 ? 0 : 1);
  plan.f16 = args.out_bf16 ? floats == 2 : floats > 0;
  uint64_t at = 0;
  double moved = 0;
  for (int i = 0; i < 2; ++i) {
    const Operand& o = i == 0 ? args.a : args.b;
    const uint64_t size = i == 0 ? m : n, rows = o.along_k ? size : k, wide = tiles_of(o.along_k ? k : size, 8) * 8;
    plan.packed[i] = plan.f16 || !lies_well(o, args.k);
    plan.parts[i] = plan.f16 && !o.bf16 ? (args.out_bf16 ? 2 : 3) : 1;
    plan.packed_at[i] = at;
    if (!plan.packed[i]) continue;
    at += whole(W * rows * wide * 2 * plan.parts[i]);
    moved += double(W) * rows * wide * ((o.bf16 ? 2 : 4) * (plan.f16 ? 2 : 1) + (plan.parts[i] == 3 ? 4 : 2));
  }
  plan.largest_at = at;
  at += plan.f16 ? whole(W * 2 * 2 * kPackParts * sizeof(float)) : 0;
  plan.exponents_at = at;
  at += plan.f16 ? whole(W * 4 * sizeof(int32_t)) : 0;
  plan.parts_at = at;
  // of binary16, which workers are nearly always in
  const uint64_t segments = 1 + (plan.parts[0] == 3) + (plan.parts[1] == 3), stages = tiles_of(k, 64) * segments, left = room > at ? room - at : 0;
  const double packing = (moved > 0 ? 3 : 0) + (plan.f16 ? 3 : 0) + moved / 3.5e6;
  double best = of_small;
  ProductPlan chosen = small;
  for (int tile : {32, 128, 256}) {
    if ((tile == 32) != (m <= 32 && args.a.along_k)) continue;
    const uint64_t tiles = tiles_of(m, tile) * tiles_of(n, tile == 32 ? 256 : tile) * W, target = tile == 128 ? 512 : 256;
    if (tiles > kMostGroups) continue;
    plan.tile = tile;
    plan.splits = static_cast<uint32_t>(std::max<uint64_t>(1, std::min({target / tiles, stages / 8, parts_in(left), uint64_t(32)})));
    plan.bytes = at + (plan.splits > 1 ? plan.splits * part : 0);
    const uint64_t each = tiles_of(stages, plan.splits), groups = tiles * plan.splits, on_cu = tiles_of(groups, 256);
    double us = 5 + packing + (plan.splits > 1 ? 3 + 2 * plan.splits * part / 5e6 : 0);
    if (tile == 32) us += std::max(0.4 * each * on_cu, 2e-6 * W * n * k / 5.5);
    else if (tile == 128) us += groups <= 256 ? 0.85 * each + 3 : on_cu * (0.52 * each + 2.5);
    else us += groups < 200 ? 1.1 * each + 6 : on_cu * (1.6 * each + 6);
    if (us >= best) continue;
    best = us;
    chosen = plan;
  }
  return chosen;
}

}  // namespace noloco

namespace {

// Workspace that one worker's gradient needs: dz in binary32, and the bias's sums.
uint64_t dz_bytes(const noloco_linear_layer& l, int64_t tokens) { return whole(static_cast<uint64_t>(tokens) * l.outputs * sizeof(float)); }
uint64_t packed_bytes(const noloco_linear_layer& l, int64_t tokens) {
  return std::max({noloco::pack_bytes(tokens, l.outputs, l.inputs), noloco::pack_bytes(tokens, l.inputs, l.outputs), noloco::pack_bytes(l.inputs, l.outputs, tokens)});
}
uint64_t sums_bytes(const noloco_linear_layer& l, int64_t tokens) { return whole(static_cast<uint64_t>(noloco::slope_groups(tokens)) * l.outputs * sizeof(float)); }

// Does a run of `count` elements from `at` on share one with a matrix of `rows` rows of `cols`?
bool meets(int64_t at, int64_t count, const noloco_linear_layer& l, int64_t rows, int64_t cols) {
  const int64_t end = at + count, last_end = l.offset + (rows - 1) * l.row_stride + cols;
  if (end <= l.offset || at >= last_end) return false;
  // the last row that begins at or before the run's last element ends behind its first
  const int64_t row = std::min(rows - 1, (end - 1 - l.offset) / l.row_stride);
  return l.offset + row * l.row_stride + cols > at;
}

noloco_status check_layer(const noloco_linear_layer& l, int64_t worker_stride, int64_t max_tokens) {
  if (l.offset < 0 || l.inputs < 1 || l.outputs < 1 || l.bias < -1 || !is_flag(l.transposed)) return NOLOCO_ERR_INVALID_ARG;
  if (l.inputs > kMostSide || l.outputs > kMostSide) return NOLOCO_ERR_UNSUPPORTED;
  const int64_t rows = l.transposed ? l.outputs : l.inputs, cols = l.transposed ? l.inputs : l.outputs;
  if (l.row_stride < cols) return NOLOCO_ERR_INVALID_ARG;
  // the last element's place, without a product that could overflow
  if (l.offset > worker_stride || cols > worker_stride - l.offset) return NOLOCO_ERR_SEGMENT_OVERLAP;
  if (rows > 1 && l.row_stride > (worker_stride - l.offset - cols) / (rows - 1)) return NOLOCO_ERR_SEGMENT_OVERLAP;
  if (l.bias > worker_stride || (l.bias >= 0 && l.outputs > worker_stride - l.bias)) return NOLOCO_ERR_SEGMENT_OVERLAP;
  if (l.row_stride > kMostNumbers / rows || max_tokens * std::max(l.inputs, l.outputs) > kMostNumbers) return NOLOCO_ERR_UNSUPPORTED;
  if (l.bias >= 0 && meets(l.bias, l.outputs, l, rows, cols)) return NOLOCO_ERR_SEGMENT_OVERLAP;
  return NOLOCO_OK;
}

}  // namespace

extern "C" noloco_status noloco_linear_plan_create(const noloco_linear_layer* layers, int32_t num_layers, int64_t worker_stride, int32_t W,
                                                   int64_t max_tokens, int64_t workspace_bytes, noloco_linear_plan** out) {
  if (out == nullptr) return NOLOCO_ERR_NULL;
  *out = nullptr;
  if (workspace_bytes < 0) return NOLOCO_ERR_INVALID_ARG;
  noloco_status st = check_rows(num_layers, layers, worker_stride, W, max_tokens);
  if (st != NOLOCO_OK) return st;
  if (max_tokens > kMostTokens) return NOLOCO_ERR_UNSUPPORTED;
  uint64_t one = 0, parts = 0;
  for (int32_t i = 0; i < num_layers; ++i) {
    const noloco_linear_layer& l = layers[i];
    st = check_layer(l, worker_stride, max_tokens);
    if (st != NOLOCO_OK) return st;
    one = std::max(one, dz_bytes(l, max_tokens) + sums_bytes(l, max_tokens) + packed_bytes(l, max_tokens));
    const int64_t sides[2] = {l.inputs, l.outputs};
    for (int i = 0; i < 2; ++i)
      parts = std::max({parts, noloco::parts_bytes(W, max_tokens, sides[i], sides[1 - i]), noloco::parts_bytes(W, sides[i], sides[1 - i], max_tokens)});
  }
  try {
    std::unique_ptr<noloco_linear_plan> plan(new noloco_linear_plan);
    plan->layers.assign(layers, layers + num_layers);
    plan->stride = worker_stride;
    plan->max_tokens = max_tokens;
    plan->W = W;
    const uint64_t asked = workspace_bytes > 0 ? workspace_bytes : kDefaultWorkspace;
    plan->room = std::max(one, std::min(one * W, asked)) + whole(parts);
    if (!plan->block.allocate(plan->room)) return NOLOCO_ERR_DEVICE;
    *out = plan.release();
    return NOLOCO_OK;
  } catch (const std::bad_alloc&) {
    return NOLOCO_ERR_NO_MEMORY;
  } catch (...) {
    return NOLOCO_ERR_INVALID_ARG;
  }
}

extern "C" noloco_status noloco_linear_plan_destroy(noloco_linear_plan* plan) { return destroy(plan); }

namespace {

const char* offset(const void* p, int64_t elements, int32_t dtype) { return static_cast<const char*>(p) + elements * static_cast<int64_t>(bytes_of(dtype)); }
char* offset(void* p, int64_t elements, int32_t dtype) { return static_cast<char*>(p) + elements * static_cast<int64_t>(bytes_of(dtype)); }

// Activations [tokens][width] as an operand whose k runs along the width, or along the tokens.
noloco::Operand rows_operand(const void* p, int64_t tokens, int64_t width, int32_t dtype, bool along_width) {
  return {p, tokens * width, width, along_width ? 1 : 0, dtype == NOLOCO_BF16 ? 1 : 0};
}

// A product, in batches of workers whose packed operands fit `bytes` of the workspace from `room` on.
bool run_product(noloco::ProductArgs args, char* room, uint64_t bytes, int32_t W, void* stream) {
  for (int32_t w = 0; w < W; w += args.W) {
    args.W = W - w;
    noloco::ProductPlan plan = noloco::plan_product(args, bytes);
    while (plan.bytes > bytes && args.W > 1) {
      args.W = (args.W + 1) / 2;
      plan = noloco::plan_product(args, bytes);
    }
    if (noloco::launch_product(args, plan, room, stream) != 0) return false;
    for (noloco::Operand* o : {&args.a, &args.b}) o->p = static_cast<const char*>(o->p) + args.W * o->worker_stride * (o->bf16 ? 2 : 4);
    const int32_t out_dtype = args.out_bf16 ? NOLOCO_BF16 : NOLOCO_F32;
    args.out = offset(args.out, args.W * args.out_stride, out_dtype);
    if (args.more != nullptr) args.more = offset(args.more, args.W * args.out_stride, out_dtype);
    if (args.before != nullptr) args.before = offset(args.before, args.W * args.out_stride, out_dtype);
    if (args.bias != nullptr) args.bias = offset(args.bias, args.W * args.bias_stride, args.bias_bf16 ? NOLOCO_BF16 : NOLOCO_F32);
  }
  return true;
}

noloco_status check_linear(const noloco_linear_plan* plan, int32_t layer, int64_t num_tokens, int32_t activation) {
  if (layer < 0 || static_cast<size_t>(layer) >= plan->layers.size() || num_tokens < 0 || num_tokens > plan->max_tokens) return NOLOCO_ERR_INVALID_ARG;
  return activation < NOLOCO_ACT_NONE || activation > NOLOCO_ACT_SILU ? NOLOCO_ERR_INVALID_ARG : NOLOCO_OK;
}

}  // namespace

extern "C" noloco_status noloco_linear(const noloco_linear_plan* plan, int32_t layer, const void* x, int32_t x_dtype, const void* theta,
                                       int32_t theta_dtype, int64_t num_tokens, int32_t activation, const void* residual, void* before,
                                       void* out, int32_t out_dtype, void* hip_stream) {
  if (plan == nullptr || theta == nullptr) return NOLOCO_ERR_NULL;
  const noloco_status st = check_linear(plan, layer, num_tokens, activation);
  if (st != NOLOCO_OK) return st;
  if (num_tokens > 0 && (x == nullptr || out == nullptr)) return NOLOCO_ERR_NULL;
  if (!is_dtype(x_dtype) || !is_dtype(theta_dtype) || !is_dtype(out_dtype)) return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(theta, NOLOCO_BASE_ALIGN_BYTES) || !aligned(x, 16) || !aligned(out, 16) || !aligned(residual, 16) || !aligned(before, 16))
    return NOLOCO_ERR_ALIGNMENT;
  const noloco_linear_layer& l = plan->layers[layer];
  const uint64_t rows = static_cast<uint64_t>(plan->W) * num_tokens;
  const Range of_theta{theta, static_cast<uint64_t>(plan->W) * plan->stride * bytes_of(theta_dtype)}, of_x{x, rows * l.inputs * bytes_of(x_dtype)};
  const Range of_out{out, rows * l.outputs * bytes_of(out_dtype)}, of_before{before, of_out.bytes}, of_residual{residual == out ? nullptr : residual, of_out.bytes};
  if (!apart(of_out, {of_theta, of_x, of_before, of_residual}) || !apart(of_before, {of_theta, of_x, of_residual})) return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens == 0) return NOLOCO_OK;
  noloco::ProductArgs args{};
  args.a = rows_operand(x, num_tokens, l.inputs, x_dtype, true);
  args.b = {offset(theta, l.offset, theta_dtype), plan->stride, l.row_stride, l.transposed, theta_dtype == NOLOCO_BF16 ? 1 : 0};
  args.m = static_cast<uint32_t>(num_tokens);
  args.n = static_cast<uint32_t>(l.outputs);
  args.k = static_cast<uint32_t>(l.inputs);
  args.W = plan->W;
  args.out = out;
  args.out_stride = num_tokens * l.outputs;
  args.out_ld = l.outputs;
  args.out_bf16 = out_dtype == NOLOCO_BF16;
  if (l.bias >= 0) {
    args.bias = offset(theta, l.bias, theta_dtype);
    args.bias_stride = plan->stride;
    args.bias_bf16 = theta_dtype == NOLOCO_BF16;
  }
  args.activation = activation;
  args.more = residual;
  args.before = before;
  const noloco_status there = check_device(plan->block.device);
  if (there != NOLOCO_OK) return there;
  return run_product(args, plan->block.memory, plan->room, plan->W, hip_stream) ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}

extern "C" noloco_status noloco_linear_gradient(const noloco_linear_plan* plan, int32_t layer, const void* dout, int32_t dout_dtype,
                                                const void* x, int32_t x_dtype, const void* theta, int32_t theta_dtype, int64_t num_tokens,
                                                int32_t activation, const void* before, const void* add, void* dx, int32_t dx_dtype,
                                                void* grad, int32_t grad_dtype, int32_t accumulate, void* hip_stream) {
  if (plan == nullptr || theta == nullptr) return NOLOCO_ERR_NULL;
  noloco_status st = check_linear(plan, layer, num_tokens, activation);
  if (st != NOLOCO_OK) return st;
  const bool acts = activation != NOLOCO_ACT_NONE;
  if (num_tokens > 0 && (dout == nullptr || (acts && before == nullptr) || (grad != nullptr && x == nullptr))) return NOLOCO_ERR_NULL;
  if (!is_dtype(dout_dtype) || !is_dtype(x_dtype) || !is_dtype(theta_dtype) || !is_dtype(dx_dtype) || !is_dtype(grad_dtype) || !is_flag(accumulate))
    return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(theta, NOLOCO_BASE_ALIGN_BYTES) || !aligned(grad, NOLOCO_BASE_ALIGN_BYTES) || !aligned(dout, 16) || !aligned(x, 16) ||
      !aligned(before, 16) || !aligned(add, 16) || !aligned(dx, 16))
    return NOLOCO_ERR_ALIGNMENT;
  const noloco_linear_layer& l = plan->layers[layer];
  const int64_t T = num_tokens;
  const uint64_t rows = static_cast<uint64_t>(plan->W) * T, elements = static_cast<uint64_t>(plan->W) * plan->stride;
  const Range of_theta{theta, elements * bytes_of(theta_dtype)}, of_grad{grad, elements * bytes_of(grad_dtype)}, of_x{x, rows * l.inputs * bytes_of(x_dtype)};
  const Range of_dout{dout, rows * l.outputs * bytes_of(dout_dtype)}, of_before{before, of_dout.bytes}, of_dx{dx, rows * l.inputs * bytes_of(dx_dtype)};
  const Range of_add{add == dx ? nullptr : add, of_dx.bytes};
  if (!apart(of_dx, {of_theta, of_x, of_dout, of_before, of_add, of_grad}) || !apart(of_grad, {of_theta, of_x, of_dout, of_before, of_add}))
    return NOLOCO_ERR_INVALID_ARG;
  if ((dx == nullptr || T == 0) && (grad == nullptr || (T == 0 && accumulate))) return NOLOCO_OK;
  const noloco_status there = check_device(plan->block.device);
  if (there != NOLOCO_OK) return there;

  // dz is kept in binary32 where a float result takes it, or a product with a float operand (one of two operands may be rounded to
  // bf16, as the result is), unless it is dout itself, or zeros in places of it.
  const bool fine = (dx != nullptr && (dx_dtype == NOLOCO_F32 || theta_dtype == NOLOCO_F32)) ||
                    (grad != nullptr && (grad_dtype == NOLOCO_F32 || x_dtype == NOLOCO_F32)) ||
                    double(plan->W) * T * l.inputs * l.outputs < noloco::kSmallWork;
  const int32_t dz_dtype = !acts || activation == NOLOCO_ACT_RELU ? dout_dtype : (fine ? NOLOCO_F32 : NOLOCO_BF16);
  const bool sums = grad != nullptr && l.bias >= 0;
  const uint64_t room_dz = acts ? whole(static_cast<uint64_t>(T) * l.outputs * bytes_of(dz_dtype)) : 0, room_sums = sums ? sums_bytes(l, T) : 0;
  const uint64_t packed = packed_bytes(l, T);
  const int32_t batch = room_dz + room_sums == 0 ? plan->W : static_cast<int32_t>(std::min<uint64_t>(plan->W, (plan->room - packed) / (room_dz + room_sums)));
  for (int32_t w = 0; w < plan->W; w += batch) {
    const int32_t W = std::min(batch, plan->W - w);
    char* const dz_room = plan->block.memory;
    const uint64_t used = W * (room_dz + room_sums);
    const void* dz = offset(dout, w * T * l.outputs, dout_dtype);
    if (acts || sums) {
      noloco::SlopeArgs args{};
      args.dout = dz;
      args.before = acts ? offset(before, w * T * l.outputs, dout_dtype) : nullptr;
      args.dz = acts ? dz_room : nullptr;
      args.partial = sums ? reinterpret_cast<float*>(dz_room + W * room_dz) : nullptr;
      args.grad = sums ? offset(grad, w * plan->stride + l.bias, grad_dtype) : nullptr;
      args.stride = plan->stride;
      args.tokens = T;
      args.outputs = static_cast<uint32_t>(l.outputs);
      args.groups = noloco::slope_groups(T);
      args.W = W;
      args.activation = activation;
      args.dout_bf16 = dout_dtype == NOLOCO_BF16;
      args.dz_bf16 = dz_dtype == NOLOCO_BF16;
      args.grad_bf16 = grad_dtype == NOLOCO_BF16;
      args.accumulate = accumulate;
      if (noloco::launch_slope(args, hip_stream) != 0) return NOLOCO_ERR_DEVICE;
      if (acts) dz = dz_room;
    }
    if (dx != nullptr && T > 0) {
      noloco::ProductArgs args{};
      args.a = rows_operand(dz, T, l.outputs, dz_dtype, true);
      args.b = {offset(theta, w * plan->stride + l.offset, theta_dtype), plan->stride, l.row_stride, 1 - l.transposed, theta_dtype == NOLOCO_BF16 ? 1 : 0};
      args.m = static_cast<uint32_t>(T);
      args.n = static_cast<uint32_t>(l.inputs);
      args.k = static_cast<uint32_t>(l.outputs);
      args.W = W;
      args.out = offset(dx, w * T * l.inputs, dx_dtype);
      args.out_stride = T * l.inputs;
      args.out_ld = l.inputs;
      args.out_bf16 = dx_dtype == NOLOCO_BF16;
      args.more = add == nullptr ? nullptr : offset(add, w * T * l.inputs, dx_dtype);
      if (!run_product(args, dz_room + used, plan->room - used, W, hip_stream)) return NOLOCO_ERR_DEVICE;
    }
    if (grad != nullptr) {
      noloco::ProductArgs args{};
      const noloco::Operand of_inputs = rows_operand(x == nullptr ? nullptr : offset(x, w * T * l.inputs, x_dtype), T, l.inputs, x_dtype, false);
      const noloco::Operand of_outputs = rows_operand(dz, T, l.outputs, dz_dtype, false);
      args.a = l.transposed ? of_outputs : of_inputs;
      args.b = l.transposed ? of_inputs : of_outputs;
      args.m = static_cast<uint32_t>(l.transposed ? l.outputs : l.inputs);
      args.n = static_cast<uint32_t>(l.transposed ? l.inputs : l.outputs);
      args.k = static_cast<uint32_t>(T);
      args.W = W;
      args.out = offset(grad, w * plan->stride + l.offset, grad_dtype);
      args.out_stride = plan->stride;
      args.out_ld = l.row_stride;
      args.out_bf16 = grad_dtype == NOLOCO_BF16;
      args.accumulate = accumulate;
      if (!run_product(args, dz_room + used, plan->room - used, W, hip_stream)) return NOLOCO_ERR_DEVICE;
    }
  }
  return NOLOCO_OK;
}

// ---------------------------------------------------------------------------
// Log probabilities
// ---------------------------------------------------------------------------

extern "C" noloco_status noloco_log_prob_plan_create(int64_t vocab, int64_t row_stride, int32_t W, int64_t max_tokens, int32_t max_top,
                                                     noloco_log_prob_plan** out) {
  if (out == nullptr) return NOLOCO_ERR_NULL;
  *out = nullptr;
  if (vocab < 1 || row_stride < vocab || W < 1 || max_tokens < 0 || max_top < 0) return NOLOCO_ERR_INVALID_ARG;
  if (vocab > kMostVocab || W > NOLOCO_MAX_WORKERS || max_top > NOLOCO_MAX_TOP || max_tokens > kMostRows / W) return NOLOCO_ERR_UNSUPPORTED;
  const int64_t rows = W * max_tokens;
  if (rows > 0 && row_stride > (1ll << 60) / rows) return NOLOCO_ERR_UNSUPPORTED;
  std::unique_ptr<noloco_log_prob_plan> plan(new (std::nothrow) noloco_log_prob_plan);
  if (plan == nullptr) return NOLOCO_ERR_NO_MEMORY;
  plan->vocab = vocab;
  plan->row_stride = row_stride;
  plan->max_tokens = max_tokens;
  plan->W = W;
  plan->max_top = max_top;
  // Few rows are cut into more parts than many: the most parts of all are those of any number of rows.
  const uint64_t least = noloco::log_prob_parts(std::numeric_limits<int64_t>::max(), vocab);
  const uint64_t parts = std::max<uint64_t>(least > 1 ? least * rows : 0, 256 + noloco::log_prob_parts(1, vocab));
  plan->parts_bytes = whole(parts * sizeof(noloco::LogPart));
  if (!plan->block.allocate(plan->parts_bytes + whole(parts * max_top * sizeof(uint64_t)))) return NOLOCO_ERR_DEVICE;
  *out = plan.release();
  return NOLOCO_OK;
}

extern "C" noloco_status noloco_log_prob_plan_destroy(noloco_log_prob_plan* plan) { return destroy(plan); }

namespace {

noloco_status log_prob_args(const noloco_log_prob_plan* plan, const void* logits, int32_t logits_dtype, const void* tokens, int32_t token_type,
                            int64_t num_tokens, noloco::LogProbArgs* args) {
  if (num_tokens < 0 || num_tokens > plan->max_tokens) return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens > 0 && (logits == nullptr || tokens == nullptr)) return NOLOCO_ERR_NULL;
  if (!is_dtype(logits_dtype) || (token_type != NOLOCO_I32 && token_type != NOLOCO_I64)) return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(logits, 16) || !aligned(tokens, token_type == NOLOCO_I64 ? 8 : 4)) return NOLOCO_ERR_ALIGNMENT;
  *args = noloco::LogProbArgs{};
  args->logits = logits;
  args->tokens = tokens;
  args->rows = plan->W * num_tokens;
  args->row_stride = plan->row_stride;
  args->vocab = static_cast<uint32_t>(plan->vocab);
  args->logits_bf16 = logits_dtype == NOLOCO_BF16;
  args->tokens_i64 = token_type == NOLOCO_I64;
  return NOLOCO_OK;
}

}  // namespace

extern "C" noloco_status noloco_token_log_probs(const noloco_log_prob_plan* plan, const void* logits, int32_t logits_dtype, const void* tokens,
                                                int32_t token_type, int64_t num_tokens, float* log_probs, float* entropy, float* norms,
                                                int32_t top, int32_t* top_tokens, float* top_log_probs, void* hip_stream) {
  if (plan == nullptr) return NOLOCO_ERR_NULL;
  noloco::LogProbArgs args;
  const noloco_status st = log_prob_args(plan, logits, logits_dtype, tokens, token_type, num_tokens, &args);
  if (st != NOLOCO_OK) return st;
  if (top < 0 || top > plan->max_top) return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens > 0 && (log_probs == nullptr || (top > 0 && (top_tokens == nullptr || top_log_probs == nullptr)))) return NOLOCO_ERR_NULL;
  if (!aligned(log_probs, 4) || !aligned(entropy, 4) || !aligned(norms, 4) || !aligned(top_tokens, 4) || !aligned(top_log_probs, 4)) return NOLOCO_ERR_ALIGNMENT;
  const uint64_t rows = args.rows;
  const Range of_logits{logits, rows * plan->row_stride * bytes_of(logits_dtype)}, of_tokens{tokens, rows * (token_type == NOLOCO_I64 ? 8 : 4)};
  const Range outs[5] = {{log_probs, rows * 4}, {entropy, rows * 4}, {norms, rows * 4},
                         {top > 0 ? top_tokens : nullptr, rows * top * 4}, {top > 0 ? top_log_probs : nullptr, rows * top * 4}};
  for (int i = 0; i < 5; ++i) {
    if (!apart(outs[i], {of_logits, of_tokens})) return NOLOCO_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (!apart(outs[i], {outs[j]})) return NOLOCO_ERR_INVALID_ARG;
  }
  if (num_tokens == 0) return NOLOCO_OK;
  args.log_probs = log_probs;
  args.entropy = entropy;
  args.norms = norms;
  args.top = top;
  args.top_tokens = top_tokens;
  args.top_log_probs = top_log_probs;
  const uint32_t parts = noloco::log_prob_parts(args.rows, plan->vocab);
  args.part = static_cast<uint32_t>((plan->vocab + parts - 1) / parts + 7) / 8 * 8;
  args.num_parts = static_cast<uint32_t>((plan->vocab + args.part - 1) / args.part);
  args.parts = reinterpret_cast<noloco::LogPart*>(plan->block.memory);
  args.keys = reinterpret_cast<uint64_t*>(plan->block.memory + plan->parts_bytes);
  const noloco_status there = check_device(plan->block.device);
  if (there != NOLOCO_OK) return there;
  return noloco::launch_log_probs(args, hip_stream) == 0 ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}

extern "C" noloco_status noloco_token_log_probs_gradient(const noloco_log_prob_plan* plan, const void* logits, int32_t logits_dtype,
                                                         const void* tokens, int32_t token_type, int64_t num_tokens, const float* norms,
                                                         const float* dlog_probs, const float* dentropy, const float* entropy, void* dlogits,
                                                         int32_t dlogits_dtype, void* hip_stream) {
  if (plan == nullptr) return NOLOCO_ERR_NULL;
  noloco::LogProbArgs args;
  const noloco_status st = log_prob_args(plan, logits, logits_dtype, tokens, token_type, num_tokens, &args);
  if (st != NOLOCO_OK) return st;
  if (num_tokens > 0 && (norms == nullptr || dlog_probs == nullptr || dlogits == nullptr || (dentropy != nullptr && entropy == nullptr))) return NOLOCO_ERR_NULL;
  if (!is_dtype(dlogits_dtype)) return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(dlogits, 16) || !aligned(norms, 4) || !aligned(dlog_probs, 4) || !aligned(dentropy, 4) || !aligned(entropy, 4)) return NOLOCO_ERR_ALIGNMENT;
  const uint64_t rows = args.rows, numbers = rows * plan->row_stride;
  const bool in_place = dlogits == logits && dlogits_dtype == logits_dtype;
  const Range of_logits{in_place ? nullptr : logits, numbers * bytes_of(logits_dtype)}, of_tokens{tokens, rows * (token_type == NOLOCO_I64 ? 8 : 4)};
  if (!apart({dlogits, numbers * bytes_of(dlogits_dtype)},
             {of_logits, of_tokens, {norms, rows * 4}, {dlog_probs, rows * 4}, {dentropy, rows * 4}, {entropy, rows * 4}}))
    return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens == 0) return NOLOCO_OK;
  args.norms = const_cast<float*>(norms);
  args.dlog_probs = dlog_probs;
  args.dentropy = dentropy;
  args.entropy = const_cast<float*>(entropy);
  args.dlogits = dlogits;
  args.dlogits_bf16 = dlogits_dtype == NOLOCO_BF16;
  const noloco_status there = check_device(plan->block.device);
  if (there != NOLOCO_OK) return there;
  return noloco::launch_log_probs_gradient(args, hip_stream) == 0 ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}
