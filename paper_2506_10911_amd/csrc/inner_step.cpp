// C ABI of the inner step's operators: argument checking, plans, and the split of a call into kernel launches.  All
// arithmetic is in newton_schulz.hip and embedding.hip.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <limits>
#include <memory>
#include <new>
#include <vector>

#include "inner_internal.h"

namespace {

using noloco::NsArgs;
using noloco::NsArrays;
using noloco::NsClass;
using noloco::NsItem;
using noloco::NsTable;

constexpr int64_t kDefaultWorkspace = 4ll << 30;
constexpr int64_t kMostNumbers = 1ll << 28, kMostSide = 1ll << 22, kMostItems = 1ll << 24;
constexpr uint64_t kMostGroups = 1u << 22;      // workgroups of a launch

bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a_bytes > 0 && b_bytes > 0 && a0 < b0 + b_bytes && b0 < a0 + a_bytes;
}

bool is_dtype(int32_t t) { return t == NOLOCO_F32 || t == NOLOCO_BF16; }
uint64_t bytes_of(int32_t dtype) { return dtype == NOLOCO_BF16 ? 2 : 4; }

uint32_t padded(int64_t v, int tile) { return static_cast<uint32_t>((v + tile - 1) / tile * tile); }

// A plan's tables and workspace are in the memory of the GPU that was current when it was made.
noloco_status check_device(int of_plan) {
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) return NOLOCO_ERR_DEVICE;
  return device == of_plan ? NOLOCO_OK : NOLOCO_ERR_INVALID_ARG;
}

// Matrices of one shape.
struct Shape {
  uint32_t rows, cols;      // as stored
  uint32_t first_item, items;
  // with one binary16 a number, and with pairs
  int tiles[2];
  bool alone[2];            // goes through all steps in one workgroup
  uint32_t parts[2];        // that X X^T is summed in
  uint32_t m() const { return std::min(rows, cols); }
  uint32_t n() const { return std::max(rows, cols); }
  int tile(int planes) const { return tiles[planes - 1]; }
  uint32_t mp(int planes) const { return padded(m(), tile(planes)); }
  uint32_t np(int planes) const { return padded(n(), tile(planes)); }
  uint64_t item_bytes(int planes) const { return noloco::ns_item_bytes(mp(planes), np(planes), planes); }
  uint64_t small_bytes(int planes) const { return noloco::ns_small_bytes(m(), n(), planes); }
  // Four rows of P are what a wave keeps of a column: 128.
  bool small(int planes) const { return alone[planes - 1]; }
  bool fits_lds(int planes) const { return m() <= 128 && uint64_t(m()) * ((n() + 7) / 8 * 8) <= noloco::ns_small_numbers(planes) && small_bytes(planes) <= noloco::kNsSmallLds; }
};

// What goes through the products together: where the tables of its launches are among all of them, and their workgroups.
// Small matrices (tile 0) take one launch of a workgroup each, with the first table.
enum { kSums, kStart, kSymmetric, kApply, kTables };
struct Batch {
  int tile;
  uint32_t first_table;
  uint32_t groups[kTables];
  uint32_t lds;             // of a workgroup of small matrices
  uint32_t splits;          // the most of the classes
  NsClass first[kTables];   // of the tables
  uint32_t first_end[kTables];
};

// Tiles of 256 have the highest rate (eight matrices of 4096^2, binary16, us a step: 1972, tiles of 128 2556) but take whole
// CUs: with less than two rounds of them smaller ones are ahead (eight of 2048^2 327 / 285, thirty-two 1060 / 1254), and below
// 1024 rows too (96 of 768^2 in pairs 685 / 630; 48 of 768 x 3072 1091 / 971).  Tiles of 64 pay where there are less of 128
// than CUs: one 1024 x 4096 39 / 70, four of 768^2 32 / 37, eight 44 / 48, sixteen (336 tiles) 72 / 74, one of 2048^2 76 / 76.
// Tiles of X X^T are counted, of all matrices that go through launches together in the format that is asked for (256 of 128 x 256
// in pairs: tiles of 64 249 us, of 128 221; 1152 1054 and 946).
constexpr int64_t kTiles256 = 512, kTiles128 = 256, kRows256 = 1024, kJoined = 256;

int64_t lower_tiles(int64_t m, int tile) {
  const int64_t t = padded(m, tile) / tile;
  return t * (t + 1) / 2;
}

// X has to be one buffer, whose offsets have 32 bits.
bool one_buffer(int64_t m, int64_t n, int tile, int planes) { return noloco::ns_x_bytes(padded(m, tile), padded(n, tile), planes) >> 32 == 0; }

// Padding to 256 may cost a tenth of the products.
bool pads_well(int64_t m, int64_t n, int planes) {
  const double big = double(padded(m, 256)) * padded(m, 256) * padded(n, 256), less = double(padded(m, 128)) * padded(m, 128) * padded(n, 128);
  return m >= kRows256 && big <= 1.1 * less && one_buffer(m, n, 256, planes);
}

// X X^T of few rows is few tiles of long sums: where there are less tiles than twice the CUs the long side is shared out, as
// long as each share has kShare stages (64 numbers, or 32 pairs) and the shares' sums have room where the next X comes.  Adding
// them up is a launch more: five steps of float matrices with 33 stages (ragged, up to 1031) 164 us, shared out 184; with 125
// (eight of 64 x 4000) 193 / 121; with 512 (130 x 16384) 546 / 166; 16384 x 1 in bf16 507 / 116.
constexpr int64_t kSplitGroups = 512, kSplitStages = 48, kShare = 8, kMostSplits = 64;

void choose_tiles(std::vector<Shape>* shapes, int planes) {
  int64_t big = 0, all = 0;
  for (const Shape& s : *shapes) {
    if (s.fits_lds(planes)) continue;
    if (pads_well(s.m(), s.n(), planes)) big += s.items * lower_tiles(s.m(), 256);
    all += s.items * lower_tiles(s.m(), 128);
  }
  for (Shape& s : *shapes) {
    int& tile = s.tiles[planes - 1];
    tile = all < kTiles128 ? 64 : (big >= kTiles256 && pads_well(s.m(), s.n(), planes) ? 256 : 128);
    if (!one_buffer(s.m(), s.n(), tile, planes)) tile = 64;
  }
  // Small matrices beside others of their tile: the others' launches are there anyway, and up to kJoined tiles of P X more cost them
  // less than a launch of their own, which lasts as long as its slowest workgroup (ragged float matrices, 32 small ones 41 us of
  // 212).  Beside others of another tile they would need launches of their own for each product.
  bool others[257] = {};
  int64_t tiles = 0;
  for (const Shape& s : *shapes) {
    if (!s.fits_lds(planes)) others[s.tile(planes)] = true;
    else tiles += int64_t(s.items) * (s.mp(planes) / s.tile(planes)) * (s.np(planes) / s.tile(planes));
  }
  int64_t grams = 0;
  for (Shape& s : *shapes) {
    s.alone[planes - 1] = s.fits_lds(planes) && !(others[s.tile(planes)] && tiles <= kJoined);
    if (!s.alone[planes - 1]) grams += s.items * lower_tiles(s.m(), s.tile(planes));
  }
  for (Shape& s : *shapes) {
    s.parts[planes - 1] = 1;
    if (s.alone[planes - 1] || s.tile(planes) != noloco::kNsSplitTile) continue;
    const int64_t stages = (s.n() + 64 / planes - 1) / (64 / planes);
    if (stages < kSplitStages) continue;
    const int64_t room = noloco::ns_x_bytes(s.mp(planes), s.np(planes), planes) / (lower_tiles(s.m(), s.tile(planes)) * noloco::kNsSplitBytes);
    s.parts[planes - 1] = static_cast<uint32_t>(std::max<int64_t>(1, std::min({kSplitGroups / grams, stages / kShare, room, kMostSplits})));
  }
}

}  // namespace

struct noloco_muon_plan {
  int device = -1;
  int32_t W = 0;
  int64_t stride = 0;
  int64_t elements = 0;
  int64_t workspace_bytes = 0;
  std::vector<Batch> batches[2];     // one binary16 a number, pairs
  bool pairs = false;                // also bf16 results take pairs
  const NsTable* tables = nullptr;   // these four point into the block
  const NsItem* items = nullptr;
  double* sums = nullptr;
  char* workspace = nullptr;
  char* block = nullptr;             // the one device allocation

  noloco_muon_plan() = default;
  noloco_muon_plan(const noloco_muon_plan&) = delete;
  noloco_muon_plan& operator=(const noloco_muon_plan&) = delete;
  ~noloco_muon_plan() {
    if (block != nullptr) (void)hipFree(block);
  }
};

struct noloco_embedding_plan {
  int device = -1;
  int64_t offset = 0, vocab = 0, width = 0, stride = 0, max_tokens = 0;
  int32_t W = 0;
  char* block = nullptr;
  uint32_t* lists[4] = {};          // tokens and positions, twice
  float* partial = nullptr;

  noloco_embedding_plan() = default;
  noloco_embedding_plan(const noloco_embedding_plan&) = delete;
  noloco_embedding_plan& operator=(const noloco_embedding_plan&) = delete;
  ~noloco_embedding_plan() {
    if (block != nullptr) (void)hipFree(block);
  }
};

namespace {

// Do two matrices share an element?  Those whose rows touch each other are one run of elements, others a run for each row.
noloco_status check_overlap(const std::vector<noloco_matrix>& matrices) {
  std::vector<std::pair<int64_t, int64_t>> runs;
  for (const noloco_matrix& m : matrices) {
    if (m.row_stride == m.cols || m.rows == 1) {
      runs.emplace_back(m.offset, m.offset + m.rows * m.cols);
    } else {
      for (int64_t r = 0; r < m.rows; ++r) runs.emplace_back(m.offset + r * m.row_stride, m.offset + r * m.row_stride + m.cols);
    }
  }
  std::sort(runs.begin(), runs.end());
  for (size_t i = 1; i < runs.size(); ++i)
    if (runs[i].first < runs[i - 1].second) return NOLOCO_ERR_SEGMENT_OVERLAP;
  return NOLOCO_OK;
}

// Splits the items of all shapes into batches that fit `room` bytes and a launch's table of classes.  Returns the most items
// that a batch has.
uint32_t make_batches(std::vector<Shape> shapes, int planes, uint64_t room, std::vector<Batch>* out, std::vector<NsTable>* tables) {
  // Small ones last and by size: a launch claims as much LDS as its largest matrix needs.  Where there are more of them than
  // CUs, those that let two workgroups share a CU have a launch of their own.
  uint64_t smalls = 0;
  for (const Shape& s : shapes) smalls += s.small(planes) ? s.items : 0;
  auto sharing = [&](const Shape& s) { return smalls <= 256 ? 1 : std::min<uint64_t>(noloco::kNsSmallLds / s.small_bytes(planes), 2); };
  std::stable_sort(shapes.begin(), shapes.end(), [&](const Shape& a, const Shape& b) {
    const bool as = a.small(planes), bs = b.small(planes);
    if (as != bs) return bs;
    return as ? a.small_bytes(planes) > b.small_bytes(planes) : a.tile(planes) > b.tile(planes);
  });
  size_t shape = 0;
  uint32_t done = 0, most = 0;      // of that shape's items; of a batch
  while (shape < shapes.size()) {
    const Shape& head = shapes[shape];
    const bool small = head.small(planes);
    Batch b{};
    b.tile = small ? 0 : head.tile(planes);
    b.lds = small ? static_cast<uint32_t>(head.small_bytes(planes)) : 0;
    b.first_table = static_cast<uint32_t>(tables->size());
    NsTable table[kTables];
    for (NsTable& t : table) {
      std::fill(t.end, t.end + noloco::kNsClasses, 0xffffffffu);
      std::fill(t.cls, t.cls + noloco::kNsClasses, NsClass{});
    }
    uint64_t used = 0;
    uint32_t items = 0;
    int classes = 0;
    while (shape < shapes.size() && classes < noloco::kNsClasses) {
      const Shape& s = shapes[shape];
      if (s.small(planes) != small || (small ? sharing(s) != sharing(head) : s.tile(planes) != b.tile)) break;
      const uint64_t each = small ? 0 : s.item_bytes(planes), elements = uint64_t(s.rows) * s.cols;
      const uint32_t mt = s.mp(planes) / s.tile(planes), nt = s.np(planes) / s.tile(planes);
      const uint32_t chunks = static_cast<uint32_t>(std::min<uint64_t>(std::max<uint64_t>((elements + noloco::kNsChunkElems - 1) / noloco::kNsChunkElems, 1), noloco::kNsChunks));
      const uint32_t per[kTables] = {small ? 1 : chunks, s.mp(planes) / 64 * (s.np(planes) / 64), mt * (mt + 1) / 2, mt * nt};
      uint64_t fit = s.items - done;
      if (!small) fit = std::min<uint64_t>(fit, (room - used) / each);
      for (int k = 0; k < (small ? 1 : kTables); ++k) {
        const uint64_t left = b.groups[k] < kMostGroups ? kMostGroups - b.groups[k] : 0;
        fit = std::min(fit, std::max<uint64_t>(left / per[k], items == 0 ? 1 : 0));
      }
      if (fit == 0) break;
      NsClass c{};
      c.base = used;
      c.item_bytes = each;
      c.first_item = s.first_item + done;
      c.first_sum = items;
      c.m = s.m();
      c.n = s.n();
      c.mp = s.mp(planes);
      c.np = s.np(planes);
      c.tall = s.rows > s.cols ? 1 : 0;
      c.splits = s.parts[planes - 1];
      b.splits = std::max(b.splits, c.splits);
      for (int k = 0; k < (small ? 1 : kTables); ++k) {
        c.per_item = per[k];
        b.groups[k] += per[k] * static_cast<uint32_t>(fit);
        table[k].cls[classes] = c;
        table[k].end[classes] = b.groups[k];
      }
      ++classes;
      used += each * fit;
      items += static_cast<uint32_t>(fit);
      done += static_cast<uint32_t>(fit);
      if (done < s.items) break;
      ++shape;
      done = 0;
    }
    for (int k = 0; k < kTables; ++k) {
      b.first[k] = table[k].cls[0];
      b.first_end[k] = table[k].end[0];
    }
    out->push_back(b);
    tables->insert(tables->end(), table, table + (small ? 1 : kTables));
    if (!small) most = std::max(most, items);
  }
  return most;
}

noloco_status create_muon_plan(const noloco_matrix* given, int32_t num, int64_t stride, int32_t W, int64_t workspace,
                               noloco_muon_plan** out) {
  std::unique_ptr<noloco_muon_plan> plan(new noloco_muon_plan);
  plan->W = W;
  plan->stride = stride;
  std::vector<noloco_matrix> matrices;
  for (int32_t i = 0; i < num; ++i) {
    const noloco_matrix& m = given[i];
    if (m.offset < 0 || m.rows < 0 || m.cols < 0 || m.row_stride < m.cols || !std::isfinite(m.scale)) return NOLOCO_ERR_INVALID_ARG;
    if (m.rows == 0 || m.cols == 0) continue;
    if (m.rows > kMostSide || m.cols > kMostSide || m.rows * m.cols > kMostNumbers) return NOLOCO_ERR_UNSUPPORTED;
    // the last element's place, without a product that could overflow
    if (m.offset > stride || m.cols > stride - m.offset) return NOLOCO_ERR_SEGMENT_OVERLAP;
    if (m.rows > 1 && m.row_stride > (stride - m.offset - m.cols) / (m.rows - 1)) return NOLOCO_ERR_SEGMENT_OVERLAP;
    matrices.push_back(m);
    plan->elements += m.rows * m.cols;
  }
  if (static_cast<int64_t>(matrices.size()) * W > kMostItems) return NOLOCO_ERR_UNSUPPORTED;
  const noloco_status st = check_overlap(matrices);
  if (st != NOLOCO_OK) return st;

  // Those with the longest products first, so that a launch does not end with them.
  std::stable_sort(matrices.begin(), matrices.end(), [](const noloco_matrix& a, const noloco_matrix& b) {
    const int64_t an = std::max(a.rows, a.cols), bn = std::max(b.rows, b.cols);
    if (an != bn) return an > bn;
    if (a.rows * a.cols != b.rows * b.cols) return a.rows * a.cols > b.rows * b.cols;
    return a.rows > b.rows;
  });
  std::vector<Shape> shapes;
  std::vector<NsItem> items;
  for (size_t i = 0; i < matrices.size();) {
    size_t end = i;
    Shape s{};
    s.rows = static_cast<uint32_t>(matrices[i].rows);
    s.cols = static_cast<uint32_t>(matrices[i].cols);
    s.first_item = static_cast<uint32_t>(items.size());
    while (end < matrices.size() && matrices[end].rows == matrices[i].rows && matrices[end].cols == matrices[i].cols) {
      for (int32_t w = 0; w < W; ++w)
        items.push_back(NsItem{w * stride + matrices[end].offset, matrices[end].row_stride, matrices[end].scale, 0});
      ++end;
    }
    s.items = static_cast<uint32_t>(items.size()) - s.first_item;
    shapes.push_back(s);
    i = end;
  }
  for (int planes = 1; planes <= 2; ++planes) choose_tiles(&shapes, planes);
  plan->pairs = std::all_of(shapes.begin(), shapes.end(), [](const Shape& s) { return s.fits_lds(2) || (s.m() <= 64 && !s.fits_lds(1)); });

  uint64_t all[2] = {0, 0}, largest = 0;
  for (const Shape& s : shapes)
    for (int planes = 1; planes <= 2; ++planes)
      if (!s.small(planes)) {
        all[planes - 1] += s.item_bytes(planes) * s.items;
        largest = std::max(largest, s.item_bytes(planes));
      }
  const uint64_t room = std::max(largest, std::min(std::max(all[0], all[1]), static_cast<uint64_t>(workspace > 0 ? workspace : kDefaultWorkspace)));
  plan->workspace_bytes = static_cast<int64_t>(room);
  std::vector<NsTable> tables;
  uint32_t summed = 0;
  for (int planes = 1; planes <= 2; ++planes)
    summed = std::max(summed, make_batches(shapes, planes, room, &plan->batches[planes - 1], &tables));
  // Tables and items, filled by one copy; then the sums and the workspace.
  std::vector<char> host;
  auto append = [&host](const void* data, size_t bytes) {
    const size_t at = host.size();
    host.resize((at + bytes + 4095) / 4096 * 4096);
    if (bytes > 0) std::memcpy(host.data() + at, data, bytes);
    return at;
  };
  const size_t tables_at = append(tables.data(), tables.size() * sizeof(NsTable));
  const size_t items_at = append(items.data(), items.size() * sizeof(NsItem));
  const uint64_t sum_bytes = (uint64_t(summed) * noloco::kNsChunks * sizeof(double) + 4095) / 4096 * 4096;
  if (hipGetDevice(&plan->device) != hipSuccess ||
      hipMalloc(reinterpret_cast<void**>(&plan->block), host.size() + sum_bytes + room + 4096) != hipSuccess) {
    plan->block = nullptr;
    return NOLOCO_ERR_DEVICE;
  }
  if (!host.empty() && hipMemcpy(plan->block, host.data(), host.size(), hipMemcpyHostToDevice) != hipSuccess)
    return NOLOCO_ERR_DEVICE;
  plan->tables = reinterpret_cast<const NsTable*>(plan->block + tables_at);
  plan->items = reinterpret_cast<const NsItem*>(plan->block + items_at);
  plan->sums = reinterpret_cast<double*>(plan->block + host.size());
  plan->workspace = plan->block + host.size() + sum_bytes;
  *out = plan.release();
  return NOLOCO_OK;
}

// Do the coefficients keep what binary16 holds in its range?  Singular values start at most at 1.
noloco_status check_method(const noloco_newton_schulz* method) {
  if (method == nullptr || method->coefficients == nullptr) return NOLOCO_ERR_NULL;
  if (method->steps > NOLOCO_MAX_NEWTON_SCHULZ_STEPS) return NOLOCO_ERR_UNSUPPORTED;
  if (method->steps < 1 || !(method->eps >= 0.f) || !std::isfinite(method->eps)) return NOLOCO_ERR_INVALID_ARG;
  if (method->products < NOLOCO_PRODUCTS_AUTO || method->products > NOLOCO_PRODUCTS_PAIRS) return NOLOCO_ERR_INVALID_ARG;
  for (int32_t i = 0; i < 3 * method->steps; ++i)
    if (!std::isfinite(method->coefficients[i])) return NOLOCO_ERR_INVALID_ARG;
  double most = 1.002;      // of a singular value, with room for the rounding of X
  for (int32_t s = 0; s < method->steps; ++s) {
    const double a = method->coefficients[3 * s], b = method->coefficients[3 * s + 1], c = method->coefficients[3 * s + 2];
    auto poly = [&](double square) { return a + square * (b + square * c); };
    const double square = most * most;
    // extremes of P on [0, square], and of x P(x^2) on [0, most]
    double p = std::max(std::fabs(a), std::fabs(poly(square))), x = most * std::fabs(poly(square));
    if (c != 0. && -b / (2 * c) > 0. && -b / (2 * c) < square) p = std::max(p, std::fabs(poly(-b / (2 * c))));
    const double root = 9 * b * b - 20 * a * c;
    double at[2] = {-1., -1.};
    if (c == 0.) {
      if (b != 0.) at[0] = -a / (3 * b);
    } else if (root >= 0.) {
      at[0] = (-3 * b + std::sqrt(root)) / (10 * c);
      at[1] = (-3 * b - std::sqrt(root)) / (10 * c);
    }
    for (double v : at)
      if (v > 0. && v < square) x = std::max(x, std::sqrt(v) * std::fabs(poly(v)));
    most = x * 1.002;
    if (!(p <= noloco::kNsMostP) || !(most * most <= noloco::kNsMostA)) return NOLOCO_ERR_UNSUPPORTED;
  }
  return NOLOCO_OK;
}

noloco_status run_batches(const noloco_muon_plan* plan, const NsArrays& arrays, const noloco_newton_schulz* method, void* stream) {
  // One binary16 a number leaves an error below a bf16 result's own rounding (0.0005 to 0.0011 of the norm, the rounding 0.0017),
  // the more the fewer numbers average it and the smaller the least singular value is (4 x 4 and 8 x 8 of noise 0.0014, one in a
  // hundred 0.006).  Small matrices, whose step waits more than it computes, take pairs (us, binary16 and pairs: eight of 16 x 64
  // 16.4 / 15.6, 32 of 64 x 64 19.0 / 21.7) and have the rounding alone.  So have long ones of few rows that go through launches
  // (4 x 6000 beside nothing larger 94 / 113, eight of 64 x 4000 95 / 119, errors 0.0017 either way).
  const bool one = method->products == NOLOCO_PRODUCTS_F16 || (method->products == NOLOCO_PRODUCTS_AUTO && arrays.out_bf16 && !plan->pairs);
  const int planes = one ? 1 : 2;
  if (plan->batches[planes - 1].empty()) return NOLOCO_OK;
  const noloco_status st = check_device(plan->device);
  if (st != NOLOCO_OK) return st;
  noloco::NsSteps steps{};
  steps.count = method->steps;
  std::copy(method->coefficients, method->coefficients + 3 * method->steps, steps.k);
  for (const Batch& b : plan->batches[planes - 1]) {
    auto args = [&](int table) { return NsArgs{plan->tables + b.first_table + table, plan->items, plan->workspace, plan->sums, b.splits, b.first[table], b.first_end[table]}; };
    if (b.tile == 0) {
      if (noloco::launch_ns_small(args(kSums), arrays, steps, planes, b.groups[kSums], b.lds, stream) != 0) return NOLOCO_ERR_DEVICE;
      continue;
    }
    if (noloco::launch_ns_sums(args(kSums), arrays, b.groups[kSums], stream) != 0) return NOLOCO_ERR_DEVICE;
    if (noloco::launch_ns_start(args(kStart), arrays, planes, b.groups[kStart], stream) != 0) return NOLOCO_ERR_DEVICE;
    for (int32_t s = 0; s < method->steps; ++s) {
      const float* k = method->coefficients + 3 * s;
      const int kinds[3] = {noloco::kNsGram, noloco::kNsSquare, s + 1 == method->steps ? noloco::kNsLast : noloco::kNsApply};
      for (int kind : kinds) {
        const int table = kind == noloco::kNsGram || kind == noloco::kNsSquare ? kSymmetric : kApply;
        if (noloco::launch_ns_product(args(table), arrays, kind, b.tile, planes, s, k[0], k[1], k[2], b.groups[table], stream) != 0)
          return NOLOCO_ERR_DEVICE;
      }
    }
  }
  return NOLOCO_OK;
}

}  // namespace

extern "C" noloco_status noloco_muon_plan_create(const noloco_matrix* matrices, int32_t num_matrices, int64_t worker_stride,
                                                 int32_t W, int64_t workspace_bytes, noloco_muon_plan** out) {
  if (out == nullptr) return NOLOCO_ERR_NULL;
  *out = nullptr;
  if (num_matrices < 0 || worker_stride < 0 || W < 1 || workspace_bytes < 0) return NOLOCO_ERR_INVALID_ARG;
  if (matrices == nullptr && num_matrices > 0) return NOLOCO_ERR_NULL;
  if (W > NOLOCO_MAX_WORKERS) return NOLOCO_ERR_UNSUPPORTED;
  if (worker_stride > std::numeric_limits<int64_t>::max() / 8 / W) return NOLOCO_ERR_UNSUPPORTED;
  if (worker_stride % NOLOCO_STRIDE_ALIGN_ELEMS != 0) return NOLOCO_ERR_ALIGNMENT;
  try {
    return create_muon_plan(matrices, num_matrices, worker_stride, W, workspace_bytes, out);
  } catch (const std::bad_alloc&) {
    return NOLOCO_ERR_NO_MEMORY;
  } catch (...) {
    return NOLOCO_ERR_INVALID_ARG;
  }
}

extern "C" noloco_status noloco_muon_plan_destroy(noloco_muon_plan* plan) {
  if (plan == nullptr) return NOLOCO_OK;
  noloco_status st = NOLOCO_OK;
  if (plan->block != nullptr && hipFree(plan->block) != hipSuccess) st = NOLOCO_ERR_DEVICE;
  plan->block = nullptr;
  delete plan;
  return st;
}

extern "C" noloco_status noloco_muon_plan_info(const noloco_muon_plan* plan, int64_t* elements_per_worker,
                                               int64_t* workspace_bytes, int32_t* bf16_batches, int32_t* f32_batches) {
  if (plan == nullptr) return NOLOCO_ERR_NULL;
  if (elements_per_worker != nullptr) *elements_per_worker = plan->elements;
  if (workspace_bytes != nullptr) *workspace_bytes = plan->workspace_bytes;
  if (bf16_batches != nullptr) *bf16_batches = static_cast<int32_t>(plan->batches[0].size());
  if (f32_batches != nullptr) *f32_batches = static_cast<int32_t>(plan->batches[1].size());
  return NOLOCO_OK;
}

extern "C" noloco_status noloco_orthogonalize(const noloco_muon_plan* plan, const void* x, int32_t x_dtype, void* out,
                                              int32_t out_dtype, const noloco_newton_schulz* method, void* hip_stream) {
  if (plan == nullptr || x == nullptr || out == nullptr) return NOLOCO_ERR_NULL;
  const noloco_status st = check_method(method);
  if (st != NOLOCO_OK) return st;
  if (!is_dtype(x_dtype) || !is_dtype(out_dtype)) return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(x, NOLOCO_BASE_ALIGN_BYTES) || !aligned(out, NOLOCO_BASE_ALIGN_BYTES)) return NOLOCO_ERR_ALIGNMENT;
  const uint64_t numbers = static_cast<uint64_t>(plan->W) * static_cast<uint64_t>(plan->stride);
  if (!(x == out && x_dtype == out_dtype) && overlap(x, numbers * bytes_of(x_dtype), out, numbers * bytes_of(out_dtype)))
    return NOLOCO_ERR_INVALID_ARG;
  NsArrays arrays{};
  arrays.in = x;
  arrays.out = out;
  arrays.in_bf16 = x_dtype == NOLOCO_BF16;
  arrays.out_bf16 = out_dtype == NOLOCO_BF16;
  arrays.eps = method->eps;
  return run_batches(plan, arrays, method, hip_stream);
}

extern "C" noloco_status noloco_muon_step(const noloco_muon_plan* plan, void* theta, int32_t theta_dtype, const void* grad,
                                          int32_t grad_dtype, float* momentum, const noloco_muon_hparams* hparams,
                                          const noloco_newton_schulz* method, void* hip_stream) {
  if (plan == nullptr || theta == nullptr || grad == nullptr || momentum == nullptr || hparams == nullptr) return NOLOCO_ERR_NULL;
  const noloco_status st = check_method(method);
  if (st != NOLOCO_OK) return st;
  if (!is_dtype(theta_dtype) || !is_dtype(grad_dtype) || (hparams->nesterov != 0 && hparams->nesterov != 1)) return NOLOCO_ERR_INVALID_ARG;
  if (!aligned(theta, NOLOCO_BASE_ALIGN_BYTES) || !aligned(grad, NOLOCO_BASE_ALIGN_BYTES) || !aligned(momentum, NOLOCO_BASE_ALIGN_BYTES))
    return NOLOCO_ERR_ALIGNMENT;
  const uint64_t numbers = static_cast<uint64_t>(plan->W) * static_cast<uint64_t>(plan->stride);
  const uint64_t tb = numbers * bytes_of(theta_dtype), gb = numbers * bytes_of(grad_dtype), mb = numbers * 4;
  if (overlap(theta, tb, grad, gb) || overlap(theta, tb, momentum, mb) || overlap(grad, gb, momentum, mb)) return NOLOCO_ERR_INVALID_ARG;
  NsArrays arrays{};
  arrays.in = grad;
  arrays.momentum = momentum;
  arrays.out = theta;
  arrays.in_bf16 = grad_dtype == NOLOCO_BF16;
  arrays.out_bf16 = theta_dtype == NOLOCO_BF16;
  arrays.mu = hparams->mu;
  arrays.nesterov = hparams->nesterov;
  arrays.keep = static_cast<float>(1.0 - static_cast<double>(hparams->lr) * hparams->weight_decay);
  arrays.lr = hparams->lr;
  arrays.update = 1;
  arrays.eps = method->eps;
  return run_batches(plan, arrays, method, hip_stream);
}

// ---------------------------------------------------------------------------
// Embedding
// ---------------------------------------------------------------------------

extern "C" noloco_status noloco_embedding_plan_create(int64_t offset, int64_t vocab, int64_t width, int64_t worker_stride,
                                                      int32_t W, int64_t max_tokens, noloco_embedding_plan** out) {
  if (out == nullptr) return NOLOCO_ERR_NULL;
  *out = nullptr;
  if (offset < 0 || vocab < 1 || width < 1 || worker_stride < 0 || W < 1 || max_tokens < 0) return NOLOCO_ERR_INVALID_ARG;
  if (W > NOLOCO_MAX_WORKERS || vocab > (1 << 29) || width > (1 << 24) || max_tokens > (1 << 27) ||
      W * max_tokens > std::numeric_limits<int32_t>::max() || worker_stride > std::numeric_limits<int64_t>::max() / 8 / W)
    return NOLOCO_ERR_UNSUPPORTED;
  if (worker_stride % NOLOCO_STRIDE_ALIGN_ELEMS != 0) return NOLOCO_ERR_ALIGNMENT;
  if (offset > worker_stride || vocab > (worker_stride - offset) / width) return NOLOCO_ERR_SEGMENT_OVERLAP;
  std::unique_ptr<noloco_embedding_plan> plan(new (std::nothrow) noloco_embedding_plan);
  if (plan == nullptr) return NOLOCO_ERR_NO_MEMORY;
  plan->offset = offset;
  plan->vocab = vocab;
  plan->width = width;
  plan->stride = worker_stride;
  plan->W = W;
  plan->max_tokens = max_tokens;
  auto whole = [](uint64_t bytes) { return (bytes + 255) / 256 * 256; };
  const uint64_t list = whole(static_cast<uint64_t>(W) * max_tokens * sizeof(uint32_t));
  const uint64_t chunks = static_cast<uint64_t>(max_tokens + noloco::kSumChunk - 1) / noloco::kSumChunk;
  const uint64_t partial = static_cast<uint64_t>(W) * chunks * 2 * width * sizeof(float);
  if (hipGetDevice(&plan->device) != hipSuccess ||
      hipMalloc(reinterpret_cast<void**>(&plan->block), 4 * list + partial + 256) != hipSuccess) {
    plan->block = nullptr;
    return NOLOCO_ERR_DEVICE;
  }
  for (int i = 0; i < 4; ++i) plan->lists[i] = reinterpret_cast<uint32_t*>(plan->block + i * list);
  plan->partial = reinterpret_cast<float*>(plan->block + 4 * list);
  *out = plan.release();
  return NOLOCO_OK;
}

extern "C" noloco_status noloco_embedding_plan_destroy(noloco_embedding_plan* plan) {
  if (plan == nullptr) return NOLOCO_OK;
  noloco_status st = NOLOCO_OK;
  if (plan->block != nullptr && hipFree(plan->block) != hipSuccess) st = NOLOCO_ERR_DEVICE;
  plan->block = nullptr;
  delete plan;
  return st;
}

namespace {

// Checks what lookup and gradient share; fills the kernels' arguments.
noloco_status embed_args(const noloco_embedding_plan* plan, const void* table, int32_t table_dtype, const void* rows,
                         int32_t rows_dtype, const void* tokens, int32_t token_type, int64_t num_tokens, float scale,
                         noloco::EmbedArgs* out) {
  if (plan == nullptr || table == nullptr) return NOLOCO_ERR_NULL;
  if (num_tokens < 0 || num_tokens > plan->max_tokens) return NOLOCO_ERR_INVALID_ARG;
  if (num_tokens > 0 && (rows == nullptr || tokens == nullptr)) return NOLOCO_ERR_NULL;
  if (!is_dtype(table_dtype) || !is_dtype(rows_dtype) || (token_type != NOLOCO_I32 && token_type != NOLOCO_I64))
    return NOLOCO_ERR_INVALID_ARG;
  const uint64_t token_bytes = token_type == NOLOCO_I64 ? 8 : 4;
  if (!aligned(table, NOLOCO_BASE_ALIGN_BYTES) || !aligned(rows, 16) || !aligned(tokens, token_bytes)) return NOLOCO_ERR_ALIGNMENT;
  const uint64_t tokens_all = static_cast<uint64_t>(plan->W) * num_tokens;
  const uint64_t table_all = static_cast<uint64_t>(plan->W) * plan->stride * bytes_of(table_dtype);
  const uint64_t rows_all = tokens_all * plan->width * bytes_of(rows_dtype);
  if (overlap(table, table_all, rows, rows_all) || overlap(tokens, tokens_all * token_bytes, rows, rows_all) ||
      overlap(table, table_all, tokens, tokens_all * token_bytes))
    return NOLOCO_ERR_INVALID_ARG;
  *out = noloco::EmbedArgs{};
  out->table = static_cast<char*>(const_cast<void*>(table)) + plan->offset * static_cast<int64_t>(bytes_of(table_dtype));
  out->rows = const_cast<void*>(rows);
  out->tokens = tokens;
  out->stride = plan->stride;
  out->num_tokens = num_tokens;
  out->vocab = static_cast<uint32_t>(plan->vocab);
  out->width = static_cast<uint32_t>(plan->width);
  out->W = plan->W;
  out->scale = scale;
  out->table_bf16 = table_dtype == NOLOCO_BF16;
  out->rows_bf16 = rows_dtype == NOLOCO_BF16;
  out->tokens_i64 = token_type == NOLOCO_I64;
  out->vectors = (plan->width | plan->offset) % 8 == 0 ? 8 : ((plan->width | plan->offset) % 4 == 0 ? 4 : 1);
  for (int i = 0; i < 2; ++i) {
    out->token[i] = plan->lists[2 * i];
    out->position[i] = plan->lists[2 * i + 1];
  }
  out->partial = plan->partial;
  return NOLOCO_OK;
}

}  // namespace

extern "C" noloco_status noloco_embed_lookup(const noloco_embedding_plan* plan, const void* table, int32_t table_dtype,
                                             const void* tokens, int32_t token_type, int64_t num_tokens, float scale,
                                             void* out, int32_t out_dtype, void* hip_stream) {
  noloco::EmbedArgs args;
  const noloco_status st = embed_args(plan, table, table_dtype, out, out_dtype, tokens, token_type, num_tokens, scale, &args);
  if (st != NOLOCO_OK) return st;
  if (num_tokens == 0) return NOLOCO_OK;
  const noloco_status there = check_device(plan->device);
  if (there != NOLOCO_OK) return there;
  return noloco::launch_embed_lookup(args, hip_stream) == 0 ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}

extern "C" noloco_status noloco_embed_gradient(const noloco_embedding_plan* plan, const void* dout, int32_t dout_dtype,
                                               const void* tokens, int32_t token_type, int64_t num_tokens, float scale,
                                               void* grad, int32_t grad_dtype, int32_t accumulate, void* hip_stream) {
  if (accumulate != 0 && accumulate != 1) return NOLOCO_ERR_INVALID_ARG;
  noloco::EmbedArgs args;
  const noloco_status st = embed_args(plan, grad, grad_dtype, dout, dout_dtype, tokens, token_type, num_tokens, scale, &args);
  if (st != NOLOCO_OK) return st;
  args.accumulate = accumulate;
  if (num_tokens == 0 && accumulate) return NOLOCO_OK;
  const noloco_status there = check_device(plan->device);
  if (there != NOLOCO_OK) return there;
  return noloco::launch_embed_gradient(args, hip_stream) == 0 ? NOLOCO_OK : NOLOCO_ERR_DEVICE;
}
