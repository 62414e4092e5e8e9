// Host side of the activation operators declared in gws.h: 8-bit activation checkpoints, the weight gradient from a checkpoint
// the gated feed-forward block and the linear layer with epilogue.  Argument validation, tensor maps, choice of tile and launch geometry; no device memory is
// allocated here.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "gws.h"
#include "gws_host.h"
#include "gws_linear.cuh"
#include "gws_tc.cuh"

namespace {

bool is_act8(int format) { return format == GWS_ACT8_INT8 || format == GWS_ACT8_E4M3; }

// ---- layout of a checkpoint --------------------------------------------------------------------------------------------
int64_t act8_ld(int64_t cols) { return round_up(cols, kGroup); }
int64_t act8_codes(int64_t rows, int64_t cols) { return rows * act8_ld(cols); }
int64_t act8_total(int64_t rows, int64_t cols) { return round_up(act8_codes(rows, cols), 256) + rows * (act8_ld(cols) / kGroup); }
Act8View act8_view(const void* buffer, int64_t rows, int64_t cols) {
  uint8_t* p = static_cast<uint8_t*>(const_cast<void*>(buffer));
  return {p, p + round_up(act8_codes(rows, cols), 256), act8_ld(cols)};
}
int zero(void* p, int64_t rows, int64_t cols, int64_t ld, cudaStream_t s) {
  if (p == nullptr || rows == 0 || cols == 0) return GWS_OK;
  const cudaError_t err = cudaMemset2DAsync(p, static_cast<size_t>(ld) * 2u, 0, static_cast<size_t>(cols) * 2u, static_cast<size_t>(rows), s);
  return err == cudaSuccess ? GWS_OK : gws::report_cuda(err, "clearing a gradient");
}

// Whether every group of a [rows, cols] BF16 tensor is 64 whole bytes on a 32-byte boundary: a thread then takes a group.
bool whole_groups(const void* p, int64_t cols, int64_t ld) { return cols % kGroup == 0 && ld % 16 == 0 && on(p, 32); }

int launch_act8(bool save, int format, const void* x, int64_t ldx, const Act8View& c, int64_t rows, int64_t cols, cudaStream_t s) {
  const int64_t per_row = c.ld / kGroup, groups = rows * per_row;
  const bool fast = whole_groups(x, cols, ldx), i8 = format == GWS_ACT8_INT8;
  if (groups / 8 >= 0x7FFFFFFFLL) return GWS_ERR_LIMIT;
  uint16_t* px = static_cast<uint16_t*>(const_cast<void*>(x));
  const uint32_t pr = static_cast<uint32_t>(per_row);
  const char* what = "activation checkpoint kernel";
  if (fast) {
    const unsigned grid = blocks_for(groups, kJobs);
    if (save) return launch(i8 ? k_act8_save<GWS_ACT8_INT8> : k_act8_save<GWS_ACT8_E4M3>, grid, kJobs, 0, 1, s, what, px, ldx, c, groups, pr);
    return launch(i8 ? k_act8_load<GWS_ACT8_INT8> : k_act8_load<GWS_ACT8_E4M3>, grid, kJobs, 0, 1, s, what, c, px, ldx, groups, pr);
  }
  if (save)
    return launch(i8 ? k_act8_save_any<GWS_ACT8_INT8> : k_act8_save_any<GWS_ACT8_E4M3>, blocks_for(groups * 4, kJobs), kJobs, 0, 1, s, what, px, ldx, c, groups * 4,
                  pr * 4u, cols);
  const uint32_t runs = (pr + 7) / 8;
  return launch(i8 ? k_act8_load_any<GWS_ACT8_INT8> : k_act8_load_any<GWS_ACT8_E4M3>, blocks_for(rows * runs, 8), kJobs, 0, 1, s, what, c, px, ldx, rows * runs, runs,
                cols);
}

// ---- tensor maps ---------------------------------------------------------------------------------------------------------
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static const Encode fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
    return reinterpret_cast<Encode>(p);
  }();
  return fn;
}

int encode_map(CUtensorMap& map, CUtensorMapDataType type, CUtensorMapSwizzle swizzle, const void* p, int64_t rows, int64_t cols, int64_t ld_bytes,
               uint32_t box_cols, uint32_t box_rows) {
  const Encode encode = encoder();
  if (encode == nullptr) return gws::report_text("cuTensorMapEncodeTiled is not available from this driver");
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld_bytes)};
  const cuuint32_t box[2] = {box_cols, box_rows}, steps[2] = {1u, 1u};
  const CUresult res = encode(&map, type, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (res != CUDA_SUCCESS) return gws::report_text(("cuTensorMapEncodeTiled failed with CUresult " + std::to_string(static_cast<int>(res))).c_str());
  return GWS_OK;
}
// A BF16 matrix whose copies are boxes of 64 columns by `box_rows` rows, 128-byte swizzle; outside it copies bring zeros.
int make_map(CUtensorMap& map, const void* p, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows) {
  return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_SWIZZLE_128B, p, rows, cols, ld * 2, 64u, box_rows);
}
// The codes of a checkpoint in boxes of `box_cols` = 128 or 64 columns, swizzled over that width.
int make_codes_map(CUtensorMap& map, const Act8View& c, int64_t rows, uint32_t box_cols, uint32_t box_rows) {
  return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, box_cols == 128u ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, c.codes, rows, c.ld, c.ld,
                    box_cols, box_rows);
}

// A matrix as the GEMM reads it: rows on 16-byte boundaries, in place or as a copy in the workspace.  Copies have rows of whole 128
// bytes: checkpoints are restored into them, and gradients written to them, a group at a time whatever the width, and the TMA copies
// fetch whole lines (3499 x 728 restored: 23 us of product with rows of 1472 bytes, 19 with 1536).
struct Mat {
  const void* p;
  int64_t rows, cols, ld;
};
bool in_place(int64_t rows, int64_t ld) { return rows <= 1 || ld % 8 == 0; }
int64_t packed_ld(int64_t cols) { return round_up(cols, 64); }
int64_t packed_bytes(int64_t rows, int64_t cols) { return round_up(rows * packed_ld(cols) * 2, 256); }

// What has to be made ready before a GEMM of a call: matrices to copy, a checkpoint to restore.
struct Ready {
  Prep prep;
  int n = 0;
  Ready() { std::memset(&prep, 0, sizeof prep); }
  // `to`: room of packed_bytes(a) in the workspace, used if the matrix cannot be read in place.
  void align(Mat& a, void* to) { align(a, to, !in_place(a.rows, a.ld)); }
  void align(Mat& a, void* to, bool moves) {
    if (!moves) {
      a.ld = round_up(a.rows <= 1 ? a.cols : a.ld, 8);
      return;
    }
    const int64_t ld = packed_ld(a.cols);
    prep.from[n] = static_cast<const uint16_t*>(a.p);
    prep.to[n] = static_cast<uint16_t*>(to);
    prep.ld_from[n] = a.ld;
    prep.cols[n] = a.cols;
    prep.per_row[n] = static_cast<uint32_t>(ld / 8);
    const int64_t end = (n > 0 ? prep.end[n - 1] : 0) + a.rows * (ld / 8);
    for (int i = n; i < 3; ++i) prep.end[i] = end;
    ++n;
    a.p = to;
    a.ld = ld;
  }
  // The checkpoint's matrix, in `to`.
  Mat restore(const Act8View& kept, int format, int64_t rows, int64_t cols, void* to) {
    prep.kept = kept;
    prep.format = format;
    prep.restored = static_cast<uint16_t*>(to);
    prep.ld_restored = packed_ld(cols);
    prep.groups = rows * (kept.ld / kGroup);
    return {to, rows, cols, prep.ld_restored};
  }
  int64_t blocks() {                     // GWS_ERR_LIMIT if there are too many for a launch
    const int64_t moves = (prep.end[2] + kJobs - 1) / kJobs, restores = (prep.groups + kJobs - 1) / kJobs;
    if (moves + restores >= 0x3FFFFFFFLL) return GWS_ERR_LIMIT;
    prep.move_blocks = static_cast<uint32_t>(moves);
    prep.restore_blocks = static_cast<uint32_t>(restores);
    return moves + restores;
  }
  int run(cudaStream_t s) {
    const int64_t grid = blocks();
    if (grid <= 0) return static_cast<int>(grid);
    return launch(k_prepare, static_cast<unsigned>(grid), kJobs, 0, 1, s, "operand preparation kernel", prep);
  }
};

std::atomic<int64_t> g_wait_limit{kTcWaitCycles};

// ---- choice of tile --------------------------------------------------------------------------------------------------------
// What make() returns for a key of sizes, options and SM count, which it depends on alone.  The last 64 or so are kept per thread: weighing the
// tiles of a call takes the host 0.5 to 1.5 us, as long as launching a kernel.
template <class Value, size_t N, class F>
const Value& remembered(const int64_t (&key)[N], F&& make) {
  struct Slot { int64_t key[N]; bool used; Value value; };
  static thread_local Slot slots[64];
  uint64_t hash = 0;
  for (const int64_t v : key) hash = (hash ^ static_cast<uint64_t>(v)) * 0x9E3779B97F4A7C15ull;
  Slot& slot = slots[hash >> 58];
  if (!slot.used || std::memcmp(slot.key, key, sizeof key) != 0) {
    slot.value = make();
    std::memcpy(slot.key, key, sizeof key);
    slot.used = true;
  }
  return slot.value;
}

// Stages along a contraction (TcShape::kHalves copies of 64 elements each).
int64_t stages_of(int64_t len, int bn) { const int64_t per = kTcHalf * (bn == 256 ? 1 : 2); return (len + per - 1) / per; }

struct Tile {
  int cg, bn;                              // blocks per tile, columns of accumulator
  uint32_t m_tiles, n_tiles, whole, cut, splits, kb_split;
  bool clustered;                          // the parts of a tile are the blocks of a cluster
  double cost;                             // estimated cycles
  uint32_t width;                          // kGatedFew: columns of h in a tile, else 0
};

// The tile, and the cut of the tiles that do not fill a wave, with the least estimated time, in SM cycles.  A tile takes a block its
// steps of 64 along the contraction, each the longest of the products (2 cycles a column), the operand bytes over the 67 (in pairs 77) a
// cycle that an SM drew from L2 with all SMs busy, and the issue of a stage, but no less than its epilogue (two chunks of 32 columns at a time).
// Joining costs a launch and the parts' way through memory (3400 bytes a cycle).  Measured on 2048 x 5632 (forward, us): 128 rows
// {2, 128} 14.7, {1, 128} 11.3, {2, 256} 16.0; 512 rows 21.0, 26.6, 25.1; 1024 rows 35.2, 43.4, 35.8.
Tile choose(int mode, int64_t rows, int64_t cols, int outs, int64_t len, int segments, int sms) {
  static const struct { int cg, bn; } kinds[] = {{2, 256}, {2, 128}, {1, 128}};
  Tile best{};
  double least = 0.0;
  for (const auto& kind : kinds) {
    const int64_t width = mode == kGated ? kind.bn / 2 : kind.bn;
    const int64_t mt = outs * ((rows + 128 * kind.cg - 1) / (128 * kind.cg)), nt = (cols + width - 1) / width, tiles = mt * nt;
    const int64_t slots = kind.cg == 2 ? sms / 2 : sms, kb = segments * stages_of(len, kind.bn);
    const double convert = mode == kDw8 ? 220.0 : 0.0;          // what a copy of codes adds to its step
    const double step = (kind.bn == 256 ? 1 : 2) * (convert + std::max(250.0, std::max(2.0 * kind.bn, (16384.0 + 128.0 * kind.bn / kind.cg) / (kind.cg == 2 ? 77.0 : 67.0))));
    const double epilogue = mode == kGated || mode == kLinear ? 10.0 * kind.bn + 400.0 : 5.0 * kind.bn + 400.0, start = kind.cg == 2 ? 4500.0 : 3300.0;
    // one row of tiles reads the weights once: no faster than from memory
    const double bytes = mt == 1 && (mode == kGated || mode == kLinear) ? (mode == kGated ? 4.0 : 2.0) * width * len / 3400.0 : 0.0, tile = std::max({kb * step, epilogue, std::min(tiles, slots) * bytes}) + 100.0;
    auto offer = [&](int64_t whole, int64_t splits, double cost, bool clustered) {
      if (best.cg != 0 && cost >= least) return;
      least = cost;
      const int64_t per = (kb + splits - 1) / splits;
      best = {kind.cg, kind.bn, static_cast<uint32_t>(mt), static_cast<uint32_t>(nt), static_cast<uint32_t>(whole), static_cast<uint32_t>(tiles - whole),
              static_cast<uint32_t>(splits), static_cast<uint32_t>(per), clustered, cost, 0};
    };
    offer(tiles, 1, start + epilogue + std::ceil(static_cast<double>(tiles) / slots) * tile, false);
    const int64_t whole = tiles / slots * slots, cut = tiles - whole;
    if (start + 5.0 * kind.bn + (mode == kGated || kind.cg == 2 ? 5900.0 + static_cast<double>(whole / slots) * tile : 2400.0) >= least) continue;
    for (int64_t splits = 2; cut > 0 && splits <= std::min<int64_t>(32, kb); ++splits) {
      const int64_t per = (kb + splits - 1) / splits;
      if ((kb + per - 1) / per != splits) continue;
      const double part = std::max(per * step, 5.0 * kind.bn + 400.0) + 100.0;
      offer(whole, splits, start + 5.0 * kind.bn + 400.0 + static_cast<double>(whole / slots) * tile +
                               std::max(std::ceil(static_cast<double>(cut * splits) / slots) * part, cut * bytes) +
                               5500.0 + 128.0 * kind.cg * kind.bn * cut * (8.0 * splits + 2.0) / 3400.0,
            false);
      // clusters of up to 4 blocks on 120 SMs, of up to 6 on 96: a cluster lives inside a group of some 18 SMs, and 16 clusters of 8 took two
      // waves (1 token, 5632 x 2048: 17.5 us, 10.9 with 6)
      if (kind.cg == 1 && mode != kGated && tiles * splits * 148 <= (splits <= 4 ? 120 : splits <= 6 ? 96 : 0) * sms)
        offer(0, splits, start + part + 5.0 * kind.bn + 2400.0 + 40.0 * std::min<int64_t>(rows, 128), true);
    }
  }
  return best;
}

int64_t part_bytes(const Tile& t) {
  if (t.clustered) return 0;
  return round_up(static_cast<int64_t>(t.cut) * (t.splits > 1 ? t.splits : 0) * 128 * t.cg * t.bn * 4, 256);
}

template <int CG, int BN, int MODE>
int launch_tc(const CUtensorMap (&maps)[4], const TcArgs& args, int sms, cudaStream_t s) {
  using S = TcShape<CG, BN, MODE>;
  static std::atomic<uint64_t> ready{0};        // devices on which this kernel has been given its shared memory
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (err == cudaSuccess && (dev > 63 || (ready.load(std::memory_order_relaxed) & bit) == 0)) {
    err = cudaFuncSetAttribute(k_tc<CG, BN, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::kSmemBytes));
    if (err == cudaSuccess) ready.fetch_or(bit, std::memory_order_relaxed);
  }
  if (err != cudaSuccess) return gws::report_cuda(err, "shared memory of the block GEMM");
  const uint32_t work = args.whole + args.cut * args.splits, slots = static_cast<uint32_t>(sms / CG);
  const int st = launch(k_tc<CG, BN, MODE>, args.clustered ? work : std::min(work, slots) * CG, S::kThreads, S::kSmemBytes,
                        args.clustered ? args.splits : CG, s, "block GEMM", maps[0], maps[1], maps[2], maps[3], args);
  if constexpr (MODE == kGatedFew || MODE == kLinearFew) return st;
  if (st != GWS_OK || args.cut == 0 || args.clustered) return st;
  constexpr uint32_t kWarps = (MODE == kGated ? BN / 64 : BN / 32) * (128 * CG / kJoinRows);       // per tile
  return launch(k_join<CG, BN, MODE == kLinearAlone ? kLinear : MODE>, args.cut * (kWarps / 8), 256, 0, 1, s, "join of a cut contraction", args);
}

template <int MODE>
int launch_mode(const Tile& t, const CUtensorMap (&maps)[4], const TcArgs& args, int sms, cudaStream_t s) {
  if (t.cg == 2 && t.bn == 256) return launch_tc<2, 256, MODE>(maps, args, sms, s);
  if (t.cg == 2) return launch_tc<2, 128, MODE>(maps, args, sms, s);
  return launch_tc<1, 128, MODE>(maps, args, sms, s);
}

TcArgs base_args(const Tile& t, int64_t rows, int64_t cols, int64_t len, int segments, int* status) {
  TcArgs a;
  std::memset(&a, 0, sizeof a);
  a.m_tiles = t.m_tiles;
  a.n_tiles = t.n_tiles;
  a.whole = t.whole;
  a.cut = t.cut;
  a.splits = t.splits;
  a.clustered = t.clustered;
  a.tiles_per_out = t.m_tiles;
  a.len = static_cast<uint32_t>(len);
  a.kb_first = static_cast<uint32_t>(stages_of(len, t.bn));
  a.kb = a.kb_first * segments;
  a.kb_split = t.kb_split;
  a.group = 8;
  a.parts = kTcHalf / 16;
  a.half_bytes = static_cast<uint32_t>(t.cg) * kTcABytes + static_cast<uint32_t>(t.bn) * kTcHalf * 2u;
  a.rows = rows;
  a.cols = cols;
  a.status = status;
  a.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
  return a;
}

// Elements that a store may take at once in BF16 rows `ld` apart (the second pointer may be null).
int32_t widest(int64_t ld, const void* p, const void* q) {
  for (int32_t v = 16; v > 1; v /= 2)
    if (ld % v == 0 && on(p, static_cast<size_t>(v) * 2) && on(q, static_cast<size_t>(v) * 2)) return v;
  return 1;
}

void set_out(TcArgs& a, void* out0, void* out1, int64_t ld) {
  a.out[0] = out0;
  a.out[1] = out1;
  a.ld_out = ld;
  a.wide = widest(ld, out0, out1);
}

// Copies fill rows outside a matrix with zeros at a fraction of the speed of rows inside it (one token, 128-row boxes: 31 us
// where 128 tokens take 14), so a matrix of few rows gets boxes of few rows.  What the rest of the shared memory holds reaches only
// accumulator rows that are not stored.
uint32_t a_box(int64_t rows) { return static_cast<uint32_t>(std::min<int64_t>(128, round_up(rows, 8))); }

// Tile of a weight gradient, and whether a checkpointed X is converted inside the GEMM, by its own warps, rather than restored into the
// workspace by a pass before it.  Inside, every tile converts its columns again, some 220 cycles a copy; the pass moves 3.1 bytes an
// element and is a launch more unless one is made anyway (`before`).  Measured, inside against before, on the device: 515 tokens, 768 x
// 768 7.1 against 6.9 us and 2.5 us less on the host; 16384, 512 x 2048 39.8 against 48.8; 2048, 2048 x 1024 15.4 against 13.1; 16384,
// 2048 x 5632 349 against 315.
struct DwChoice {
  Tile tile;
  bool inside;
};
DwChoice weigh_dw(int64_t tokens, int64_t rows, int64_t cols, int outs, bool kept, bool before, int sms) {
  const Tile plain = choose(kDw, rows, cols, outs, tokens, 1, sms);
  if (!kept) return {plain, false};
  const Tile inside = choose(kDw8, rows, cols, outs, tokens, 1, sms);
  const double pass = (before ? 0.0 : 4500.0) + static_cast<double>(tokens) * cols * 3.1 / 3400.0;
  return inside.cost < plain.cost + pass ? DwChoice{inside, true} : DwChoice{plain, false};
}
DwChoice choose_dw(int64_t tokens, int64_t rows, int64_t cols, int outs, bool kept, bool before, int sms) {
  return remembered<DwChoice>({tokens, rows, cols, outs, kept, before, sms}, [&] { return weigh_dw(tokens, rows, cols, outs, kept, before, sms); });
}

// dW (one or two outputs) = A^T X, A [m, rows] and X [m, cols] as they lie.
// X: a BF16 matrix, or a checkpoint of the same shape (x8, format) to be converted inside.
int run_dw(const Tile& t, const Mat& a0, const Mat* a1, const Mat& x, const Act8View* x8, int format, void* out0, void* out1, int64_t ld_out, void* part, int* status,
           int sms, cudaStream_t s) {
  const int outs = a1 != nullptr ? 2 : 1;
  TcArgs args = base_args(t, a0.cols, x.cols, a0.rows, 1, status);
  args.tiles_per_out = t.m_tiles / outs;
  set_out(args, out0, out1, ld_out);
  args.part = static_cast<float*>(part);
  // tokens fewer than a step: boxes and products of only the 16-token parts that hold any
  const uint32_t box = static_cast<uint32_t>(std::min<int64_t>(kTcHalf, round_up(a0.rows, 16)));
  args.parts = box / 16;
  args.box_tokens = static_cast<int32_t>(box);
  args.half_bytes = args.half_bytes / kTcHalf * box;
  CUtensorMap maps[4];
  int st = make_map(maps[0], a0.p, a0.rows, a0.cols, a0.ld, box);
  if (st == GWS_OK) st = a1 != nullptr ? make_map(maps[1], a1->p, a1->rows, a1->cols, a1->ld, box) : (maps[1] = maps[0], GWS_OK);
  if (st == GWS_OK) st = x8 != nullptr ? make_codes_map(maps[2], *x8, x.rows, static_cast<uint32_t>(t.bn / t.cg), box) : make_map(maps[2], x.p, x.rows, x.cols, x.ld, box);
  if (st != GWS_OK) return st;
  maps[3] = maps[2];
  if (x8 == nullptr) return launch_mode<kDw>(t, maps, args, sms, s);
  args.half_bytes = static_cast<uint32_t>(t.cg) * kTcABytes / kTcHalf * box;
  args.scales = x8->scales;
  args.scales_ld = x8->ld / kGroup;
  args.x_format = format;
  return launch_mode<kDw8>(t, maps, args, sms, s);
}

// ---- the gated block ---------------------------------------------------------------------------------------------------------
int check_gated(const gws_gated_desc* d) {
  if (d == nullptr) return GWS_ERR_NULL;
  const int st = check_dims(d->m, d->n, d->k);
  if (st != GWS_OK) return st;
  if ((d->m > 0 && d->k > 0 && d->ld_x < d->k) || (d->n > 0 && d->k > 0 && d->ld_w < d->k) || (d->m > 0 && d->n > 0 && d->ld_h < d->n)) return GWS_ERR_SHAPE;
  if (d->ld_x > kMaxDim || d->ld_w > kMaxDim || d->ld_h > kMaxDim) return GWS_ERR_LIMIT;
  if (d->activation < GWS_GATED_SILU || d->activation > GWS_GATED_RELU) return GWS_ERR_UNSUPPORTED;
  return GWS_OK;
}

int64_t saved_bytes(const gws_gated_desc* d) {
  return d->save_format == GWS_SAVE_NONE ? 0 : d->save_format == GWS_SAVE_BF16 ? d->m * d->n * 2 : act8_total(d->m, d->n);
}

struct BackLayout {
  int64_t x, w_gate, w_up, grad_gate, grad_up, part, total;
  Tile dx;
  DwChoice dw;
};
BackLayout weigh_backward(const gws_gated_desc* d, int sms) {
  BackLayout l{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t here = at; at += round_up(bytes, 256); return here; };
  l.dx = choose(kDx, d->m, d->k, 1, d->n, 2, sms);
  l.dw = choose_dw(d->m, d->n, d->k, 2, is_act8(d->x_format), true, sms);
  const bool direct_x = is_act8(d->x_format) ? l.dw.inside : in_place(d->m, d->ld_x);
  l.x = take(direct_x ? 0 : packed_bytes(d->m, d->k));
  const int64_t w = in_place(d->n, d->ld_w) ? 0 : packed_bytes(d->n, d->k);
  l.w_gate = take(w);
  l.w_up = take(w);
  l.grad_gate = take(packed_bytes(d->m, d->n));
  l.grad_up = take(packed_bytes(d->m, d->n));
  l.part = take(std::max(part_bytes(l.dx), part_bytes(l.dw.tile)));
  l.total = at;
  return l;
}
const BackLayout& back_layout(const gws_gated_desc* d, int sms) {
  return remembered<BackLayout>({d->m, d->n, d->k, d->ld_x, d->ld_w, d->x_format, sms}, [&] { return weigh_backward(d, sms); });
}
// Forward: tile, and which operands are copied into the workspace - those that no tensor map can read, and, where both operands have rows
// that start in the middle of a 32-byte sector, the smaller one if that pays.  With the contraction contiguous such rows cost a third more
// when both operands have them and 7 % when one does: 4096 tokens, 2048 x 1000 34.1 us, 27.2 with either side on whole lines, 25.3 with
// both; 4096, 5632 x 2040 157, 127, 121.  (Where the other axis is contiguous, in dx and dW, they cost 0 to 4 %.)
struct ForwardPlan {
  Tile tile;
  bool move_x, move_w;
  bool rows;                               // linear layer of a few tokens: k_linear_row
};
// kGatedFew, kLinearFew: bytes of a copy of 64 elements along the contraction (`operands`: weights that a tile reads `width` rows of), and the stages that fit; the products read
// 128 rows of A from where the last copy begins.
uint32_t few_half(int64_t rows, uint32_t width, uint32_t operands) { return a_box(rows) * kTcHalf * 2u + width * kTcHalf * 2u * operands; }
uint32_t few_stages(int64_t rows, uint32_t width, uint32_t operands) {
  const uint32_t half = few_half(rows, width, operands), ring = TcShape<1, 128, kGatedFew>::kRing;
  return std::min({8u, ring / (2u * half), (ring + half - kTcABytes) / (2u * half)});
}
// The width of tile with the least estimated time, for up to 128 tokens.  A stage of 128 steps costs 620 cycles however narrow the tile (eight
// products that read 128 rows of A), or its bytes at 67 a cycle; a wave of tiles costs no less than its weights at 3400 bytes a cycle from
// memory.  What narrow tiles win is an even share for every SM and more weights on their way (us, weights from memory, against the best of
// choose): one token, 2048 x 5632, 40 columns 12.0 (13.1), 48 11.9, 64 12.3, 32 in two waves 16.1; 128 tokens 13.2 (13.5); one token, 4096 x 11008,
// 40 columns 33 (42), 48 40.3, 64 42.5.  A long contraction into few columns is better cut: 5632 x 2048, 16 columns 18.1 (16.5).
// Checkpoints want whole groups of 32: 64 columns 13.1 (13.7), 32 16.9.
Tile choose_few(int64_t rows, int64_t cols, int64_t len, uint32_t unit, uint32_t operands, int sms) {
  const int64_t kb = stages_of(len, 128);
  const uint32_t slots = static_cast<uint32_t>(sms);
  Tile best{};
  for (uint32_t width = 128 / operands; width >= std::max(unit, 16u); width -= unit) {
    const uint32_t tiles = (static_cast<uint32_t>(cols) + width - 1) / width, rest = tiles % slots;
    const double stage = std::max(620.0, 2.0 * few_half(rows, width, operands) / 67.0), epilogue = 10.0 * operands * width + 400.0;
    auto wave = [&](uint32_t n) { return std::max({static_cast<double>(kb) * stage, epilogue, n * width * 2.0 * operands * len / 3400.0}) + 100.0; };
    const double cost = 3300.0 + epilogue + static_cast<double>(tiles / slots) * wave(slots) + (rest != 0 ? wave(rest) : 0.0);
    if (best.cg == 0 || cost < best.cost)
      best = {1, 128, 1, tiles, tiles, 0, 1, static_cast<uint32_t>(kb), false, cost, width};
  }
  return best;
}

ForwardPlan weigh_forward(const gws_gated_desc* d, int sms) {
  ForwardPlan f{choose(kGated, d->m, d->n, 1, d->k, 1, sms), !in_place(d->m, d->ld_x), !in_place(d->n, d->ld_w), false};
  if (d->m <= 128) {
    const Tile few = choose_few(d->m, d->n, d->k, 8, 2, sms);
    if (few.cost < f.tile.cost) f.tile = is_act8(d->save_format) ? choose_few(d->m, d->n, d->k, 32, 2, sms) : few;     // h does not depend on what is kept
  }
  if (!f.move_x && !f.move_w && d->m > 1 && d->n > 1 && d->ld_x % 16 != 0 && d->ld_w % 16 != 0) {
    const double smaller = static_cast<double>(d->k) * std::min(d->m, 2 * d->n);
    if (0.25 * f.tile.cost > 4500.0 + smaller * 4.0 / 3400.0) (d->m <= 2 * d->n ? f.move_x : f.move_w) = true;
  }
  return f;
}
const ForwardPlan& plan_forward(const gws_gated_desc* d, int sms) {
  return remembered<ForwardPlan>({d->m, d->n, d->k, d->ld_x, d->ld_w, d->save_format, sms}, [&] { return weigh_forward(d, sms); });
}
int64_t forward_copies(const gws_gated_desc* d, const ForwardPlan& f) {
  return (f.move_x ? packed_bytes(d->m, d->k) : 0) + (f.move_w ? 2 * packed_bytes(d->n, d->k) : 0);
}
int64_t forward_bytes(const gws_gated_desc* d, const ForwardPlan& f) { return forward_copies(d, f) + part_bytes(f.tile); }

template <int SAVE, int ACT>
int launch_pre(const PreArgs& p, Ready& ready, bool fast, cudaStream_t s) {
  const char* what = "gated backward, element-wise part";
  const int64_t first = ready.blocks(), items = fast ? p.groups : p.rows * ((p.per_row + 7) / 8), per = fast ? kJobs : 8;
  if (first < 0) return static_cast<int>(first);
  if ((items + per - 1) / per >= 0x3FFFFFFFLL) return GWS_ERR_LIMIT;
  const unsigned grid = static_cast<unsigned>(first) + blocks_for(items, per);
  return launch(fast ? k_gated_pre<SAVE, ACT> : k_gated_pre_any<SAVE, ACT>, grid, kJobs, 0, 1, s, what, p, ready.prep);
}
template <int SAVE>
int launch_pre_act(const PreArgs& p, Ready& ready, int act, bool fast, cudaStream_t s) {
  if (act == GWS_GATED_SILU) return launch_pre<SAVE, GWS_GATED_SILU>(p, ready, fast, s);
  if (act == GWS_GATED_GELU_TANH) return launch_pre<SAVE, GWS_GATED_GELU_TANH>(p, ready, fast, s);
  return launch_pre<SAVE, GWS_GATED_RELU>(p, ready, fast, s);
}

// ---- the linear layer with epilogue -----------------------------------------------------------------------------------------------
int check_linear(const gws_linear_desc* d) {
  if (d == nullptr) return GWS_ERR_NULL;
  const int st = check_dims(d->m, d->n, d->k);
  if (st != GWS_OK) return st;
  if (d->k == 0) return GWS_ERR_SHAPE;
  for (const int64_t ld : {d->ld_x, d->ld_w, d->ld_y, d->ld_residual}) {
    if (ld < 0) return GWS_ERR_SHAPE;
    if (ld > kMaxDim) return GWS_ERR_LIMIT;
  }
  if ((d->m > 0 && d->ld_x < d->k) || (d->n > 0 && d->ld_w < d->k) || (d->m > 0 && d->n > 0 && d->ld_y < d->n)) return GWS_ERR_SHAPE;
  if (d->activation < GWS_GATED_SILU || d->activation > GWS_ACT_NONE) return GWS_ERR_UNSUPPORTED;
  if (d->bias_type != GWS_TYPE_BF16 && d->bias_type != GWS_TYPE_F32) return GWS_ERR_UNSUPPORTED;
  return GWS_OK;
}
int64_t kept_bytes(int format, int64_t m, int64_t n) { return format == GWS_SAVE_NONE ? 0 : format == GWS_SAVE_BF16 ? m * n * 2 : act8_total(m, n); }
int64_t bias_bytes(const gws_linear_desc& d) { return d.n * (d.bias_type == GWS_TYPE_F32 ? 4 : 2); }

// Whether warps stream the rows of W (k_linear_row).  Each token costs them reads of x, where the narrow tiles of the tensor cores take eight for the price of one but some 4 us more
// around them.  On the device, us, rows against tiles: one token, 2048 x 5632 6.9, 9.7, 4096 x 11008 20.1, 19.2; two 8.5, 9.7 and 26.7, 19.2; four 15, 9.7; 768 x 768: one 1.8, 5.8;
// four 3.0, 5.9.
bool streams_rows(const gws_linear_desc& d) {
  const int64_t weights = d.n * d.k, most = d.m == 1 ? 1 << 25 : d.m == 2 ? 1 << 24 : d.m <= 4 ? 1 << 22 : 0;
  return weights <= most && d.k % 8 == 0 && in_place(d.m, d.ld_x) && in_place(d.n, d.ld_w);
}
// Columns of y to a block of eight warps: one or two to a warp, or two to four warps where there are few columns and long rows (one token, 5632 x 2048: 11.3 us with a warp to a row,
// 6.5 with four to two).  A checkpoint's 32 columns stay within a cluster of eight blocks.
unsigned row_columns(const gws_linear_desc& d) {
  const unsigned most = d.m == 1 ? 8u : 16u;
  const int64_t warps = d.m == 1 ? d.n : (d.n + 1) / 2;
  unsigned per = most;
  for (int64_t split = 1; per > 4u && warps * split < 32 * 148 && d.k >= 512 * split; split *= 2) per /= 2;
  return per;
}
// Forward: tile, and which operands are copied into the workspace; rows in the middle of a sector as in weigh_forward.
ForwardPlan weigh_linear(const gws_linear_desc* d, int sms) {
  ForwardPlan f{choose(kLinear, d->m, d->n, 1, d->k, 1, sms), !in_place(d->m, d->ld_x), !in_place(d->n, d->ld_w), false};
  f.rows = streams_rows(*d);
  if (f.rows) {
    f.tile.cut = 0;                              // no parts in the workspace
    return f;
  }
  if (d->m <= 128) {                             // widths are multiples of 16 (a product's columns), or of 32 (whole groups of a checkpoint)
    const Tile few = choose_few(d->m, d->n, d->k, 16, 1, sms);
    if (few.cost < f.tile.cost) f.tile = is_act8(d->save_format) ? choose_few(d->m, d->n, d->k, 32, 1, sms) : few;     // y does not depend on what is kept
  }
  if (!f.move_x && !f.move_w && d->m > 1 && d->n > 1 && d->ld_x % 16 != 0 && d->ld_w % 16 != 0) {
    const double smaller = static_cast<double>(d->k) * std::min(d->m, d->n);
    if (0.25 * f.tile.cost > 4500.0 + smaller * 4.0 / 3400.0) (d->m <= d->n ? f.move_x : f.move_w) = true;
  }
  return f;
}
const ForwardPlan& plan_linear(const gws_linear_desc* d, int sms) {
  return remembered<ForwardPlan>({d->m, d->n, d->k, d->ld_x, d->ld_w, is_act8(d->save_format), sms}, [&] { return weigh_linear(d, sms); });
}
int64_t linear_copies(const gws_linear_desc* d, const ForwardPlan& f) {
  return (f.move_x ? packed_bytes(d->m, d->k) : 0) + (f.move_w ? packed_bytes(d->n, d->k) : 0);
}

// Shares of a strip's rows: of at least 16 rows, and as many blocks as the SMs hold at once (six each).
uint32_t pre_shares(int64_t rows, int64_t cols, int sms) {
  const int64_t strips = (cols + 63) / 64, fill = std::max<int64_t>(1, 6 * sms / strips), most = (rows + 15) / 16;
  if (most <= 8) return rows > 64 ? 8u : rows > 32 ? 4u : rows > 16 ? 2u : 1u;
  return static_cast<uint32_t>(std::max<int64_t>(8, std::min(fill, (rows + 63) / 64)));
}
int64_t pre_part_bytes(int64_t rows, int64_t cols, int sms) {
  const uint32_t shares = pre_shares(rows, cols, sms);
  return shares <= 8u ? 0 : round_up(static_cast<int64_t>(shares) * cols * 4, 256);
}

// Backward: places in the workspace, whatever the call asks for.  dz is grad_y itself without an activation (aligned if its rows are not).
struct LinearBack {
  int64_t x, w, dz, sums, part, total;
  Tile dx;
  DwChoice dw;
};
LinearBack weigh_linear_back(const gws_linear_desc* d, int sms) {
  LinearBack l{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t here = at; at += round_up(bytes, 256); return here; };
  const bool makes = d->activation != GWS_ACT_NONE, moves = !makes && !in_place(d->m, d->ld_y);
  l.dx = choose(kDx, d->m, d->k, 1, d->n, 1, sms);
  l.dw = choose_dw(d->m, d->n, d->k, 1, is_act8(d->x_format), makes || moves, sms);
  const bool direct_x = is_act8(d->x_format) ? l.dw.inside : in_place(d->m, d->ld_x);
  l.x = take(direct_x ? 0 : packed_bytes(d->m, d->k));
  l.w = take(in_place(d->n, d->ld_w) ? 0 : packed_bytes(d->n, d->k));
  l.dz = take(makes || moves ? packed_bytes(d->m, d->n) : 0);
  l.sums = take(pre_part_bytes(d->m, d->n, sms));
  l.part = take(std::max(part_bytes(l.dx), part_bytes(l.dw.tile)));
  l.total = at;
  return l;
}
const LinearBack& linear_back(const gws_linear_desc* d, int sms) {
  return remembered<LinearBack>({d->m, d->n, d->k, d->ld_x, d->ld_w, d->ld_y, d->activation != GWS_ACT_NONE, d->x_format, sms}, [&] { return weigh_linear_back(d, sms); });
}

template <int SAVE, bool WIDE>
auto pre_kernel(int act) {
  return act == GWS_GATED_SILU        ? k_linear_pre<SAVE, GWS_GATED_SILU, WIDE>
         : act == GWS_GATED_GELU_TANH ? k_linear_pre<SAVE, GWS_GATED_GELU_TANH, WIDE>
         : act == GWS_GATED_RELU      ? k_linear_pre<SAVE, GWS_GATED_RELU, WIDE>
                                      : k_linear_pre<SAVE, GWS_ACT_NONE, WIDE>;
}
// `part`: room of pre_part_bytes.
int launch_linear_pre(LinearPre p, Ready& ready, int act, int save, bool wide, void* part, int sms, cudaStream_t s) {
  const int64_t moved = ready.blocks(), strips = (p.cols + 63) / 64;
  if (moved < 0) return static_cast<int>(moved);
  p.shares = pre_shares(p.rows, p.cols, sms);
  const bool clustered = p.db != nullptr && p.shares <= 8u;
  if (p.db != nullptr && !clustered) p.part = static_cast<float*>(part);
  p.first = static_cast<uint32_t>(clustered ? round_up(moved, p.shares) : moved);
  if (strips * p.shares >= 0x3FFFFFFFLL) return GWS_ERR_LIMIT;
  const unsigned grid = p.first + static_cast<unsigned>(strips) * p.shares;
  auto kernel = save == GWS_ACT8_INT8   ? (wide ? pre_kernel<GWS_ACT8_INT8, true>(act) : pre_kernel<GWS_ACT8_INT8, false>(act))
                : save == GWS_ACT8_E4M3 ? (wide ? pre_kernel<GWS_ACT8_E4M3, true>(act) : pre_kernel<GWS_ACT8_E4M3, false>(act))
                : save == GWS_SAVE_BF16 ? (wide ? pre_kernel<GWS_SAVE_BF16, true>(act) : pre_kernel<GWS_SAVE_BF16, false>(act))
                                        : (wide ? k_linear_pre<GWS_SAVE_NONE, GWS_ACT_NONE, true> : k_linear_pre<GWS_SAVE_NONE, GWS_ACT_NONE, false>);
  const int st = launch(kernel, grid, kPreThreads, 0, clustered ? p.shares : 1, s, "linear backward, element-wise part", p, ready.prep);
  if (st != GWS_OK || p.part == nullptr) return st;
  return launch(k_column_sums, blocks_for(p.cols, 32), 32 * kSumWarps, 0, 1, s, "join of column sums", static_cast<const float*>(p.part), p.shares, p.cols, 1u, p.db, static_cast<void*>(nullptr), p.db_f32);
}

void describe(const Tile& t, int sms, gws_product_plan* p) {
  std::memset(p, 0, sizeof *p);
  p->blocks = t.cg;
  p->columns = t.width != 0 ? static_cast<int32_t>(2 * t.width) : t.bn;
  p->narrow = static_cast<int32_t>(t.width);
  p->whole = static_cast<int32_t>(t.whole);
  p->cut = static_cast<int32_t>(t.cut);
  p->splits = static_cast<int32_t>(t.splits);
  p->clustered = t.clustered;
  const uint32_t work = t.whole + t.cut * t.splits, slots = static_cast<uint32_t>(sms / t.cg);
  p->waves = t.clustered ? 1 : static_cast<int32_t>((work + slots - 1) / slots);
}

}  // namespace

extern "C" {

int64_t gws_set_wait_limit(int64_t cycles) { return g_wait_limit.exchange(cycles > 0 ? cycles : kTcWaitCycles, std::memory_order_relaxed); }

int gws_act8_layout(int64_t rows, int64_t cols, size_t* codes_bytes, size_t* scales_offset, size_t* total_bytes) {
  const int st = check_dims(rows, cols, 0);
  if (st != GWS_OK) return st;
  if (codes_bytes != nullptr) *codes_bytes = static_cast<size_t>(act8_codes(rows, cols));
  if (scales_offset != nullptr) *scales_offset = static_cast<size_t>(round_up(act8_codes(rows, cols), 256));
  if (total_bytes != nullptr) *total_bytes = static_cast<size_t>(act8_total(rows, cols));
  return GWS_OK;
}

static int act8_move(bool save, int64_t rows, int64_t cols, int64_t ld, int format, const void* x, const void* act8, void* stream) {
  const int st = check_dims(rows, cols, 0);
  if (st != GWS_OK) return st;
  if (!is_act8(format)) return GWS_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return GWS_OK;
  if (ld < cols) return GWS_ERR_SHAPE;
  if (ld > kMaxDim) return GWS_ERR_LIMIT;
  if (x == nullptr || act8 == nullptr) return GWS_ERR_NULL;
  if (!on(x, 2) || !on(act8, 32)) return GWS_ERR_ALIGN;
  if (overlap(rows_of(x, rows, cols, ld), {act8, act8_total(rows, cols)})) return GWS_ERR_ALIAS;
  return launch_act8(save, format, x, rows == 1 ? act8_ld(cols) : ld, act8_view(act8, rows, cols), rows, cols, static_cast<cudaStream_t>(stream));
}

int gws_act8_save(int64_t rows, int64_t cols, int64_t ld, int format, const void* x, void* act8, void* stream) {
  return act8_move(true, rows, cols, ld, format, x, act8, stream);
}

int gws_act8_load(int64_t rows, int64_t cols, int64_t ld, int format, const void* act8, void* x, void* stream) {
  return act8_move(false, rows, cols, ld, format, x, act8, stream);
}

int64_t gws_wgrad_act8_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ld_y) {
  const int st = check_dims(m, n, k);
  if (st != GWS_OK) return st;
  if (m == 0 || n == 0 || k == 0) return 0;
  const bool moved = !in_place(m, ld_y);
  const DwChoice dw = choose_dw(m, n, k, 1, true, moved, sm_count());
  return (moved ? packed_bytes(m, n) : 0) + (dw.inside ? 0 : packed_bytes(m, k)) + part_bytes(dw.tile);
}

int gws_wgrad_act8(int64_t m, int64_t n, int64_t k, int format, const void* grad_y, int64_t ld_y, const void* x8, void* grad_w, int64_t ld_w,
                   void* workspace, size_t workspace_bytes, int* status, void* stream) {
  int st = check_dims(m, n, k);
  if (st != GWS_OK) return st;
  if (!is_act8(format)) return GWS_ERR_UNSUPPORTED;
  if (n == 0 || k == 0) return GWS_OK;
  if (ld_w < k || (m > 0 && ld_y < n)) return GWS_ERR_SHAPE;
  if (ld_w > kMaxDim || ld_y > kMaxDim) return GWS_ERR_LIMIT;
  if (grad_w == nullptr || (m > 0 && (grad_y == nullptr || x8 == nullptr))) return GWS_ERR_NULL;
  if (!on(grad_w, 2) || !on(status, 4)) return GWS_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (m == 0) return zero(grad_w, n, k, ld_w, s);
  if (!on(grad_y, in_place(m, ld_y) ? 16 : 2) || !on(x8, 32)) return GWS_ERR_ALIGN;
  const int64_t need = gws_wgrad_act8_workspace_bytes(m, n, k, ld_y);
  if (clash({rows_of(grad_w, n, k, ld_w), {workspace, need}}, {rows_of(grad_y, m, n, ld_y), {x8, act8_total(m, k)}})) return GWS_ERR_ALIAS;
  if (!workspace_ok(workspace, workspace_bytes, need)) return GWS_ERR_WORKSPACE;
  char* ws = static_cast<char*>(workspace);
  const Act8View kept = act8_view(x8, m, k);
  Ready ready;
  Mat y{grad_y, m, n, ld_y}, x{nullptr, m, k, 0};
  ready.align(y, ws);
  const bool moved = !in_place(m, ld_y);
  if (moved) ws += packed_bytes(m, n);
  const int sms = sm_count();
  const DwChoice dw = choose_dw(m, n, k, 1, true, moved, sms);
  if (!dw.inside) {
    x = ready.restore(kept, format, m, k, ws);
    ws += packed_bytes(m, k);
  }
  if ((st = ready.run(s)) != GWS_OK) return st;
  return run_dw(dw.tile, y, nullptr, x, dw.inside ? &kept : nullptr, format, grad_w, nullptr, ld_w, ws, status, sms, s);
}

int64_t gws_gated_workspace_bytes(const gws_gated_desc* desc, int backward) {
  const int st = check_gated(desc);
  if (st != GWS_OK) return st;
  if (desc->m == 0 || desc->n == 0 || desc->k == 0) return 0;
  return backward != 0 ? back_layout(desc, sm_count()).total : forward_bytes(desc, plan_forward(desc, sm_count()));
}

int gws_gated_plan(const gws_gated_desc* desc, int product, gws_product_plan* plan) {
  if (plan == nullptr) return GWS_ERR_NULL;
  const int st = check_gated(desc);
  if (st != GWS_OK) return st;
  if (product < 0 || product > 2) return GWS_ERR_UNSUPPORTED;
  std::memset(plan, 0, sizeof *plan);
  if (desc->m == 0 || desc->n == 0 || desc->k == 0) return GWS_OK;
  const int sms = sm_count();
  if (product == 0) {
    const ForwardPlan& f = plan_forward(desc, sms);
    describe(f.tile, sms, plan);
    plan->moves_x = f.move_x;
    plan->moves_w = f.move_w;
  } else {
    const BackLayout& l = back_layout(desc, sms);
    describe(product == 1 ? l.dx : l.dw.tile, sms, plan);
    plan->inside = product == 2 && l.dw.inside;
  }
  return GWS_OK;
}

int gws_wgrad_act8_plan(int64_t m, int64_t n, int64_t k, int64_t ld_y, gws_product_plan* plan) {
  if (plan == nullptr) return GWS_ERR_NULL;
  const int st = check_dims(m, n, k);
  if (st != GWS_OK) return st;
  std::memset(plan, 0, sizeof *plan);
  if (m == 0 || n == 0 || k == 0) return GWS_OK;
  const int sms = sm_count();
  const DwChoice dw = choose_dw(m, n, k, 1, true, !in_place(m, ld_y), sms);
  describe(dw.tile, sms, plan);
  plan->inside = dw.inside;
  return GWS_OK;
}

int gws_gated_fwd(const gws_gated_desc* desc, const void* x, const void* w_gate, const void* w_up, void* h, void* save_gate, void* save_up,
                  void* workspace, size_t workspace_bytes, int* status, void* stream) {
  int st = check_gated(desc);
  if (st != GWS_OK) return st;
  const gws_gated_desc& d = *desc;
  const bool saves = d.save_format != GWS_SAVE_NONE, bytes8 = is_act8(d.save_format);
  if (saves && !bytes8 && d.save_format != GWS_SAVE_BF16) return GWS_ERR_UNSUPPORTED;
  if (d.m == 0 || d.n == 0) return GWS_OK;
  if (h == nullptr || (saves && (save_gate == nullptr || save_up == nullptr))) return GWS_ERR_NULL;
  if (!on(h, 2) || !on(status, 4) || (saves && (!on(save_gate, bytes8 ? 32 : 2) || !on(save_up, bytes8 ? 32 : 2)))) return GWS_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d.k == 0) {                              // both projections are zero, and so is act(0)
    st = zero(h, d.m, d.n, d.ld_h, s);
    for (void* p : {save_gate, save_up})
      if (st == GWS_OK && saves) {
        const cudaError_t err = cudaMemsetAsync(p, 0, static_cast<size_t>(saved_bytes(desc)), s);
        if (err != cudaSuccess) st = gws::report_cuda(err, "clearing a saved projection");
      }
    return st;
  }
  if (x == nullptr || w_gate == nullptr || w_up == nullptr) return GWS_ERR_NULL;
  const int sms = sm_count();
  const ForwardPlan& f = plan_forward(desc, sms);
  if (!on(x, in_place(d.m, d.ld_x) ? 16 : 2) || !on(w_gate, in_place(d.n, d.ld_w) ? 16 : 2) || !on(w_up, in_place(d.n, d.ld_w) ? 16 : 2)) return GWS_ERR_ALIGN;
  const int64_t need = forward_bytes(desc, f), kept = saved_bytes(desc);
  if (clash({rows_of(h, d.m, d.n, d.ld_h), {save_gate, kept}, {save_up, kept}, {workspace, need}},
            {rows_of(x, d.m, d.k, d.ld_x), rows_of(w_gate, d.n, d.k, d.ld_w), rows_of(w_up, d.n, d.k, d.ld_w)}))
    return GWS_ERR_ALIAS;
  if (!workspace_ok(workspace, workspace_bytes, need)) return GWS_ERR_WORKSPACE;
  Mat mx{x, d.m, d.k, d.ld_x}, mg{w_gate, d.n, d.k, d.ld_w}, mu{w_up, d.n, d.k, d.ld_w};
  Ready ready;
  char* ws = static_cast<char*>(workspace);
  ready.align(mx, ws, f.move_x);
  if (f.move_x) ws += packed_bytes(d.m, d.k);
  ready.align(mg, ws, f.move_w);
  if (f.move_w) ws += packed_bytes(d.n, d.k);
  ready.align(mu, ws, f.move_w);
  if ((st = ready.run(s)) != GWS_OK) return st;

  const Tile& t = f.tile;
  const uint32_t width = t.width != 0 ? t.width : static_cast<uint32_t>(t.bn / 2);
  TcArgs args = base_args(t, d.m, d.n, d.k, 1, status);
  set_out(args, h, nullptr, d.ld_h);
  args.half_bytes -= static_cast<uint32_t>(t.cg) * (128u - a_box(d.m)) * kTcHalf * 2u;
  args.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + forward_copies(desc, f));
  args.activation = d.activation;
  args.save = d.save_format;
  if (bytes8) {
    args.save8[0] = act8_view(save_gate, d.m, d.n);
    args.save8[1] = act8_view(save_up, d.m, d.n);
  } else if (saves) {
    args.save16[0] = static_cast<uint16_t*>(save_gate);
    args.save16[1] = static_cast<uint16_t*>(save_up);
    args.save_wide = widest(d.n, save_gate, save_up);
  }
  if (t.width != 0) {
    args.width = width;
    args.a_bytes = a_box(d.m) * kTcHalf * 2u;
    args.stages = few_stages(d.m, width, 2);
    args.half_bytes = few_half(d.m, width, 2);
    if (width % 16 != 0) args.wide = std::min(args.wide, 8), args.save_wide = std::min(args.save_wide, 8);
  }
  CUtensorMap maps[4];
  if ((st = make_map(maps[0], mx.p, d.m, d.k, mx.ld, a_box(d.m))) != GWS_OK) return st;
  maps[1] = maps[0];
  if ((st = make_map(maps[2], mg.p, d.n, d.k, mg.ld, width)) != GWS_OK) return st;
  if ((st = make_map(maps[3], mu.p, d.n, d.k, mu.ld, width)) != GWS_OK) return st;
  return t.width != 0 ? launch_tc<1, 128, kGatedFew>(maps, args, sms, s) : launch_mode<kGated>(t, maps, args, sms, s);
}

int gws_gated_bwd(const gws_gated_desc* desc, const void* grad_h, const void* x, const void* w_gate, const void* w_up, const void* save_gate,
                  const void* save_up, void* grad_x, void* grad_w_gate, void* grad_w_up, void* h_out, void* workspace, size_t workspace_bytes,
                  int* status, void* stream) {
  int st = check_gated(desc);
  if (st != GWS_OK) return st;
  const gws_gated_desc& d = *desc;
  const bool saved8 = is_act8(d.save_format), x8 = is_act8(d.x_format);
  if ((!saved8 && d.save_format != GWS_SAVE_BF16) || (!x8 && d.x_format != GWS_SAVE_BF16)) return GWS_ERR_UNSUPPORTED;
  if ((grad_w_gate == nullptr) != (grad_w_up == nullptr)) return GWS_ERR_NULL;
  if (!on(grad_x, 2) || !on(grad_w_gate, 2) || !on(grad_w_up, 2) || !on(h_out, 2) || !on(status, 4)) return GWS_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d.m == 0 || d.n == 0 || d.k == 0) {      // empty sums; with k = 0 the projections are zero, and so is h
    if ((st = zero(grad_x, d.m, d.k, d.k, s)) != GWS_OK || (st = zero(grad_w_gate, d.n, d.k, d.k, s)) != GWS_OK ||
        (st = zero(grad_w_up, d.n, d.k, d.k, s)) != GWS_OK)
      return st;
    return zero(h_out, d.m, d.n, d.n, s);
  }
  const bool wants_dw = grad_w_gate != nullptr, wants_dx = grad_x != nullptr;
  if (grad_h == nullptr || save_gate == nullptr || save_up == nullptr || (wants_dw && x == nullptr) || (wants_dx && (w_gate == nullptr || w_up == nullptr)))
    return GWS_ERR_NULL;
  const bool moves_x = !x8 && !in_place(d.m, d.ld_x), moves_w = !in_place(d.n, d.ld_w);
  if (!on(grad_h, 2) || !on(save_gate, saved8 ? 32 : 2) || !on(save_up, saved8 ? 32 : 2) || (wants_dw && !on(x, x8 ? 32 : moves_x ? 2 : 16)) ||
      (wants_dx && (!on(w_gate, moves_w ? 2 : 16) || !on(w_up, moves_w ? 2 : 16))))
    return GWS_ERR_ALIGN;
  const int sms = sm_count();
  const BackLayout& l = back_layout(desc, sms);
  const int64_t kept = saved_bytes(desc);
  const Span in_x = x8 ? Span{x, act8_total(d.m, d.k)} : rows_of(x, d.m, d.k, d.ld_x);
  if (clash({rows_of(grad_x, d.m, d.k, d.k), rows_of(grad_w_gate, d.n, d.k, d.k), rows_of(grad_w_up, d.n, d.k, d.k), rows_of(h_out, d.m, d.n, d.n),
             {workspace, l.total}},
            {rows_of(grad_h, d.m, d.n, d.ld_h), in_x, rows_of(w_gate, d.n, d.k, d.ld_w), rows_of(w_up, d.n, d.k, d.ld_w), {save_gate, kept}, {save_up, kept}}))
    return GWS_ERR_ALIAS;
  if (!workspace_ok(workspace, workspace_bytes, l.total)) return GWS_ERR_WORKSPACE;
  char* ws = static_cast<char*>(workspace);

  PreArgs p;
  std::memset(&p, 0, sizeof p);
  p.grad_h = static_cast<const uint16_t*>(grad_h);
  p.ld_grad_h = d.m == 1 ? d.n : d.ld_h;
  if (saved8) {
    p.save8[0] = act8_view(save_gate, d.m, d.n);
    p.save8[1] = act8_view(save_up, d.m, d.n);
  } else {
    p.save16[0] = static_cast<const uint16_t*>(save_gate);
    p.save16[1] = static_cast<const uint16_t*>(save_up);
  }
  p.grad_gate = reinterpret_cast<uint16_t*>(ws + l.grad_gate);
  p.grad_up = reinterpret_cast<uint16_t*>(ws + l.grad_up);
  p.ld = packed_ld(d.n);
  p.rows = d.m;
  p.h = static_cast<uint16_t*>(h_out);
  p.cols = d.n;
  p.per_row = static_cast<uint32_t>(act8_ld(d.n) / kGroup);
  p.groups = d.m * p.per_row;
  // A thread with a group of its own needs some 75,000 groups to fill the GPU; below that its 32 elements in a row are all latency, and
  // the form with eight to a lane takes over (33 x 2048: 5.4 -> 3.5 us).
  const bool fast = p.groups >= 148 * 512 && whole_groups(grad_h, d.n, p.ld_grad_h) && on(h_out, 32) && (saved8 || (on(save_gate, 32) && on(save_up, 32)));
  Ready ready;
  Mat mg{w_gate, d.n, d.k, d.ld_w}, mu{w_up, d.n, d.k, d.ld_w}, mx{x, d.m, d.k, d.ld_x};
  const Act8View kept_x = act8_view(x, d.m, d.k);
  if (wants_dx) {
    ready.align(mg, ws + l.w_gate);
    ready.align(mu, ws + l.w_up);
  }
  if (wants_dw && x8 && !l.dw.inside) mx = ready.restore(kept_x, d.x_format, d.m, d.k, ws + l.x);
  if (wants_dw && !x8) ready.align(mx, ws + l.x);
  st = d.save_format == GWS_ACT8_INT8   ? launch_pre_act<GWS_ACT8_INT8>(p, ready, d.activation, fast, s)
       : d.save_format == GWS_ACT8_E4M3 ? launch_pre_act<GWS_ACT8_E4M3>(p, ready, d.activation, fast, s)
                                        : launch_pre_act<GWS_SAVE_BF16>(p, ready, d.activation, fast, s);
  if (st != GWS_OK) return st;
  const Mat dg{p.grad_gate, d.m, d.n, p.ld}, du{p.grad_up, d.m, d.n, p.ld};

  if (wants_dx) {
    const Tile& t = l.dx;
    TcArgs args = base_args(t, d.m, d.k, d.n, 2, status);
    args.half_bytes -= static_cast<uint32_t>(t.cg) * (128u - a_box(d.m)) * kTcHalf * 2u;
    set_out(args, grad_x, nullptr, d.k);
    args.part = reinterpret_cast<float*>(ws + l.part);
    CUtensorMap maps[4];
    if ((st = make_map(maps[0], dg.p, d.m, d.n, dg.ld, a_box(d.m))) != GWS_OK || (st = make_map(maps[1], du.p, d.m, d.n, du.ld, a_box(d.m))) != GWS_OK ||
        (st = make_map(maps[2], mg.p, d.n, d.k, mg.ld, kTcHalf)) != GWS_OK || (st = make_map(maps[3], mu.p, d.n, d.k, mu.ld, kTcHalf)) != GWS_OK)
      return st;
    if ((st = launch_mode<kDx>(t, maps, args, sms, s)) != GWS_OK) return st;
  }
  if (wants_dw) return run_dw(l.dw.tile, dg, &du, mx, l.dw.inside ? &kept_x : nullptr, d.x_format, grad_w_gate, grad_w_up, d.k, ws + l.part, status, sms, s);
  return GWS_OK;
}

int64_t gws_linear_workspace_bytes(const gws_linear_desc* desc, int backward) {
  const int st = check_linear(desc);
  if (st != GWS_OK) return st;
  if (desc->m == 0 || desc->n == 0) return 0;
  const int sms = sm_count();
  if (backward != 0) return linear_back(desc, sms).total;
  const ForwardPlan& f = plan_linear(desc, sms);
  return linear_copies(desc, f) + part_bytes(f.tile);
}

int gws_linear_plan(const gws_linear_desc* desc, int product, gws_product_plan* plan) {
  if (plan == nullptr) return GWS_ERR_NULL;
  const int st = check_linear(desc);
  if (st != GWS_OK) return st;
  if (product < 0 || product > 2) return GWS_ERR_UNSUPPORTED;
  std::memset(plan, 0, sizeof *plan);
  if (desc->m == 0 || desc->n == 0) return GWS_OK;
  const int sms = sm_count();
  if (product == 0) {
    const ForwardPlan& f = plan_linear(desc, sms);
    describe(f.tile, sms, plan);
    if (f.tile.width != 0) plan->columns = plan->narrow;
    if (f.rows) {
      std::memset(plan, 0, sizeof *plan);
      plan->columns = static_cast<int32_t>(row_columns(*desc));
      plan->waves = 1;
    }
    plan->moves_x = f.move_x;
    plan->moves_w = f.move_w;
  } else {
    const LinearBack& l = linear_back(desc, sms);
    describe(product == 1 ? l.dx : l.dw.tile, sms, plan);
    plan->inside = product == 2 && l.dw.inside;
  }
  return GWS_OK;
}

int gws_linear_fwd(const gws_linear_desc* desc, const void* x, const void* w, const void* bias, const void* residual, void* y, void* save, void* workspace,
                   size_t workspace_bytes, int* status, void* stream) {
  int st = check_linear(desc);
  if (st != GWS_OK) return st;
  const gws_linear_desc& d = *desc;
  const bool saves = d.save_format != GWS_SAVE_NONE, bytes8 = is_act8(d.save_format);
  if (saves && !bytes8 && d.save_format != GWS_SAVE_BF16) return GWS_ERR_UNSUPPORTED;
  if (d.m == 0 || d.n == 0) return GWS_OK;
  if (residual != nullptr && d.ld_residual < d.n) return GWS_ERR_SHAPE;
  if (x == nullptr || w == nullptr || y == nullptr || (saves && save == nullptr)) return GWS_ERR_NULL;
  const size_t bias_each = d.bias_type == GWS_TYPE_F32 ? 4 : 2;
  if (!on(y, 2) || !on(residual, 2) || !on(bias, bias_each) || !on(status, 4) || (saves && !on(save, bytes8 ? 32 : 2)) || !on(x, in_place(d.m, d.ld_x) ? 16 : 2) ||
      !on(w, in_place(d.n, d.ld_w) ? 16 : 2))
    return GWS_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int sms = sm_count();
  const ForwardPlan& f = plan_linear(desc, sms);
  const int64_t copies = linear_copies(desc, f), need = copies + part_bytes(f.tile);
  if (clash({rows_of(y, d.m, d.n, d.ld_y), {save, kept_bytes(d.save_format, d.m, d.n)}, {workspace, need}},
            {rows_of(x, d.m, d.k, d.ld_x), rows_of(w, d.n, d.k, d.ld_w), {bias, bias != nullptr ? bias_bytes(d) : 0}, rows_of(residual, d.m, d.n, d.ld_residual)}))
    return GWS_ERR_ALIAS;
  if (!workspace_ok(workspace, workspace_bytes, need)) return GWS_ERR_WORKSPACE;
  Mat mx{x, d.m, d.k, d.ld_x}, mw{w, d.n, d.k, d.ld_w};
  Ready ready;
  char* ws = static_cast<char*>(workspace);
  ready.align(mx, ws, f.move_x);
  if (f.move_x) ws += packed_bytes(d.m, d.k);
  ready.align(mw, ws, f.move_w);
  if ((st = ready.run(s)) != GWS_OK) return st;

  if (f.rows) {
    LinearRow p;
    std::memset(&p, 0, sizeof p);
    p.x = static_cast<const uint16_t*>(x);
    p.w = static_cast<const uint16_t*>(w);
    p.residual = static_cast<const uint16_t*>(residual);
    p.bias = bias;
    p.y = static_cast<uint16_t*>(y);
    p.save16 = static_cast<uint16_t*>(save);
    if (bytes8) p.save8 = act8_view(save, d.m, d.n);
    p.ld_x = round_up(d.ld_x, 8);                // of one token any
    p.ld_w = d.ld_w;
    p.ld_y = d.ld_y;
    p.ld_residual = d.ld_residual;
    p.cols = d.n;
    p.octets = static_cast<uint32_t>(d.k / 8);
    p.tokens = static_cast<int32_t>(d.m);
    p.activation = d.activation;
    p.save = d.save_format;
    p.bias_f32 = d.bias_type == GWS_TYPE_F32;
    const unsigned per = row_columns(d), cluster = bytes8 ? 32u / per : 1u;
    const unsigned grid = static_cast<unsigned>(round_up((d.n + per - 1) / per, cluster));
    auto kernel = d.m == 1   ? (per == 8u ? k_linear_row<1, 1, 1> : k_linear_row<1, 2, 4>)
                  : d.m == 2 ? (per == 16u ? k_linear_row<2, 2, 1> : per == 8u ? k_linear_row<2, 2, 2> : k_linear_row<2, 2, 4>)
                             : (per == 16u ? k_linear_row<4, 2, 1> : per == 8u ? k_linear_row<4, 2, 2> : k_linear_row<4, 2, 4>);
    return launch(kernel, grid, 256, 0, cluster, s, "linear layer of a few tokens", p);
  }
  const Tile& t = f.tile;
  TcArgs args = base_args(t, d.m, d.n, d.k, 1, status);
  set_out(args, y, nullptr, d.ld_y);
  args.half_bytes -= static_cast<uint32_t>(t.cg) * (128u - a_box(d.m)) * kTcHalf * 2u;
  args.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + copies);
  args.activation = d.activation;
  args.bias = bias;
  args.bias_f32 = d.bias_type == GWS_TYPE_F32;
  args.residual = static_cast<const uint16_t*>(residual);
  args.ld_residual = d.ld_residual;
  args.residual_wide = widest(d.m > 1 ? d.ld_residual : round_up(d.ld_residual, 16), residual, nullptr);
  args.save = d.save_format;
  if (bytes8) {
    args.save8[0] = act8_view(save, d.m, d.n);
  } else if (saves) {
    args.save16[0] = static_cast<uint16_t*>(save);
    args.save_wide = widest(d.n, save, nullptr);
  }
  if (t.width != 0) {
    args.width = t.width;
    args.a_bytes = a_box(d.m) * kTcHalf * 2u;
    args.stages = few_stages(d.m, t.width, 1);
    args.half_bytes = few_half(d.m, t.width, 1);
  }
  CUtensorMap maps[4];
  if ((st = make_map(maps[0], mx.p, d.m, d.k, mx.ld, a_box(d.m))) != GWS_OK) return st;
  maps[1] = maps[0];
  if ((st = make_map(maps[2], mw.p, d.n, d.k, mw.ld, t.width != 0 ? t.width : static_cast<uint32_t>(t.bn / t.cg))) != GWS_OK) return st;
  maps[3] = maps[2];
  if (t.width != 0) return launch_tc<1, 128, kLinearFew>(maps, args, sms, s);
  return residual != nullptr ? launch_mode<kLinear>(t, maps, args, sms, s) : launch_mode<kLinearAlone>(t, maps, args, sms, s);
}

int gws_linear_bwd(const gws_linear_desc* desc, const void* grad_y, const void* x, const void* w, const void* save, void* grad_x, void* grad_w, void* grad_bias,
                   void* act_out, void* workspace, size_t workspace_bytes, int* status, void* stream) {
  int st = check_linear(desc);
  if (st != GWS_OK) return st;
  const gws_linear_desc& d = *desc;
  const bool acts = d.activation != GWS_ACT_NONE, reads = acts || act_out != nullptr, saved8 = is_act8(d.save_format), x8 = is_act8(d.x_format);
  if ((reads && !saved8 && d.save_format != GWS_SAVE_BF16) || (!x8 && d.x_format != GWS_SAVE_BF16)) return GWS_ERR_UNSUPPORTED;
  const size_t bias_each = d.bias_type == GWS_TYPE_F32 ? 4 : 2;
  if (!on(grad_x, 2) || !on(grad_w, 2) || !on(grad_bias, bias_each) || !on(act_out, 2) || !on(status, 4)) return GWS_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d.m == 0 || d.n == 0) {              // empty sums
    if ((st = zero(grad_x, d.m, d.k, d.k, s)) != GWS_OK || (st = zero(grad_w, d.n, d.k, d.k, s)) != GWS_OK) return st;
    if (grad_bias == nullptr || d.n == 0) return GWS_OK;
    const cudaError_t err = cudaMemsetAsync(grad_bias, 0, static_cast<size_t>(bias_bytes(d)), s);
    return err == cudaSuccess ? GWS_OK : gws::report_cuda(err, "clearing a gradient");
  }
  const bool wants_dw = grad_w != nullptr, wants_dx = grad_x != nullptr, products = wants_dw || wants_dx;
  if (!products && grad_bias == nullptr && act_out == nullptr) return GWS_OK;
  const bool wants_dy = products || grad_bias != nullptr;
  if ((wants_dy && grad_y == nullptr) || (reads && save == nullptr) || (wants_dw && x == nullptr) || (wants_dx && w == nullptr)) return GWS_ERR_NULL;
  // without an activation the products read grad_y where it lies
  const bool moves_y = !acts && products && !in_place(d.m, d.ld_y), moves_x = !x8 && !in_place(d.m, d.ld_x), moves_w = !in_place(d.n, d.ld_w);
  if ((wants_dy && !on(grad_y, acts || moves_y || !products ? 2 : 16)) || (reads && !on(save, saved8 ? 32 : 2)) || (wants_dw && !on(x, x8 ? 32 : moves_x ? 2 : 16)) ||
      (wants_dx && !on(w, moves_w ? 2 : 16)))
    return GWS_ERR_ALIGN;
  const int sms = sm_count();
  const LinearBack& l = linear_back(desc, sms);
  const Span in_x = x8 ? Span{x, act8_total(d.m, d.k)} : rows_of(x, d.m, d.k, d.ld_x);
  if (clash({rows_of(grad_x, d.m, d.k, d.k), rows_of(grad_w, d.n, d.k, d.k), {grad_bias, grad_bias != nullptr ? bias_bytes(d) : 0}, rows_of(act_out, d.m, d.n, d.n),
             {workspace, l.total}},
            {rows_of(grad_y, d.m, d.n, d.ld_y), in_x, rows_of(w, d.n, d.k, d.ld_w), {save, reads ? kept_bytes(d.save_format, d.m, d.n) : 0}}))
    return GWS_ERR_ALIAS;
  if (!workspace_ok(workspace, workspace_bytes, l.total)) return GWS_ERR_WORKSPACE;
  char* ws = static_cast<char*>(workspace);

  Ready ready;
  Mat dz{grad_y, d.m, d.n, d.ld_y}, mw{w, d.n, d.k, d.ld_w}, mx{x, d.m, d.k, d.ld_x};
  const Act8View kept_x = act8_view(x, d.m, d.k);
  if (wants_dx) ready.align(mw, ws + l.w);
  if (wants_dw && x8 && !l.dw.inside) mx = ready.restore(kept_x, d.x_format, d.m, d.k, ws + l.x);
  if (wants_dw && !x8) ready.align(mx, ws + l.x);
  if (!acts && products) ready.align(dz, ws + l.dz);
  if ((acts && products) || grad_bias != nullptr || act_out != nullptr) {
    LinearPre p;
    std::memset(&p, 0, sizeof p);
    p.dy = wants_dy ? static_cast<const uint16_t*>(grad_y) : nullptr;
    p.ld_dy = d.m == 1 ? round_up(d.n, 8) : d.ld_y;
    if (acts && products) {
      p.dz = reinterpret_cast<uint16_t*>(ws + l.dz);
      p.ld_dz = packed_ld(d.n);
      dz = {p.dz, d.m, d.n, p.ld_dz};
    }
    if (saved8) p.save8 = act8_view(save, d.m, d.n);
    else p.save16 = static_cast<const uint16_t*>(save);
    p.again = static_cast<uint16_t*>(act_out);
    p.db = grad_bias;
    p.db_f32 = d.bias_type == GWS_TYPE_F32;
    p.rows = d.m;
    p.cols = d.n;
    const bool wide = d.n % 8 == 0 && (p.dy == nullptr || (on(grad_y, 16) && p.ld_dy % 8 == 0)) && (act_out == nullptr || on(act_out, 16)) &&
                      (!reads || saved8 || on(save, 16));
    if ((st = launch_linear_pre(p, ready, d.activation, reads ? d.save_format : GWS_SAVE_NONE, wide, ws + l.sums, sms, s)) != GWS_OK) return st;
  } else if ((st = ready.run(s)) != GWS_OK) {
    return st;
  }

  if (wants_dx) {
    const Tile& t = l.dx;
    TcArgs args = base_args(t, d.m, d.k, d.n, 1, status);
    args.half_bytes -= static_cast<uint32_t>(t.cg) * (128u - a_box(d.m)) * kTcHalf * 2u;
    set_out(args, grad_x, nullptr, d.k);
    args.part = reinterpret_cast<float*>(ws + l.part);
    CUtensorMap maps[4];
    if ((st = make_map(maps[0], dz.p, d.m, d.n, dz.ld, a_box(d.m))) != GWS_OK || (st = make_map(maps[2], mw.p, d.n, d.k, mw.ld, kTcHalf)) != GWS_OK) return st;
    maps[1] = maps[0];
    maps[3] = maps[2];
    if ((st = launch_mode<kDx>(t, maps, args, sms, s)) != GWS_OK) return st;
  }
  if (wants_dw) return run_dw(l.dw.tile, dz, nullptr, mx, l.dw.inside ? &kept_x : nullptr, d.x_format, grad_w, nullptr, d.k, ws + l.part, status, sms, s);
  return GWS_OK;
}

}  // extern "C"
