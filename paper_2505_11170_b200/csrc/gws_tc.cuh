// The tcgen05 GEMM of the gated feed-forward block and of the weight gradients: BF16 operands, FP32 accumulation in tensor
// memory, one persistent kernel with these uses (MODE):
//
//   kGated   h = act(x Wg^T) * (x Wu^T): both projections of a tile of h are two halves of one accumulator, so the activation,
//            the product and the 8-bit copies for the backward pass happen on registers in the epilogue
//   kGatedFew  the same for up to 128 tokens, tiles of 16 to 64 columns of h: every SM gets its share of the weights, and a copy of A
//            takes only the rows that exist, so that the ring holds more weights in flight.  It is bound by the weights' way from
//            memory and some 4 us around it (one token, 2048 x 5632: 46 MB in 12 us, 10 from L2; 4096 x 11008: 180 MB in 33 us)
//   kDx      dx = dg Wg + du Wu: one accumulator, the contraction runs over the columns of dg and then over those of du
//   kDw      dW = dY^T X: both operands are read along their contiguous (not the contracted) axis, as they lie in memory
//   kDw8     the same with X an 8-bit checkpoint: its codes are copied to shared memory and eight more warps turn them into the BF16
//            operand there, under the products of earlier stages, so that X crosses L2 and HBM at one byte per element and no BF16
//            copy of it exists
//
// A tile is 128 * CG rows by BN columns of accumulator; CG = 2 is a pair of SMs working on one tile (cta_group::2: each SM
// holds its 128 rows of A and half of the columns of B, so an operand byte fetched from L2 feeds twice the products).
// Warp roles: warp 0 starts the TMA copies (64 or 128 elements along the contraction per stage, 128-byte swizzle), warp 1 issues the
// tcgen05.mma of the pair, warps 4 and up are the epilogue.  The accumulator is double-buffered in tensor memory, so the
// epilogue of a tile runs under the products of the next one.  Blocks are persistent and take tiles round robin, in groups
// of rows so that the tiles in flight share operands in L2.
//
// The tiles that do not fill a last wave of blocks (all of them, when there are few) have their contraction cut into `splits`
// parts, each written as FP32; k_join adds the parts in a fixed order, so results do not depend on timing, and finishes the tile.
// Where one wave holds all parts of all tiles, the parts of a tile are the blocks of a cluster instead, which add them through each
// other's shared memory in the same launch.
//
// What bounds it (16384 tokens, 2048 x 5632): the tensor cores and, beyond some milliseconds, the 1 kW power cap.  In a burst the forward
// pass takes 477 us (1.58 PFLOP/s; 497 us with INT8 copies), dx 463 us and both dW 464 us (1.63 PFLOP/s) against 1.68 measured for a
// large square library product; the tensor pipe is busy 83 % of a launch on 4096 tokens, ends included.  Repeated for half a second
// they take 557 to 564, 589 to 609 and 590 to 600 us (dx and dW with the element-wise pass's 137 us taken off), and torch.matmul on BF16
// operands of the same sizes, [16384, 2048] by [11264, 2048]^T, [16384, 11264] by [11264, 2048] and [16384, 11264]^T by [16384, 2048],
// 589 to 600, 568 to 582 and 577 to 595 us.
//
// Every wait of a role is a wait on an mbarrier and has a limit (about a second); one that runs out has the status word set and ends its
// role, the roles that depend on it run out in turn, the block gives its copies time to land, frees its tensor memory and returns.
// What has no limit waits for something that does not depend on a role's success:
//   __syncthreads and the cluster barriers come after the roles' loops (or before them), where every warp arrives whatever happened;
//   the allocation of tensor memory waits for blocks of other kernels on the SM: none of these kernels, since two blocks of them do not fit
//   an SM (static_assert at TcShape), and no kernel behind this one on the stream, since none of them starts before all blocks of this one
//   have their tensor memory;
//   griddepcontrol.wait waits for the kernel before, which never waits for this one.
#pragma once
#include <cuda.h>
#include <stdint.h>

#include "gws_act8.cuh"

namespace {

enum { kGated = 0, kDx = 1, kDw = 2, kDw8 = 3, kGatedFew = 4 };

constexpr uint32_t kTcHalf = 64;                           // elements along the contraction per copy: 128 bytes, one swizzle atom
constexpr uint32_t kTcABytes = 128u * kTcHalf * 2u;
constexpr uint32_t kTcSmem = 227u * 1024u;
constexpr uint32_t kTcStagingWarp = 32u * 17u * 4u;        // a 32 x 32 BF16 block per epilogue warp, rows 17 words apart
constexpr long long kTcWaitCycles = 2000000000LL;         // limit of a wait, unless gws_set_wait_limit gave another one
constexpr long long kTcLandCycles = 125000000LL;          // what a block that gave up leaves its copies and products to end

struct TcArgs {
  uint32_t m_tiles, n_tiles;              // tiles along rows (all outputs), along columns
  uint32_t whole, cut, splits;            // tiles computed in one piece, and the rest, cut into `splits` parts
  int32_t clustered;                      // the parts of a tile are the blocks of a cluster (CG = 1, no whole tiles, one part a block)
  uint32_t tiles_per_out;                 // kDw: row tiles of the first output
  uint32_t kb, kb_first, kb_split;        // stages of the contraction: all, of the first segment (kDx), of one part
  uint32_t len;                           // elements of the contraction (kDx: of each segment)
  uint32_t group;                         // row tiles per group of the tile order
  uint32_t parts;                         // kDw: 16-step parts of a copy that hold tokens (4 unless there are fewer than 64 tokens)
  uint32_t half_bytes;                    // bytes the copies of 64 elements along the contraction bring, over the CG blocks
  int64_t rows, cols;                     // of one output
  void* out[2];                           // BF16
  int64_t ld_out;
  int32_t wide;                           // elements a store to `out` may take: 1, 2, 4, 8, or 16 (32 bytes)
  float* part;                            // FP32 [splits][cut][128 * CG][BN]
  const uint8_t* scales;                  // kDw8: scale bytes of X, [tokens, scales_ld]
  int64_t scales_ld;
  int32_t x_format;
  int32_t box_tokens;                     // kDw, kDw8: tokens in a copy
  int32_t activation, save;               // kGated
  uint32_t width, stages, a_bytes;        // kGatedFew: columns of h in a tile, stages of the ring, bytes of A in a copy
  int32_t save_wide;                      // the same for the BF16 copies
  Act8View save8[2];
  uint16_t* save16[2];                    // BF16 copies, [rows, cols]
  int* status;
  int64_t wait_limit;
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t block_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
// Arrives on a barrier of any block of the pair (shared::cluster address).  What it announces is the arriving block's own shared or
// tensor memory, ordered for the tensor cores by the proxy or tcgen05 fence before it; a release at cluster scope would wait for
// all of the warp's memory traffic instead (a stage of conversion took 1900 cycles with it, 700 without).
__device__ __forceinline__ void bar_arrive(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// A whole warp waits for the phase of the given parity; false, for every lane, if it did not complete within `limit` cycles.  The
// clock is only read once the first try has failed: the two warps that feed the tensor cores pass here once per stage.
// CLUSTER: what the other block of the pair wrote before it arrived is visible afterwards.
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_try(uint32_t addr, uint32_t parity) {
  uint32_t done;
  if (CLUSTER)
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done)
                 : "r"(addr), "r"(parity)
                 : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done)
               : "r"(addr), "r"(parity)
               : "memory");
  return done != 0;
}
// The same without waiting at all.
__device__ __forceinline__ bool bar_peek(uint32_t addr, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done)
               : "r"(addr), "r"(parity)
               : "memory");
  return done != 0;
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_wait(uint32_t addr, uint32_t parity, long long limit) {
  if (__all_sync(0xFFFFFFFFu, bar_try<CLUSTER>(addr, parity))) return true;
  const long long t0 = clock64();
  for (;;) {
    if (__all_sync(0xFFFFFFFFu, bar_try<CLUSTER>(addr, parity))) return true;
    if (__any_sync(0xFFFFFFFFu, clock64() - t0 > limit)) return false;
  }
}
// One lane of a converged warp.  The loops around it are run by the whole warp, so that addresses and descriptors stay in
// uniform registers: a loop run by one lane alone spent 346 cycles on the four products and the commit of a stage.
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}

template <int CG>
__device__ __forceinline__ void copy_in(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y) {
  if (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}

// Shared-memory matrix descriptors, 128-byte swizzle (layout type 2), descriptor version 1.
// Contraction contiguous: rows of 128 bytes (64 elements along the contraction), 1024 bytes between groups of 8 rows.
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (static_cast<uint64_t>(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Other axis contiguous: blocks of 64 elements along it by 64 steps of the contraction (8192 bytes each, one row of 128 bytes
// per step); 8192 bytes between blocks, 1024 bytes between groups of 8 steps.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(8192u >> 4) << 16) | (static_cast<uint64_t>(1024u >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}

template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (CG == 2)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
// Signals the barrier (in both blocks of a pair) when all products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)),
                 "h"(static_cast<uint16_t>(3))
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

__device__ __forceinline__ void acc_load(uint32_t addr, uint32_t (&r)[32]) {
  __syncwarp();                          // the load is one of the whole warp; lanes may come from rows treated differently
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
      "%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void acc_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// act(g) and its slope.  SiLU is g sigmoid(g); GELU in its tanh form is g sigmoid(z), z = 2 sqrt(2/pi) (g + 0.044715 g^3),
// because (1 + tanh(z / 2)) / 2 = sigmoid(z).
constexpr float kGeluLin = 1.59576912160573f;    // 2 sqrt(2 / pi)
template <int ACT>
__device__ __forceinline__ float sigmoid_arg(float g) {
  return ACT == GWS_GATED_SILU ? g : g * __fmaf_rn(kGeluLin * 0.044715f, g * g, kGeluLin);
}
// 1 / (1 + 2^(-z log2 e)): two special-function operations, which set the pace of the forward epilogue where the contraction is short, and
// two others.  Both flush what is below 2^-126 to zero; an argument beyond the range gives 0 or 1.
__device__ __forceinline__ float sigmoid(float z) {
  float e, s;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
  return s;
}
template <int ACT>
__device__ __forceinline__ float act_of(float g) {
  if (ACT == GWS_GATED_RELU) return g < 0.0f ? 0.0f : g;
  return g * sigmoid(sigmoid_arg<ACT>(g));
}
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float& a, float& slope) {
  if (ACT == GWS_GATED_RELU) {
    a = g < 0.0f ? 0.0f : g;
    slope = g > 0.0f ? 1.0f : 0.0f;
    return;
  }
  const float s = sigmoid(sigmoid_arg<ACT>(g));
  a = g * s;
  // g^2 stays finite: beyond |g| = 2^50 the sigmoid is 0 or 1 and the term has to vanish, not become 0 times infinity
  const float dz = ACT == GWS_GATED_SILU ? 1.0f : __fmaf_rn(3.0f * 0.044715f * kGeluLin, fminf(g * g, 0x1p100f), kGeluLin);
  slope = __fmaf_rn(a * (1.0f - s), dz, s);
}

// The first `width` columns of a 32 x 32 block of BF16 from shared memory (rows 17 words apart) to rows that take stores of V elements: a
// lane V columns, a warp V rows at a time.
template <uint32_t V>
__device__ __forceinline__ void store_rows(uint16_t* p, int64_t ld, int64_t left, uint32_t width, const uint32_t* staging, uint32_t lane) {
  constexpr uint32_t kLanes = 32u / V, kBatch = V == 1u ? 8u : V == 2u ? 4u : 2u;
  const uint32_t row = lane / kLanes, word = (lane % kLanes) * V / 2u;
  if ((lane % kLanes) * V >= width) return;
  const uint32_t* s = staging + row * 17u + word;
  p += row * ld + (lane % kLanes) * V;
#pragma unroll
  for (uint32_t r = 0; r < 32u; r += V * kBatch) {
    uint32_t v[kBatch][V == 1u ? 1u : V / 2u];
#pragma unroll
    for (uint32_t i = 0; i < kBatch; ++i) {
      if constexpr (V == 1u) {
        v[i][0] = reinterpret_cast<const uint16_t*>(s + (r + i) * 17u)[lane & 1u];
      } else {
#pragma unroll
        for (uint32_t e = 0; e < V / 2u; ++e) v[i][e] = s[(r + i * V) * 17u + e];
      }
    }
#pragma unroll
    for (uint32_t i = 0; i < kBatch; ++i, p += V * ld) {
      if (r + i * V + row >= left) continue;
      if constexpr (V == 1u) *p = static_cast<uint16_t>(v[i][0]);
      else if constexpr (V == 2u) *reinterpret_cast<uint32_t*>(p) = v[i][0];
      else if constexpr (V == 4u) *reinterpret_cast<uint2*>(p) = make_uint2(v[i][0], v[i][1]);
      else *reinterpret_cast<uint4*>(p) = make_uint4(v[i][0], v[i][1], v[i][2], v[i][3]);
    }
  }
}

// Writes a 32 x 32 block of BF16 held one row per lane (16 words of two columns each).  `wide`: elements that a store may take at once
// (rows and base aligned to them).  16 of them: straight from the lanes.  Fewer, or a block that reaches past the width: through shared
// memory, so that the warp still writes neighbouring columns of a row with neighbouring lanes.
__device__ __forceinline__ void store_block(uint16_t* out, int64_t ld, int32_t wide, int64_t row0, int64_t col0, int64_t rows, int64_t cols,
                                            const uint32_t (&w)[16], uint32_t* staging, uint32_t lane) {
  if (wide == 16 && col0 + 32 <= cols) {
    if (row0 + lane < rows) {
      uint16_t* p = out + (row0 + lane) * ld + col0;
      V8 a, b;
#pragma unroll
      for (int i = 0; i < 8; ++i) { a.x[i] = w[i]; b.x[i] = w[8 + i]; }
      st32(p, a);
      st32(p + 16, b);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) staging[lane * 17u + i] = w[i];
  __syncwarp();
  const int64_t left = rows - row0;
  uint16_t* p = out + row0 * ld + col0;
  const uint32_t width = col0 + 32 <= cols ? 32u : static_cast<uint32_t>(cols - col0);
  if (wide >= 8 && width % 8u == 0) store_rows<8>(p, ld, left, width, staging, lane);
  else if (wide >= 4 && width % 4u == 0) store_rows<4>(p, ld, left, width, staging, lane);
  else if (wide >= 2 && width % 2u == 0) store_rows<2>(p, ld, left, width, staging, lane);
  else store_rows<1>(p, ld, left, width, staging, lane);
  __syncwarp();
}

template <int ACT>
__device__ __forceinline__ void gate_block(const uint32_t (&g)[32], const uint32_t (&u)[32], uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    w[i] = pack_bf16(act_of<ACT>(__uint_as_float(g[2 * i])) * __uint_as_float(u[2 * i]),
                     act_of<ACT>(__uint_as_float(g[2 * i + 1])) * __uint_as_float(u[2 * i + 1]));
}

// Tile number -> (row tile, column tile): groups of `group` row tiles, column by column inside a group.
__device__ __forceinline__ void tile_at(const TcArgs& p, uint32_t t, uint32_t& mt, uint32_t& nt) {
  const uint32_t per_group = p.group * p.n_tiles, g = t / per_group, rest = t - g * per_group;
  const uint32_t height = min(p.group, p.m_tiles - g * p.group);
  nt = rest / height;
  mt = g * p.group + (rest - nt * height);
}

template <int CG, int BN, int MODE>
struct TcShape {
  static constexpr uint32_t kBRows = BN / CG;                              // columns of B each block holds
  static constexpr uint32_t kEpilogueWarps = 8u;                           // two per quadrant of the accumulator's rows
  static constexpr uint32_t kConvertWarps = MODE == kDw8 ? 8u : 0u;
  static constexpr uint32_t kThreads = 128u + 32u * (kEpilogueWarps + kConvertWarps);
  static constexpr uint32_t kStaging = kEpilogueWarps * kTcStagingWarp;
  // Copies of 64 elements per stage.  A stage costs the warp that issues the products some 250 cycles whatever it holds; the
  // products of 64 elements take 512 cycles with 256 columns on a pair of SMs, 128 to 256 with the smaller tiles, which therefore
  // take two copies per stage (2048 x 5632 into 128 rows, 128 columns: 396 -> 250 cycles per 64 elements).
  static constexpr uint32_t kHalves = BN == 256 ? 1u : 2u;
  static constexpr uint32_t kBBytes = kBRows * kTcHalf * 2u;
  static constexpr uint32_t kRaw = MODE == kDw8 ? kBRows * kTcHalf : 0u;   // codes of B
  static constexpr uint32_t kHalf = kTcABytes + kBBytes + kRaw;            // A, B, codes
  static constexpr uint32_t kStage = kHalves * kHalf;
  static constexpr uint32_t kFit = (kTcSmem - 4096u - kStaging) / kStage;
  // kGatedFew parts the same memory into as many stages as its narrower copies allow
  static constexpr uint32_t kStages = kFit > 8u || MODE == kGatedFew ? 8u : kFit;
  static constexpr uint32_t kRing = (kFit > 8u ? 8u : kFit) * kStage;
  static constexpr uint32_t kSmemBytes = kRing + kStaging + 1024u;
  static constexpr uint32_t kTmemCols = 2 * BN;
  static_assert(2u * kSmemBytes > kTcSmem, "a block that holds tensor memory keeps other blocks of these kernels off its SM");
};

constexpr uint32_t kPartRow = 128u * 4u + 16u;      // bytes between rows of a part in shared memory: eight lanes' 16 bytes in different banks

// Codes of a checkpoint -> BF16 numbers, two at a time in packed BF16 arithmetic; every step is exact.
// INT8: a code c = low - 128 s (its low 7 bits and its sign bit); with 0x43 above it the byte is a BF16 number, 128 + low without the
// sign bit and 128 (1 + s) without the low bits, whose difference is c.  2 1/2 instructions a code against 3 3/4 through FP32.
// E4M3: its exponent and mantissa 4 bits up are those of a BF16 number 2^120 too small (subnormals included).
template <int FMT>
struct Units {
  __nv_bfloat162 unit;
  __device__ __forceinline__ explicit Units(uint32_t byte) : unit(__float2bfloat162_rn(unit_of<FMT>(byte))) {}
};
__device__ __forceinline__ __nv_bfloat162 as_pair(uint32_t v) { return *reinterpret_cast<const __nv_bfloat162*>(&v); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t*>(&v); }
template <int FMT>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, uint32_t half, const Units<FMT>& u) {
  if (FMT == GWS_ACT8_INT8) {
    const uint32_t p = __byte_perm(codes, 0x43434343u, half == 0u ? 0x4140u : 0x4342u);
    return as_word(__hmul2(__hsub2(as_pair(p & 0xFF7FFF7Fu), as_pair(p & 0xFF80FF80u)), u.unit));
  }
  const uint32_t p = __byte_perm(codes, 0u, half == 0u ? 0x1404u : 0x3424u), mag = (p >> 4) & 0x07F007F0u;
  return as_word(__hmul2(__hmul2(as_pair((p & 0x80008000u) | mag), __float2bfloat162_rn(0x1p120f)), u.unit));
}
template <int FMT>
__device__ __forceinline__ uint4 bf16_of_codes(uint32_t lo, uint32_t hi, const Units<FMT>& u) {
  return make_uint4(bf16_pair<FMT>(lo, 0, u), bf16_pair<FMT>(lo, 1, u), bf16_pair<FMT>(hi, 0, u), bf16_pair<FMT>(hi, 1, u));
}

// Four warps' conversion of a copy: 64 tokens by COLS columns of codes (as the copy left them, rows of COLS bytes, swizzled) to the
// BF16 operand (blocks of 64 columns, rows of 128 bytes, swizzled).  A thread takes one token's COLS / 2 columns, so that eight
// neighbouring lanes touch eight different 16-byte columns of the banks on either side.
template <int FMT, uint32_t COLS>
__device__ __forceinline__ void convert_codes(uint32_t raw, uint32_t dst, uint32_t token, uint32_t side, const uint32_t (&bytes)[COLS / 64u]) {
#pragma unroll
  for (uint32_t g = 0; g < COLS / 64u; ++g) {
    const Units<FMT> unit(bytes[g]);
#pragma unroll
    for (uint32_t h = 0; h < 2u; ++h) {
      const uint32_t c = side * (COLS / 32u) + g * 2u + h;                       // 16-byte unit of the row of codes
      const uint32_t from = raw + token * COLS + ((COLS == 128u ? c ^ (token & 7u) : c ^ ((token >> 1) & 3u)) << 4);
      uint32_t w[4];
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from));
#pragma unroll
      for (uint32_t q = 0; q < 2u; ++q) {
        const uint4 v = bf16_of_codes<FMT>(w[2 * q], w[2 * q + 1], unit);
        const uint32_t unit16 = c * 2u + q;                                      // 16-byte unit of the row of BF16 numbers
        const uint32_t to = dst + (unit16 >> 3) * 8192u + token * 128u + (((unit16 & 7u) ^ (token & 7u)) << 4);
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w));
      }
    }
  }
}

template <int CG, int BN, int MODE>
__global__ void __launch_bounds__((TcShape<CG, BN, MODE>::kThreads), 1)
    k_tc(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1, const __grid_constant__ CUtensorMap b0,
         const __grid_constant__ CUtensorMap b1, const __grid_constant__ TcArgs p) {
  using S = TcShape<CG, BN, MODE>;
  constexpr bool kFew = MODE == kGatedFew, kIsGated = MODE == kGated || kFew, kIsDw = MODE == kDw || MODE == kDw8, kMnA = kIsDw, kMnB = !kIsGated;
  constexpr uint32_t kStages = S::kStages;
  const uint32_t stages = kFew ? p.stages : kStages, width = kFew ? p.width : BN / 2;      // width: columns of h in a tile (kIsGated)
  const uint32_t a_bytes = kFew ? p.a_bytes : kTcABytes, half_pitch = kFew ? a_bytes + width * (kTcHalf * 4u) : S::kHalf, stage_pitch = S::kHalves * half_pitch;
  // instruction descriptor: FP32 accumulator, BF16 operands, which axis of A and B is contiguous, N, M
  const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((kMnA ? 1u : 0u) << 15) | ((kMnB ? 1u : 0u) << 16) |
                         ((kFew ? width >> 2 : static_cast<uint32_t>(BN >> 3)) << 17) | (static_cast<uint32_t>((128 * CG) >> 4) << 24);
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], meet[4], codes_full[kStages], converted[kStages];
  __shared__ __align__(16) uint8_t scale_bytes[2][2][kIsGated ? 128 : 1][4];      // of two tiles, gate and up projection
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int failed;
  const uint32_t raw = smem_addr(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);   // the same offset in both blocks of a pair
  uint32_t* staging = reinterpret_cast<uint32_t*>(smem + S::kRing);

  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t rank = CG == 2 ? block_rank() : 0u;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < kStages; ++s) {
      bar_init(&full[s], 1);
      bar_init(&empty[s], 1);
      bar_init(&codes_full[s], 1);
      bar_init(&converted[s], 4 * CG);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(&acc_full[b], 1);
      bar_init(&acc_empty[b], S::kEpilogueWarps * CG);
    }
    for (int q = 0; q < 4; ++q) bar_init(&meet[q], 2);
    failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(S::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(S::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) pair_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  if (warp == 0 && elected()) {          // the descriptions of the operands are on their way before the first copy asks for them
    for (const CUtensorMap* map : {&a0, &b0, &a1, &b1}) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
  }
  after_previous();

  const uint32_t work = p.whole + p.cut * p.splits;
  const uint32_t first = blockIdx.x / CG, stride = gridDim.x / CG;
  // work item -> tile and stages of the contraction
  auto place = [&](uint32_t t, uint32_t& mt, uint32_t& nt, uint32_t& k0, uint32_t& k1) {
    k0 = 0;
    k1 = p.kb;
    if (t >= p.whole) {
      const uint32_t split = p.clustered ? t % p.splits : (t - p.whole) / p.cut;
      t = p.clustered ? t / p.splits : t - split * p.cut;
      k0 = split * p.kb_split;
      k1 = min(p.kb, k0 + p.kb_split);
    }
    tile_at(p, t, mt, nt);
  };

  if (warp == 0) {
    uint32_t s = 0, parity = 1;                        // stage, and the parity of its last release (none before the first round)
    bool ok = true;
    const uint32_t full0 = CG == 2 ? at_rank(smem_addr(&full[0]), 0u) : smem_addr(&full[0]), empty0 = smem_addr(&empty[0]);
    for (uint32_t t = first; ok && t < work; t += stride) {
      uint32_t mt, nt, k0, k1;
      place(t, mt, nt, k0, k1);
      const bool second = kIsDw && mt >= p.tiles_per_out;
      const int32_t m0 = static_cast<int32_t>((second ? mt - p.tiles_per_out : mt) * (128u * CG) + rank * 128u);
      const int32_t n0 = static_cast<int32_t>(nt * (kIsGated ? width : BN) + (kIsGated ? 0u : rank * S::kBRows));
      for (uint32_t kb = k0; kb < k1; ++kb) {
        if (!bar_wait(empty0 + 8u * s, parity, p.wait_limit)) { ok = false; break; }
        const bool seg = MODE == kDx && kb >= p.kb_first;
        const uint32_t k = (seg ? kb - p.kb_first : kb) * (S::kHalves * kTcHalf);
        const uint32_t halves = S::kHalves == 1u || k + kTcHalf >= p.len ? 1u : 2u;     // a second copy past the end is left out
        if (elected()) {
          if (rank == 0) bar_expect(&full[s], halves * p.half_bytes);
          if (MODE == kDw8) bar_expect(&codes_full[s], halves * S::kBRows * static_cast<uint32_t>(p.box_tokens));
          const uint32_t bar = full0 + 8u * s;
#pragma unroll
          for (uint32_t i = 0; i < S::kHalves; ++i) {
            if (i >= halves) break;
            const uint32_t sa = smem_addr(smem) + s * stage_pitch + i * half_pitch, sb = sa + a_bytes;
            const int32_t ki = static_cast<int32_t>(k + i * kTcHalf);
            if (kIsGated) {
              copy_in<CG>(sa, &a0, bar, ki, m0);
              if (CG == 2) {                             // block 0 holds the gate's rows, block 1 the up projection's
                copy_in<CG>(sb, rank == 0 ? &b0 : &b1, bar, ki, n0);
              } else {
                copy_in<CG>(sb, &b0, bar, ki, n0);
                copy_in<CG>(sb + width * (kTcHalf * 2u), &b1, bar, ki, n0);
              }
            } else if (MODE == kDx) {
              copy_in<CG>(sa, seg ? &a1 : &a0, bar, ki, m0);
#pragma unroll
              for (uint32_t j = 0; j < S::kBRows / 64u; ++j) copy_in<CG>(sb + j * 8192u, seg ? &b1 : &b0, bar, n0 + static_cast<int32_t>(j * 64u), ki);
            } else {
#pragma unroll
              for (uint32_t j = 0; j < 2u; ++j) copy_in<CG>(sa + j * 8192u, second ? &a1 : &a0, bar, m0 + static_cast<int32_t>(j * 64u), ki);
              if (MODE == kDw8) {
                copy_in<1>(sb + S::kBBytes, &b0, smem_addr(&codes_full[s]), n0, ki);
              } else {
#pragma unroll
                for (uint32_t j = 0; j < S::kBRows / 64u; ++j) copy_in<CG>(sb + j * 8192u, &b0, bar, n0 + static_cast<int32_t>(j * 64u), ki);
              }
            }
          }
        }
        __syncwarp();
        if (++s == stages) { s = 0; parity ^= 1u; }
      }
    }
    // Every release of a stage has to have arrived before this block's shared memory may become another block's: the signal of a commit
    // comes from the other SM of the pair, on its own time, and would count on whatever barrier lies there by then.
    for (uint32_t i = 0; ok && i < stages; ++i) {
      ok = bar_wait(empty0 + 8u * s, parity, p.wait_limit);
      if (++s == stages) { s = 0; parity ^= 1u; }
    }
    if (!ok) failed = 1;
  } else if (warp == 1) {
    if (rank == 0) {
      uint32_t s = 0, parity = 0, n = 0;
      bool ok = true;
      const uint32_t full0 = smem_addr(&full[0]), acc_empty0 = smem_addr(&acc_empty[0]);
      const uint64_t da = kMnA ? desc_mn(smem_addr(smem)) : desc_k(smem_addr(smem));
      const uint64_t db = kMnB ? desc_mn(smem_addr(smem) + a_bytes) : desc_k(smem_addr(smem) + a_bytes);
      // 16 steps of the contraction in the units of a descriptor's address: 32 bytes of a row, or 16 rows of 128 bytes
      constexpr uint32_t kStepA = (kMnA ? 2048u : 32u) >> 4, kStepB = (kMnB ? 2048u : 32u) >> 4;
      for (uint32_t t = first; ok && t < work; t += stride, ++n) {
        uint32_t mt, nt, k0, k1;
        place(t, mt, nt, k0, k1);
        const uint32_t buf = n & 1u, d = tmem + buf * BN;
        if (!bar_wait<CG == 2>(acc_empty0 + 8u * buf, ((n >> 1) & 1u) ^ 1u, p.wait_limit)) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        bool ready = bar_try(full0 + 8u * s, parity);
        for (uint32_t kb = k0; kb < k1; ++kb) {
          if (!__all_sync(0xFFFFFFFFu, ready) && !bar_wait(full0 + 8u * s, parity, p.wait_limit)) { ok = false; break; }
          if (MODE == kDw8 && !bar_wait<CG == 2>(smem_addr(&converted[s]), parity, p.wait_limit)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t now = s;
          if (++s == stages) { s = 0; parity ^= 1u; }
          if (kb + 1 < k1) ready = bar_peek(full0 + 8u * s, parity);      // answered while the products below are issued
          const bool seg = MODE == kDx && kb >= p.kb_first;
          const uint32_t k = (seg ? kb - p.kb_first : kb) * (S::kHalves * kTcHalf);
          const uint32_t halves = S::kHalves == 1u || k + kTcHalf >= p.len ? 1u : 2u;
          if (elected()) {
#pragma unroll
            for (uint32_t i = 0; i < S::kHalves; ++i) {
              if (i >= halves) break;
              const uint64_t sa = da + ((now * stage_pitch + i * half_pitch) >> 4), sb = db + ((now * stage_pitch + i * half_pitch) >> 4);
              mma<CG>(d, sa, sb, idesc, kb > k0 || i > 0 ? 1u : 0u);
#pragma unroll
              for (uint32_t j = 1; j < kTcHalf / 16u; ++j)
                if (!kIsDw || j < p.parts) mma<CG>(d, sa + j * kStepA, sb + j * kStepB, idesc, 1u);
            }
            commit<CG>(&empty[now]);
          }
          __syncwarp();
        }
        if (ok && elected()) commit<CG>(&acc_full[buf]);
        __syncwarp();
      }
      // ... and so does every hand-back of an accumulator
      for (uint32_t back = 1; ok && back <= 2u && back <= n; ++back)
        ok = bar_wait<CG == 2>(acc_empty0 + 8u * ((n - back) & 1u), ((n - back) >> 1) & 1u, p.wait_limit);
      if (!ok) failed = 1;
    }
  } else if (warp >= 4 && warp < 4u + S::kEpilogueWarps) {
    const uint32_t quadrant = warp & 3u, half = (warp - 4u) >> 2;   // a warp reads the 32 accumulator rows of its quadrant
    uint32_t* stage = staging + (warp - 4u) * 32u * 17u;
    uint32_t n = 0;
    for (uint32_t t = first; t < work; t += stride, ++n) {
      uint32_t mt, nt, k0, k1;
      place(t, mt, nt, k0, k1);
      const uint32_t buf = n & 1u;
      if (!bar_wait(smem_addr(&acc_full[buf]), (n >> 1) & 1u, p.wait_limit)) {
        failed = 1;
        break;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t acc = tmem + ((quadrant * 32u) << 16) + buf * BN;
      const bool second = kIsDw && mt >= p.tiles_per_out;
      const int64_t row0 = static_cast<int64_t>(second ? mt - p.tiles_per_out : mt) * (128 * CG) + rank * 128u + quadrant * 32u;
      if (CG == 1 && !kIsGated && p.clustered) {      // a part, into this block's shared memory: its copies and products are done
#pragma unroll 1
        for (uint32_t c = half; c < BN / 32; c += S::kEpilogueWarps / 4u) {
          uint32_t v[32];
          acc_load(acc + c * 32u, v);
          acc_wait();
          uint4* to = reinterpret_cast<uint4*>(smem + (quadrant * 32u + lane) * kPartRow + c * 128u);
#pragma unroll
          for (int i = 0; i < 8; ++i) to[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
      } else if (!kFew && t >= p.whole) {     // a part of a contraction: FP32, joined by k_join
        float* part = p.part + static_cast<int64_t>(t - p.whole) * (128 * CG * BN) + (rank * 128u + quadrant * 32u + lane) * BN;
#pragma unroll 1
        for (uint32_t c = half; c < BN / 32; c += S::kEpilogueWarps / 4u) {
          uint32_t v[32];
          acc_load(acc + c * 32u, v);
          acc_wait();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            V8 x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x.x[e] = v[8 * i + e];
            st32(part + c * 32u + 8 * i, x);
          }
        }
      } else if (kIsGated) {
        const int64_t edge = kFew ? min(p.cols, static_cast<int64_t>(nt + 1u) * width) : p.cols;      // where the tile's columns end
#pragma unroll 1
        for (uint32_t c = half; c < (width + 31u) / 32u; c += S::kEpilogueWarps / 4u) {
          uint32_t g[32], u[32], w[16];
          acc_load(acc + c * 32u, g);
          acc_load(acc + width + c * 32u, u);
          acc_wait();
          const int64_t col0 = static_cast<int64_t>(nt) * width + c * 32u;
          if (col0 >= edge) continue;
          if (p.activation == GWS_GATED_SILU) gate_block<GWS_GATED_SILU>(g, u, w);
          else if (p.activation == GWS_GATED_GELU_TANH) gate_block<GWS_GATED_GELU_TANH>(g, u, w);
          else gate_block<GWS_GATED_RELU>(g, u, w);
          store_block(static_cast<uint16_t*>(p.out[0]), p.ld_out, p.wide, row0, col0, p.rows, edge, w, stage, lane);
          if (p.save == GWS_SAVE_BF16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(g[2 * i]), __uint_as_float(g[2 * i + 1]));
            store_block(p.save16[0], p.cols, p.save_wide, row0, col0, p.rows, edge, w, stage, lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
            store_block(p.save16[1], p.cols, p.save_wide, row0, col0, p.rows, edge, w, stage, lane);
          } else if (p.save != GWS_SAVE_NONE && row0 + lane < p.rows) {
            // columns past the width are products with rows of zeros: zero codes, as the layout wants them
            const int64_t row = row0 + lane;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
              float v[kGroup];
#pragma unroll
              for (int i = 0; i < kGroup; ++i) v[i] = __uint_as_float(which == 0 ? g[i] : u[i]);
              V8 codes;
              const uint32_t byte = p.save == GWS_ACT8_INT8 ? encode_group<GWS_ACT8_INT8>(v, codes) : encode_group<GWS_ACT8_E4M3>(v, codes);
              st32(p.save8[which].codes + row * p.save8[which].ld + col0, codes);
              scale_bytes[buf][which][quadrant * 32u + lane][c] = static_cast<uint8_t>(byte);
            }
          }
        }
        if (p.save == GWS_ACT8_INT8 || p.save == GWS_ACT8_E4M3) {
          // The scale bytes of a row's groups in this tile leave together: one store of a byte each cost 20 us of 514 (16384 x 2048 x 5632).
          // The two warps that share these rows meet; one writes the gate's, the other the up projection's.  A warp that fills the same
          // buffer again has passed the meeting of the tile between, and so has the other one's store.  They meet at an mbarrier, one
          // phase a tile, because a wait there has a limit: a warp that left its loop does not leave the other one behind for good.
          __syncwarp();
          if (lane == 0) bar_arrive(smem_addr(&meet[quadrant]));
          if (!bar_wait(smem_addr(&meet[quadrant]), n & 1u, p.wait_limit)) { failed = 1; break; }
          const int64_t row = row0 + lane, ld = p.save8[half].ld >> 5, g0 = static_cast<int64_t>(nt) * (width / 32u);
          if (row < p.rows) {
            uint8_t* to = p.save8[half].scales + row * ld + g0;
            const uint8_t* from = scale_bytes[buf][half][quadrant * 32u + lane];
            const uint32_t groups = width / 32u;
            if (groups > 1u && g0 + groups <= ld && ld % groups == 0) {       // the buffer's scales start at a multiple of 256 bytes
              if (groups == 4u) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
              else *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(from);
            } else {
              for (uint32_t i = 0; i < groups && g0 + i < ld; ++i) to[i] = from[i];
            }
          }
        }
      } else {
        uint16_t* out = static_cast<uint16_t*>(p.out[second ? 1 : 0]);
#pragma unroll 1
        for (uint32_t c = half; c < BN / 32; c += S::kEpilogueWarps / 4u) {
          uint32_t v[32], w[16];
          acc_load(acc + c * 32u, v);
          acc_wait();
          const int64_t col0 = static_cast<int64_t>(nt) * BN + c * 32u;
          if (col0 >= p.cols) continue;
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
          store_block(out, p.ld_out, p.wide, row0, col0, p.rows, p.cols, w, stage, lane);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) bar_arrive(CG == 2 ? at_rank(smem_addr(&acc_empty[buf]), 0u) : smem_addr(&acc_empty[buf]));
    }
  } else if (MODE == kDw8 && warp >= 4u + S::kEpilogueWarps) {
    // Two teams of four warps take the stages in turn: one waits for codes while the other converts.
    const uint32_t i = threadIdx.x - 32u * (4u + S::kEpilogueWarps), team = i >> 7, token = i & 63u, side = (i >> 6) & 1u;
    constexpr uint32_t kGroups = S::kBRows / 64u;        // scale bytes of a thread per copy
    // They come from global memory kAhead of the team's stages before they are needed.
    constexpr uint32_t kAhead = 2;
    uint32_t it = 0;                                     // stages of all tiles before the present one
    bool ok = true;
    for (uint32_t t = first; ok && t < work; t += stride) {
      uint32_t mt, nt, k0, k1;
      place(t, mt, nt, k0, k1);
      const uint32_t group = (nt * BN + rank * S::kBRows) / 32u + side * kGroups;
      const uint8_t* scales = p.scales + group;
      uint32_t bytes[kAhead][S::kHalves][kGroups];
      auto fetch = [&](uint32_t kb, uint32_t (&to)[S::kHalves][kGroups]) {
#pragma unroll
        for (uint32_t h = 0; h < S::kHalves; ++h)
#pragma unroll
          for (uint32_t g = 0; g < kGroups; ++g) {        // tokens and groups outside the checkpoint have zero codes
            const uint32_t at = kb * (S::kHalves * kTcHalf) + h * kTcHalf + token;
            to[h][g] = kb < k1 && at < p.len && group + g < p.scales_ld ? scales[static_cast<int64_t>(at) * p.scales_ld + g] : 0u;
          }
      };
      const uint32_t mine = k0 + ((it ^ team) & 1u);      // the team's first stage of this tile
#pragma unroll
      for (uint32_t d = 0; d < kAhead; ++d) fetch(mine + 2u * d, bytes[d]);
      for (uint32_t kb0 = mine; ok && kb0 < k1; kb0 += 2u * kAhead) {
#pragma unroll
        for (uint32_t d = 0; d < kAhead; ++d) {
          const uint32_t kb = kb0 + 2u * d;
          if (kb >= k1) break;
          const uint32_t n = it + (kb - k0), s = n % kStages;
          if (!bar_wait(smem_addr(&codes_full[s]), (n / kStages) & 1u, p.wait_limit)) { ok = false; break; }
          const uint32_t halves = S::kHalves == 1u || kb * (S::kHalves * kTcHalf) + kTcHalf >= p.len ? 1u : 2u;
#pragma unroll
          for (uint32_t h = 0; h < S::kHalves; ++h) {
            if (h >= halves) break;
            const uint32_t b = smem_addr(smem) + s * S::kStage + h * S::kHalf + kTcABytes;
            if (p.x_format == GWS_ACT8_INT8) convert_codes<GWS_ACT8_INT8, S::kBRows>(b + S::kBBytes, b, token, side, bytes[d][h]);
            else convert_codes<GWS_ACT8_E4M3, S::kBRows>(b + S::kBBytes, b, token, side, bytes[d][h]);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // the tensor cores read shared memory through the async proxy
          __syncwarp();
          if (lane == 0) bar_arrive(CG == 2 ? at_rank(smem_addr(&converted[s]), 0u) : smem_addr(&converted[s]));
          fetch(kb + 2u * kAhead, bytes[d]);
        }
      }
      it += k1 - k0;
    }
    if (!ok) failed = 1;
  }
  if (CG == 1 && !kIsGated && p.clustered) {
    // Every block of the cluster adds its share of the tile's rows, the parts in the order of the contraction; a warp takes a row, a
    // lane four columns.
    __syncthreads();
    pair_sync();
    const uint32_t per = (128u + p.splits - 1u) / p.splits, r1 = min(128u, (block_rank() + 1u) * per);
    uint32_t mt, nt, k0, k1;
    place(first, mt, nt, k0, k1);
    const bool second = kIsDw && mt >= p.tiles_per_out;
    const int64_t col = static_cast<int64_t>(nt) * BN + lane * 4u, row0 = static_cast<int64_t>(second ? mt - p.tiles_per_out : mt) * 128;
    uint16_t* out = static_cast<uint16_t*>(p.out[second ? 1 : 0]);
    for (uint32_t r = block_rank() * per + warp; r < r1 && row0 + r < p.rows; r += S::kThreads / 32u) {
      const uint32_t at = smem_addr(smem) + r * kPartRow + lane * 16u;
      float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
      for (uint32_t k = 0; k < p.splits; ++k) {
        float q[4];
        asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(q[0]), "=f"(q[1]), "=f"(q[2]), "=f"(q[3]) : "r"(at_rank(at, k)) : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = k == 0 ? q[i] : v[i] + q[i];
      }
      uint16_t* to = out + (row0 + r) * p.ld_out + col;
      const uint32_t lo = pack_bf16(v[0], v[1]), hi = pack_bf16(v[2], v[3]);
      if (p.wide >= 4 && col + 4 <= p.cols) {
        *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
      } else {
        if (col < p.cols) to[0] = static_cast<uint16_t>(lo);
        if (col + 1 < p.cols) to[1] = static_cast<uint16_t>(lo >> 16);
        if (col + 2 < p.cols) to[2] = static_cast<uint16_t>(hi);
        if (col + 3 < p.cols) to[3] = static_cast<uint16_t>(hi >> 16);
      }
    }
    __syncwarp();
    pair_sync();                         // the other blocks have read this block's part
  }
  __syncthreads();
  if (failed) {                          // copies and products that were started get time to end before the memory is given up
    if (threadIdx.x == 0 && p.status != nullptr) {       // device memory, or pinned host memory that the host reads meanwhile
      *static_cast<volatile int*>(p.status) = 1;
      __threadfence_system();
    }
    const long long t0 = clock64();
    while (clock64() - t0 < kTcLandCycles) {}
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) pair_sync();              // the other block's products read this block's shared memory until here
  __syncwarp();
  if (warp == 2) {
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols) : "memory");
  }
}

// Adds the parts of the cut tiles in order and does with the sums what the epilogue does with a whole tile.  A warp takes 32 columns
// of kJoinRows rows, a lane a column: parts are read, and rows of any alignment written, side by side.
constexpr int kJoinRows = 4;
template <int CG, int BN, int MODE>
__global__ void __launch_bounds__(256) k_join(const __grid_constant__ TcArgs p) {
  after_previous();
  constexpr uint32_t kChunks = MODE == kGated ? BN / 64 : BN / 32, kRuns = 128 * CG / kJoinRows;
  const uint32_t lane = threadIdx.x & 31u, w = blockIdx.x * 8u + (threadIdx.x >> 5);
  const uint32_t tile = w / (kChunks * kRuns), rest = w % (kChunks * kRuns), c = rest % kChunks, r0 = rest / kChunks * kJoinRows;
  if (tile >= p.cut) return;
  uint32_t mt, nt;
  tile_at(p, p.whole + tile, mt, nt);
  const bool second = (MODE == kDw || MODE == kDw8) && mt >= p.tiles_per_out;
  const int64_t row0 = static_cast<int64_t>(second ? mt - p.tiles_per_out : mt) * (128 * CG) + r0;
  const int64_t col0 = static_cast<int64_t>(nt) * (MODE == kGated ? BN / 2 : BN) + c * 32u, col = col0 + lane;
  if (col0 >= p.cols || row0 >= p.rows) return;
  const float* part = p.part + static_cast<int64_t>(tile) * (128 * CG * BN) + r0 * BN + c * 32u + lane;
  const int64_t stride = static_cast<int64_t>(p.cut) * (128 * CG * BN);
  float a[kJoinRows], b[kJoinRows];
#pragma unroll
  for (int i = 0; i < kJoinRows; ++i) {
    a[i] = part[i * BN];
    b[i] = MODE == kGated ? part[i * BN + BN / 2] : 0.0f;
  }
#pragma unroll 4
  for (uint32_t k = 1; k < p.splits; ++k) {
    const float* q = part + k * stride;
#pragma unroll
    for (int i = 0; i < kJoinRows; ++i) {
      a[i] += q[i * BN];
      if (MODE == kGated) b[i] += q[i * BN + BN / 2];
    }
  }
#pragma unroll
  for (int i = 0; i < kJoinRows; ++i) {
    const int64_t row = row0 + i;
    if (row >= p.rows) break;
    float v = a[i];
    if (MODE == kGated) {
      const float act = p.activation == GWS_GATED_SILU ? act_of<GWS_GATED_SILU>(a[i])
                        : p.activation == GWS_GATED_GELU_TANH ? act_of<GWS_GATED_GELU_TANH>(a[i]) : act_of<GWS_GATED_RELU>(a[i]);
      v = act * b[i];
    }
    if (col < p.cols) static_cast<uint16_t*>(p.out[second ? 1 : 0])[row * p.ld_out + col] = static_cast<uint16_t>(pack_bf16(v, 0.0f));
    if (MODE == kGated && p.save != GWS_SAVE_NONE) {
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        const float x = which == 0 ? a[i] : b[i];
        if (p.save == GWS_SAVE_BF16) {
          if (col < p.cols) p.save16[which][row * p.cols + col] = static_cast<uint16_t>(pack_bf16(x, 0.0f));
          continue;
        }
        const Act8View& o = p.save8[which];
        const uint32_t byte = scale_byte(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x) & 0x7FFFFFFFu), p.save);
        const float inv = inverse_scale_of(byte);
        const uint32_t code = byte == kNanByte ? 0u : p.save == GWS_ACT8_INT8 ? encode4_int8(x, 0.0f, 0.0f, 0.0f, inv) : encode4_e4m3(x, 0.0f, 0.0f, 0.0f, inv);
        o.codes[row * o.ld + col] = static_cast<uint8_t>(code);
        if (lane == 0) o.scales[row * (o.ld >> 5) + (col0 >> 5)] = static_cast<uint8_t>(byte);
      }
    }
  }
}

// ---- the element-wise part of the backward pass ------------------------------------------------------------------------------
// From dh and the saved g, u:  dg = dh u act'(g),  du = dh act(g),  and h = act(g) u for the next layer's weight gradient.  dg and du are
// rounded to BF16 because the tensor cores take them in that form; their sums dx and dW are FP32 again.  What that costs: the error of
// the gradients against 64 bits is 2.3e-3 of their norm instead of the 1.65e-3 of their own rounding.
// The first blocks of the launch make ready what the products after it read (prepare).
struct PreArgs {
  const uint16_t* grad_h;
  int64_t ld_grad_h;
  Act8View save8[2];
  const uint16_t* save16[2];
  uint16_t *grad_gate, *grad_up;
  int64_t ld;                      // of grad_gate and grad_up
  uint16_t* h;                     // may be null, [rows, cols]
  int64_t rows, cols, groups;      // groups: rows * ceil(cols / 32)
  uint32_t per_row;
};

// Memory-bound, one pass: 2 + 2 (1 + 1/32) bytes in, 4 or 6 bytes out per element.  A thread takes a group of 32 columns, so that a
// scale is read once.  16384 x 5632 from INT8, with h: 135 us, 6.9 TB/s of 10.06 bytes per element.
template <int SAVE, int ACT>
__global__ void __launch_bounds__(256) k_gated_pre(const __grid_constant__ PreArgs p, const __grid_constant__ Prep m) {
  after_previous();
  if (prepare(m)) return;
  const int64_t t = static_cast<int64_t>(blockIdx.x - m.move_blocks - m.restore_blocks) * 256 + threadIdx.x;
  if (t >= p.groups) return;
  const int64_t at = t * kGroup;     // saved values and h: rows side by side
  int64_t at_dh = at, at_out = at;
  if (p.ld_grad_h != p.cols || p.ld != p.cols) {
    const int64_t row = quotient(t, p.per_row);
    at_dh += row * (p.ld_grad_h - p.cols);
    at_out += row * (p.ld - p.cols);
  }
  V8 cg, cu;
  float ug = 0.0f, uu = 0.0f;
  if (SAVE != GWS_SAVE_BF16) {
    cg = ld32(p.save8[0].codes + at);
    cu = ld32(p.save8[1].codes + at);
    ug = unit_of<SAVE>(p.save8[0].scales[t]);
    uu = unit_of<SAVE>(p.save8[1].scales[t]);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {      // 16 columns at a time
    const V8 dh = ld32(p.grad_h + at_dh + 16 * q);
    float g[16], u[16];
    if (SAVE == GWS_SAVE_BF16) {
      const V8 a = ld32(p.save16[0] + at + 16 * q), b = ld32(p.save16[1] + at + 16 * q);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g[2 * i] = bf16_lo(a.x[i]); g[2 * i + 1] = bf16_hi(a.x[i]);
        u[2 * i] = bf16_lo(b.x[i]); u[2 * i + 1] = bf16_hi(b.x[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        decode4<SAVE>(cg.x[4 * q + i], ug, g + 4 * i);
        decode4<SAVE>(cu.x[4 * q + i], uu, u + 4 * i);
      }
    }
    V8 dg, du, h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a[2], d1[2], d2[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float grad = e == 0 ? bf16_lo(dh.x[i]) : bf16_hi(dh.x[i]);
        float act, slope;
        act_and_slope<ACT>(g[2 * i + e], act, slope);
        d1[e] = grad * u[2 * i + e] * slope;
        d2[e] = grad * act;
        a[e] = act * u[2 * i + e];
      }
      dg.x[i] = pack_bf16(d1[0], d1[1]);
      du.x[i] = pack_bf16(d2[0], d2[1]);
      h.x[i] = pack_bf16(a[0], a[1]);
    }
    st32(p.grad_gate + at_out + 16 * q, dg);
    st32(p.grad_up + at_out + 16 * q, du);
    if (p.h != nullptr) st32(p.h + at + 16 * q, h);
  }
}

// Any width, stride and alignment of grad_h, of kept BF16 values and of h: a warp takes a run of 256 columns of a row, a lane eight
// neighbouring ones.  What may lie at odd addresses is read and written one element at a time, side by side, and turned into the lanes'
// eight elements, or back, in shared memory: 2047 x 2729 from INT8 with h in 13 us (4.3 TB/s), with an element of each group to a lane
// 23 us.
template <int SAVE, int ACT>
__global__ void __launch_bounds__(256) k_gated_pre_any(const __grid_constant__ PreArgs p, const __grid_constant__ Prep m) {
  after_previous();
  if (prepare(m)) return;
  __shared__ uint4 turn[8][32];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, runs_per_row = (p.per_row + 7u) / 8u;
  const int64_t t = static_cast<int64_t>(blockIdx.x - m.move_blocks - m.restore_blocks) * 8 + warp, row = quotient(t, runs_per_row);
  if (row >= p.rows) return;
  const int64_t run = (t - row * runs_per_row) * 256, col = run + lane * 8;
  uint16_t* side = reinterpret_cast<uint16_t*>(turn[warp]) + lane;
  const bool real = col < static_cast<int64_t>(p.per_row) * kGroup;        // inside the padded width of checkpoints and results
  auto bring = [&](const uint16_t* from) {                                 // this lane's eight elements of a row of any alignment
    from += run + lane;
    uint16_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = run + lane + 32 * i < p.cols ? from[32 * i] : static_cast<uint16_t>(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) side[32 * i] = v[i];
    __syncwarp();
    const uint4 w = turn[warp][lane];
    __syncwarp();
    return w;
  };
  uint2 cg = make_uint2(0u, 0u), cu = cg;
  uint32_t bg = 0u, bu = 0u;
  if (SAVE != GWS_SAVE_BF16 && real) {
    const int64_t at = row * p.per_row * kGroup + col;
    cg = *reinterpret_cast<const uint2*>(p.save8[0].codes + at);
    cu = *reinterpret_cast<const uint2*>(p.save8[1].codes + at);
    bg = p.save8[0].scales[at >> 5];
    bu = p.save8[1].scales[at >> 5];
  }
  float g[8], u[8];
  if (SAVE == GWS_SAVE_BF16) {
    const uint4 a = bring(p.save16[0] + row * p.cols), b = bring(p.save16[1] + row * p.cols);
    const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g[2 * i] = bf16_lo(wa[i]); g[2 * i + 1] = bf16_hi(wa[i]);
      u[2 * i] = bf16_lo(wb[i]); u[2 * i + 1] = bf16_hi(wb[i]);
    }
  } else {
    const float ug = unit_of<SAVE>(bg), uu = unit_of<SAVE>(bu);
    decode4<SAVE>(cg.x, ug, g); decode4<SAVE>(cg.y, ug, g + 4);
    decode4<SAVE>(cu.x, uu, u); decode4<SAVE>(cu.y, uu, u + 4);
  }
  const uint4 d = bring(p.grad_h + row * p.ld_grad_h);
  const uint32_t dh[4] = {d.x, d.y, d.z, d.w};
  uint32_t dg[4], du[4], h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a[2], d1[2], d2[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float grad = e == 0 ? bf16_lo(dh[i]) : bf16_hi(dh[i]);
      float act, slope;
      act_and_slope<ACT>(g[2 * i + e], act, slope);
      d1[e] = grad * u[2 * i + e] * slope;
      d2[e] = grad * act;
      a[e] = act * u[2 * i + e];
    }
    dg[i] = pack_bf16(d1[0], d1[1]);
    du[i] = pack_bf16(d2[0], d2[1]);
    h[i] = pack_bf16(a[0], a[1]);
  }
  if (real) {
    *reinterpret_cast<uint4*>(p.grad_gate + row * p.ld + col) = make_uint4(dg[0], dg[1], dg[2], dg[3]);
    *reinterpret_cast<uint4*>(p.grad_up + row * p.ld + col) = make_uint4(du[0], du[1], du[2], du[3]);
  }
  if (p.h != nullptr) {
    turn[warp][lane] = make_uint4(h[0], h[1], h[2], h[3]);
    __syncwarp();
    uint16_t* to = p.h + row * p.cols + run + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (run + lane + 32 * i < p.cols) to[32 * i] = side[32 * i];
  }
}

}  // namespace
