// The element-wise part of the backward pass of a linear layer with epilogue:
//
//   dz = dy act'(z)  (BF16: the form in which the tensor cores take it)      db = sum_rows dz  (of the FP32 values)      act(z) once more
//
// Memory-bound, one pass: 2 + 1 1/32 bytes in (z from a checkpoint), 2 or 4 out per element.  A block takes a strip of 64 columns of a share of the rows, eight lanes to
// a row and eight columns to a lane, has the next rows' loads under way while it works on some, and keeps the column sums in registers.  The shares of a strip, where they
// are eight at most, are the blocks of a cluster and joined through each other's shared memory in a fixed order; more of them leave their sums to k_column_sums.
// 16384 x 5632, GELU from INT8, us of a call that wants no product, so that dz is not written: act(z) and db 89 (5.2 TB/s of 464 MB, the join of the sums among it), act(z) alone
// 75, db alone 80.  With dz too, a call with a narrow product less that product: 152 to 158 (4.2 TB/s of 649 MB).
// Odd widths read and write elements one by one: 2047 x 2729, act(z) and db 17 us, 8192 x 2729 50 (2.3 TB/s), with dz 57 to 60.
// The first blocks of the launch make ready what the products after it read (prepare).
#pragma once
#include <stdint.h>

#include "gws_pair.cuh"
#include "gws_sums.cuh"
#include "gws_tc.cuh"

namespace {

struct LinearPre {
  const uint16_t* dy;
  int64_t ld_dy;
  Act8View save8;
  const uint16_t* save16;          // [rows, cols]
  uint16_t* dz;                    // null where dz is dy
  int64_t ld_dz;
  uint16_t* again;                 // act(z), [rows, cols]; may be null
  void* db;                        // may be null
  float* part;                     // [shares, cols]: where the shares are no cluster
  int64_t rows, cols;
  uint32_t first;                  // blocks that prepare
  uint32_t shares;                 // blocks of a strip
  int32_t db_f32;
};

// act(z) and its slope of eight elements, as act_and_slope in gws_tc.cuh, two at a time.  FAR: z^2 may pass FP32.
template <int ACT, bool FAR>
__device__ __forceinline__ void slopes(const F2 (&z)[4], F2 (&a)[4], F2 (&slope)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (ACT == GWS_ACT_NONE || ACT == GWS_GATED_RELU) {
      const float x = first_of(z[i]), y = second_of(z[i]);
      float ax, ay, sx, sy;
      act_and_slope<ACT>(x, ax, sx);
      act_and_slope<ACT>(y, ay, sy);
      a[i] = two(ax, ay);
      slope[i] = two(sx, sy);
      continue;
    }
    constexpr float kLog2e = 1.44269504f;
    F2 zz = z[i], x = mul2(z[i], both(-kLog2e));
    if (ACT == GWS_GATED_GELU_TANH) {
      zz = mul2(z[i], z[i]);
      if (FAR) zz = two(fminf(first_of(zz), 0x1p100f), fminf(second_of(zz), 0x1p100f));
      x = mul2(z[i], fma2(zz, both(-kLog2e * kGeluLin * 0.044715f), both(-kLog2e * kGeluLin)));
    }
    float e0, e1, s0, s1;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(first_of(x)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(second_of(x)));
    const F2 d = fma2(two(e0, e1), both(1.0f), both(1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s0) : "f"(first_of(d)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s1) : "f"(second_of(d)));
    const F2 s = two(s0, s1);
    a[i] = mul2(z[i], s);
    F2 t = mul2(a[i], fma2(s, both(-1.0f), both(1.0f)));
    if (ACT == GWS_GATED_GELU_TANH) t = mul2(t, fma2(zz, both(3.0f * 0.044715f * kGeluLin), both(kGeluLin)));
    slope[i] = fma2(t, both(1.0f), s);
  }
}
// z of a thread's eight codes.
template <int FMT>
__device__ __forceinline__ void decode8(uint2 c, float unit, F2 (&z)[4]) {
  float v[8];
  if (FMT == GWS_ACT8_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = (i < 2 ? c.x : c.y) ^ 0x80808080u;        // as decode4_int8
      const F2 q = two(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540u + 2 * (i & 1))), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7541u + 2 * (i & 1))));
      z[i] = mul2(fma2(q, both(1.0f), both(-8388736.0f)), both(unit));
    }
    return;
  }
  decode4<FMT>(c.x, unit, v);
  decode4<FMT>(c.y, unit, v + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = two(v[2 * i], v[2 * i + 1]);
}

constexpr uint32_t kPreThreads = 128u, kPreSlots = kPreThreads / 8u;

// WIDE: rows of dy, of a BF16 z and of act(z) on 16-byte boundaries.  Otherwise a warp reads its four rows an element to a lane, side by side, and turns them in
// shared memory.
template <int SAVE, int ACT, bool WIDE>
__global__ void __launch_bounds__(kPreThreads, 6) k_linear_pre(const __grid_constant__ LinearPre p, const __grid_constant__ Prep m) {
  after_previous();
  if (blockIdx.x < p.first) {
    (void)prepare(m, threadIdx.x);
    (void)prepare(m, threadIdx.x + kPreThreads);
    return;
  }
  constexpr bool kIs8 = SAVE == GWS_ACT8_INT8 || SAVE == GWS_ACT8_E4M3;
  constexpr int kFmt = SAVE == GWS_ACT8_INT8 ? GWS_ACT8_INT8 : GWS_ACT8_E4M3;
  __shared__ uint4 turn[WIDE ? 1 : kPreThreads / 32u][32];
  __shared__ __align__(16) float sums[kPreSlots][68];
  __shared__ float joined[64];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, oct = threadIdx.x & 7u, slot = threadIdx.x >> 3;
  const uint32_t b = blockIdx.x - p.first, strip = b / p.shares, share = b - strip * p.shares;
  const int64_t col0 = static_cast<int64_t>(strip) * 64, col = col0 + oct * 8;
  const int64_t per = (p.rows + p.shares - 1) / p.shares, begin = min(p.rows, share * per);
  const int32_t rows = static_cast<int32_t>(min(p.rows, begin + per) - begin);            // of this share
  const bool has_dy = p.dy != nullptr;
  F2 db[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) db[i] = both(0.0f);
  struct Raw {
    uint4 g, z16;
    uint2 z8;
    uint32_t byte;
  };
  auto element_wise = [&](const Raw& r, F2 (&a)[4], F2 (&slope)[4]) {
    F2 z[4];
    if constexpr (kIs8) {
      const float unit = unit_of<kFmt>(r.byte);
      decode8<kFmt>(r.z8, unit, z);
      if (unit <= 0x1p40f) slopes<ACT, false>(z, a, slope);
      else slopes<ACT, true>(z, a, slope);
    } else {
      const uint32_t q[4] = {r.z16.x, r.z16.y, r.z16.z, r.z16.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = SAVE == GWS_SAVE_BF16 ? two(bf16_lo(q[i]), bf16_hi(q[i])) : both(0.0f);
      slopes<ACT, true>(z, a, slope);
    }
  };
  auto packed = [](const F2 (&v)[4]) {
    return make_uint4(pack_bf16(first_of(v[0]), second_of(v[0])), pack_bf16(first_of(v[1]), second_of(v[1])), pack_bf16(first_of(v[2]), second_of(v[2])),
                      pack_bf16(first_of(v[3]), second_of(v[3])));
  };
  if constexpr (WIDE) {
    // Rows slot, slot + 16, ... of the share; every stream's address moves on by 16 rows.
    constexpr int kRows = 3;                               // of a thread, under way
    const int32_t mine = col < p.cols && rows > static_cast<int32_t>(slot) ? (rows - static_cast<int32_t>(slot) + static_cast<int32_t>(kPreSlots) - 1) / static_cast<int32_t>(kPreSlots) : 0;
    const int64_t row0 = begin + slot;
    const uint16_t* dy = p.dy + row0 * p.ld_dy + col;
    const uint16_t* z16 = p.save16 + row0 * p.cols + col;
    const uint8_t* z8 = p.save8.codes + row0 * p.save8.ld + col;
    const uint8_t* byte = p.save8.scales + row0 * (p.save8.ld >> 5) + (col >> 5);
    uint16_t* dz = p.dz + row0 * p.ld_dz + col;
    uint16_t* again = p.again + row0 * p.cols + col;
    const int64_t to_dy = p.ld_dy * kPreSlots, to_z = p.cols * kPreSlots, to_z8 = p.save8.ld * kPreSlots, to_byte = (p.save8.ld >> 5) * kPreSlots, to_dz = p.ld_dz * kPreSlots;
    auto fetch = [&](Raw& r) {
      if (has_dy) {
        r.g = __ldg(reinterpret_cast<const uint4*>(dy));
        dy += to_dy;
      }
      if (SAVE == GWS_SAVE_BF16) {
        r.z16 = __ldg(reinterpret_cast<const uint4*>(z16));
        z16 += to_z;
      }
      if (kIs8) {
        r.z8 = __ldg(reinterpret_cast<const uint2*>(z8));
        r.byte = __ldg(byte);
        z8 += to_z8;
        byte += to_byte;
      }
    };
    Raw next[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k < mine) fetch(next[k]);
#pragma unroll 1
    for (int32_t j = 0; j < mine; j += kRows) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        if (j + k >= mine) break;
        const Raw now = next[k];
        if (j + k + kRows < mine) fetch(next[k]);
        F2 a[4], slope[4];
        element_wise(now, a, slope);
        if (has_dy) {
          const uint32_t q[4] = {now.g.x, now.g.y, now.g.z, now.g.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            slope[i] = mul2(two(bf16_lo(q[i]), bf16_hi(q[i])), slope[i]);
            db[i] = fma2(slope[i], both(1.0f), db[i]);
          }
          if (p.dz != nullptr) {
            *reinterpret_cast<uint4*>(dz) = packed(slope);
            dz += to_dz;
          }
        }
        if (p.again != nullptr) {
          *reinterpret_cast<uint4*>(again) = packed(a);
          again += to_z;
        }
      }
    }
  } else {
    const uint16_t* const dy0 = has_dy ? p.dy + begin * p.ld_dy : nullptr;
    const uint16_t* const z0 = SAVE == GWS_SAVE_BF16 ? p.save16 + begin * p.cols : nullptr;
    const int32_t sub = static_cast<int32_t>(lane >> 3);
    uint16_t* const side = reinterpret_cast<uint16_t*>(turn[WIDE ? 0 : warp]) + lane;
    auto load = [&](const uint16_t* base, int64_t ld, int32_t row, uint16_t (&v)[8]) {        // neighbouring elements of the warp's four rows, zeros outside
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int32_t r = row - sub + i / 2;
        const int64_t c = col0 + (i & 1) * 32 + lane;
        v[i] = r < rows && c < p.cols ? base[r * ld + c] : static_cast<uint16_t>(0);
      }
    };
    auto own = [&](const uint16_t (&v)[8]) {                                                  // this lane's eight
#pragma unroll
      for (int i = 0; i < 8; ++i) side[32 * i] = v[i];
      __syncwarp();
      const uint4 w = turn[WIDE ? 0 : warp][lane];
      __syncwarp();
      return w;
    };
    uint16_t vg[8], vz[8];
    uint2 z8 = make_uint2(0u, 0u);
    uint32_t byte = 0u;
    auto fetch = [&](int32_t row) {
      if (has_dy) load(dy0, p.ld_dy, row, vg);
      if (SAVE == GWS_SAVE_BF16) load(z0, p.cols, row, vz);
      if (kIs8) {
        const bool real = row < rows && col < p.save8.ld;
        const int64_t from = (begin + row) * p.save8.ld + col;
        z8 = real ? __ldg(reinterpret_cast<const uint2*>(p.save8.codes + from)) : make_uint2(0u, 0u);
        byte = real ? p.save8.scales[from >> 5] : 0u;
      }
    };
    fetch(static_cast<int32_t>(slot));
#pragma unroll 1
    for (int32_t at = 0; at < rows; at += kPreSlots) {
      const int32_t row = at + static_cast<int32_t>(slot);
      Raw r;
      r.z8 = z8;
      r.byte = byte;
      if (has_dy) r.g = own(vg);
      if (SAVE == GWS_SAVE_BF16) r.z16 = own(vz);
      if (at + static_cast<int32_t>(kPreSlots) < rows) fetch(row + static_cast<int32_t>(kPreSlots));
      F2 a[4], slope[4];
      element_wise(r, a, slope);
      if (has_dy) {
        const uint32_t q[4] = {r.g.x, r.g.y, r.g.z, r.g.w};
        // an element outside has dy = 0; its z may be a NaN (the group's), which must not reach the sum
        const bool whole = row < rows && col + 8 <= p.cols;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          F2 d = mul2(two(bf16_lo(q[i]), bf16_hi(q[i])), slope[i]);
          if (!whole) d = two(row < rows && col + 2 * i < p.cols ? first_of(d) : 0.0f, row < rows && col + 2 * i + 1 < p.cols ? second_of(d) : 0.0f);
          db[i] = fma2(d, both(1.0f), db[i]);
          slope[i] = d;
        }
        if (p.dz != nullptr && row < rows) *reinterpret_cast<uint4*>(p.dz + (begin + row) * p.ld_dz + col) = packed(slope);
      }
      if (p.again != nullptr) {
        turn[WIDE ? 0 : warp][lane] = packed(a);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int32_t to = row - sub + i / 2;
          const int64_t c = col0 + (i & 1) * 32 + lane;
          if (to < rows && c < p.cols) p.again[(begin + to) * p.cols + c] = side[32 * i];
        }
        __syncwarp();
      }
    }
  }
  if (p.db == nullptr) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) *reinterpret_cast<float4*>(&sums[slot][oct * 8u + 4u * i]) = make_float4(first_of(db[2 * i]), second_of(db[2 * i]), first_of(db[2 * i + 1]), second_of(db[2 * i + 1]));
  __syncthreads();
  if (threadIdx.x < 64u) {
    float t = 0.0f;
#pragma unroll 8
    for (uint32_t r = 0; r < kPreSlots; ++r) t += sums[r][threadIdx.x];
    joined[threadIdx.x] = t;
  }
  if (p.part != nullptr) {
    if (threadIdx.x < 64u && col0 + threadIdx.x < p.cols) p.part[share * p.cols + col0 + threadIdx.x] = joined[threadIdx.x];
    return;
  }
  if (p.shares > 1u) pair_sync();
  if (share == 0u && threadIdx.x < 64u && col0 + threadIdx.x < p.cols) {
    float t = joined[threadIdx.x];
    for (uint32_t r = 1; r < p.shares; ++r) {
      float q;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(q) : "r"(at_rank(smem_addr(&joined[threadIdx.x]), r)) : "memory");
      t += q;
    }
    if (p.db_f32 != 0) static_cast<float*>(p.db)[col0 + threadIdx.x] = t;
    else static_cast<uint16_t*>(p.db)[col0 + threadIdx.x] = static_cast<uint16_t>(pack_bf16(t, 0.0f));
  }
  if (p.shares > 1u) pair_sync();              // rank 0 has read this block's sums
}

// ---- forward pass of a few tokens ------------------------------------------------------------------------------------------------
// y of up to four tokens without tensor cores: a warp, or SPLIT of them together, streams R rows of W, 16 bytes to a lane at a time, and multiplies them with every token's x, which stays in L1.  One token,
// 2048 x 5632: all of W (23 MB) is under way at once, and what is left is memory and a launch.  Sums are FP32, each lane's over every 256th octet, then over the lanes.
struct LinearRow {
  const uint16_t *x, *w, *residual;
  const void* bias;
  uint16_t *y, *save16;
  Act8View save8;
  int64_t ld_x, ld_w, ld_y, ld_residual, cols;
  uint32_t octets;                 // of a row
  int32_t tokens, activation, save, bias_f32;
};

// a + b c of both numbers of two pairs, in FP32; the product of two BF16 numbers is exact.
__device__ __forceinline__ float fma_pair(uint32_t b, uint32_t c, float a) {
  asm("{\n\t.reg .b16 bl, bh, cl, ch;\n\tmov.b32 {bl, bh}, %1;\n\tmov.b32 {cl, ch}, %2;\n\tfma.rn.f32.bf16 %0, bl, cl, %0;\n\tfma.rn.f32.bf16 %0, bh, ch, %0;\n\t}" : "+f"(a) : "r"(b), "r"(c));
  return a;
}

template <int M, int R, int SPLIT>
__global__ void __launch_bounds__(256) k_linear_row(const __grid_constant__ LinearRow p) {
  after_previous();
  constexpr int kAhead = R == 1 ? 8 : 4;                                // octets of a lane and row under way
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  constexpr uint32_t rows = 8u / SPLIT * R, step = 32u * SPLIT;         // rows of a block; octets between two of a lane's
  const uint32_t part = warp % SPLIT, first = warp / SPLIT * R;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows + first;
  float sum[M][R];
#pragma unroll
  for (int t = 0; t < M; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) sum[t][r] = 0.0f;
  const uint4* w[R];
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = reinterpret_cast<const uint4*>(p.w + min(row0 + r, p.cols - 1) * p.ld_w) + part * 32u + lane;
  const uint4* x = reinterpret_cast<const uint4*>(p.x) + part * 32u + lane;
#pragma unroll 1
  for (uint32_t at = part * 32u + lane; at < p.octets; at += step * kAhead) {
    uint4 q[R][kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int r = 0; r < R; ++r) q[r][i] = at + step * i < p.octets ? __ldg(w[r] + step * i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (at + step * i >= p.octets) break;
#pragma unroll
      for (int t = 0; t < M; ++t) {
        if (t >= p.tokens) break;
        const uint4 v = __ldg(x + t * (p.ld_x / 8) + step * i);
#pragma unroll
        for (int r = 0; r < R; ++r)
          sum[t][r] = fma_pair(q[r][i].w, v.w, fma_pair(q[r][i].z, v.z, fma_pair(q[r][i].y, v.y, fma_pair(q[r][i].x, v.x, sum[t][r]))));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] += step * kAhead;
    x += step * kAhead;
  }
  __shared__ float z_of[M][8 * R], parts[8][M * R];
  float mine = 0.0f;                                                    // lane t R + r: of token t, row r
#pragma unroll
  for (int t = 0; t < M; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s = sum[t][r];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
      if (lane == static_cast<uint32_t>(t * R + r)) mine = s;
    }
  if (SPLIT > 1) {                                                   // the first warp of a row adds the parts, in their order
    if (lane < static_cast<uint32_t>(M * R)) parts[warp][lane] = mine;
    __syncthreads();
    if (part == 0u && lane < static_cast<uint32_t>(M * R))
      for (uint32_t k = 1; k < SPLIT; ++k) mine += parts[warp + k][lane];
  }
  const uint32_t t = lane / R, r = lane % R;
  const int64_t col = row0 + r;
  const bool real = part == 0u && lane < static_cast<uint32_t>(M * R) && t < static_cast<uint32_t>(p.tokens);
  if (real && col < p.cols) {
    if (p.bias != nullptr)
      mine += p.bias_f32 != 0 ? static_cast<const float*>(p.bias)[col] : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(p.bias)[col]) << 16);
    float y = act_of_kind(p.activation, mine);
    if (p.residual != nullptr) y += __uint_as_float(static_cast<uint32_t>(p.residual[t * p.ld_residual + col]) << 16);
    p.y[t * p.ld_y + col] = static_cast<uint16_t>(pack_bf16(y, 0.0f));
    if (p.save == GWS_SAVE_BF16) p.save16[t * p.cols + col] = static_cast<uint16_t>(pack_bf16(mine, 0.0f));
  }
  if (p.save != GWS_ACT8_INT8 && p.save != GWS_ACT8_E4M3) return;
  // A checkpoint's group of 32 columns is a cluster's: its first block takes a token to a warp, a column to a lane.
  if (real) z_of[t][first + r] = col < p.cols ? mine : 0.0f;
  __syncthreads();
  pair_sync();
  if (block_rank() == 0u && warp < static_cast<uint32_t>(p.tokens)) {
    float z;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(z) : "r"(at_rank(smem_addr(&z_of[warp][lane % rows]), lane / rows)) : "memory");
    const uint32_t byte = scale_byte(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(z) & 0x7FFFFFFFu), p.save);
    const float inv = inverse_scale_of(byte);
    const uint32_t code = byte == kNanByte ? 0u : p.save == GWS_ACT8_INT8 ? encode4_int8(z, 0.0f, 0.0f, 0.0f, inv) : encode4_e4m3(z, 0.0f, 0.0f, 0.0f, inv);
    const int64_t group = blockIdx.x / (32u / rows);
    p.save8.codes[warp * p.save8.ld + group * 32 + lane] = static_cast<uint8_t>(code);
    if (lane == 0u) p.save8.scales[warp * (p.save8.ld >> 5) + group] = static_cast<uint8_t>(byte);
  }
  pair_sync();                                                          // rank 0 has read this block's part
}

}  // namespace
