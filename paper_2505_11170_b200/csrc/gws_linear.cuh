// The element-wise part of the backward pass of a linear layer with epilogue:
//
//   dz = dy act'(z)  (BF16: the form in which the tensor cores take it)      db = sum_rows dz  (of the FP32 values)      act(z) once more
//
// Memory-bound, one pass: 2 + 1 1/32 bytes in (z from a checkpoint), 2 or 4 out per element.  A block takes a strip of 64 columns of a share of the rows, eight lanes to
// a row and eight columns to a lane, has the next rows' loads under way while it works on some, and keeps the column sums in registers.  The shares of a strip, where they
// are eight at most, are the blocks of a cluster and joined through each other's shared memory in a fixed order; more of them leave their sums to k_column_sums.
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

// act(z) and its slope of eight elements, as act_and_slope in gws_tc.cuh, two at a time.
template <int ACT>
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
      zz = two(fminf(first_of(z[i]) * first_of(z[i]), 0x1p100f), fminf(second_of(z[i]) * second_of(z[i]), 0x1p100f));
      x = mul2(z[i], fma2(zz, both(-kLog2e * kGeluLin * 0.044715f), both(-kLog2e * kGeluLin)));
    }
    float e0, e1, s0, s1;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(first_of(x)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(second_of(x)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s0) : "f"(1.0f + e0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s1) : "f"(1.0f + e1));
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
__global__ void __launch_bounds__(kPreThreads) k_linear_pre(const __grid_constant__ LinearPre p, const __grid_constant__ Prep m) {
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
  const uint16_t* const dy0 = p.dy != nullptr ? p.dy + begin * p.ld_dy : nullptr;
  const uint16_t* const z0 = SAVE == GWS_SAVE_BF16 ? p.save16 + begin * p.cols : nullptr;
  const bool mine = col < p.cols, coded = kIs8 && col < p.save8.ld;
  auto bring = [&](const uint16_t* base, int64_t ld, int32_t row) {           // eight elements of a row, zeros outside
    if constexpr (WIDE) return row < rows && mine ? __ldg(reinterpret_cast<const uint4*>(base + row * ld + col)) : make_uint4(0u, 0u, 0u, 0u);
    const int32_t row0 = row - static_cast<int32_t>(lane >> 3);
    uint16_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int32_t r = row0 + i / 2;
      const int64_t c = col0 + (i & 1) * 32 + lane;
      v[i] = r < rows && c < p.cols ? base[r * ld + c] : static_cast<uint16_t>(0);
    }
    uint16_t* side = reinterpret_cast<uint16_t*>(turn[WIDE ? 0 : warp]) + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) side[32 * i] = v[i];
    __syncwarp();
    const uint4 w = turn[WIDE ? 0 : warp][lane];
    __syncwarp();
    return w;
  };
  struct Raw {
    uint4 g, z16;
    uint2 z8;
    uint32_t byte;
  };
  auto fetch = [&](int32_t row, Raw& r) {
    if (dy0 != nullptr) r.g = bring(dy0, p.ld_dy, row);
    if (SAVE == GWS_SAVE_BF16) r.z16 = bring(z0, p.cols, row);
    if (kIs8) {
      const bool real = row < rows && coded;
      const int64_t at = (begin + row) * p.save8.ld + col;
      r.z8 = real ? __ldg(reinterpret_cast<const uint2*>(p.save8.codes + at)) : make_uint2(0u, 0u);
      r.byte = real ? p.save8.scales[at >> 5] : 0u;
    }
  };
  F2 db[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) db[i] = both(0.0f);
  constexpr int kRows = WIDE ? 3 : 1;                                          // rows of a thread under way
  Raw next[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) fetch(static_cast<int32_t>(slot + kPreSlots * k), next[k]);
#pragma unroll 1
  for (int32_t at = 0; at < rows; at += kPreSlots * kRows) {
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int32_t row = at + static_cast<int32_t>(slot + kPreSlots * k);
      const Raw now = next[k];
      fetch(row + static_cast<int32_t>(kPreSlots * kRows), next[k]);
      F2 z[4], a[4], slope[4];
      if (SAVE == GWS_SAVE_BF16) {
        const uint32_t q[4] = {now.z16.x, now.z16.y, now.z16.z, now.z16.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = two(bf16_lo(q[i]), bf16_hi(q[i]));
      } else if (kIs8) {
        decode8<kFmt>(now.z8, unit_of<kFmt>(now.byte), z);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = both(0.0f);
      }
      slopes<ACT>(z, a, slope);
      uint32_t w[4];
      if (dy0 != nullptr) {
        const uint32_t q[4] = {now.g.x, now.g.y, now.g.z, now.g.w};
        // an element outside has dy = 0; its z may be a NaN (the group's), which must not reach the sum
        const bool whole = WIDE ? row < rows && mine : row < rows && col + 8 <= p.cols;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          F2 d = mul2(two(bf16_lo(q[i]), bf16_hi(q[i])), slope[i]);
          if (!WIDE && !whole) d = two(row < rows && col + 2 * i < p.cols ? first_of(d) : 0.0f, row < rows && col + 2 * i + 1 < p.cols ? second_of(d) : 0.0f);
          if (!WIDE || whole) db[i] = fma2(d, both(1.0f), db[i]);
          w[i] = pack_bf16(first_of(d), second_of(d));
        }
        if (p.dz != nullptr && row < rows && (!WIDE || mine)) *reinterpret_cast<uint4*>(p.dz + (begin + row) * p.ld_dz + col) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      if (p.again != nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(first_of(a[i]), second_of(a[i]));
        if constexpr (WIDE) {
          if (row < rows && mine) *reinterpret_cast<uint4*>(p.again + (begin + row) * p.cols + col) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
          turn[WIDE ? 0 : warp][lane] = make_uint4(w[0], w[1], w[2], w[3]);
          __syncwarp();
          const uint16_t* side = reinterpret_cast<const uint16_t*>(turn[WIDE ? 0 : warp]) + lane;
          const int32_t row0 = row - static_cast<int32_t>(lane >> 3);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int32_t r = row0 + i / 2;
            const int64_t c = col0 + (i & 1) * 32 + lane;
            if (r < rows && c < p.cols) p.again[(begin + r) * p.cols + c] = side[32 * i];
          }
          __syncwarp();
        }
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

}  // namespace
