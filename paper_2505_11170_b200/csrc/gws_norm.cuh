// Layer norm over the rows of a BF16 matrix, forward and backward.
//
//   s = bf16(x + r)  (or x)      mu = mean(s)      rstd = 1 / sqrt(mean((s - mu)^2) + eps)      xh = (s - mu) rstd
//   y = xh gamma + beta
//   a = dy gamma:  ds = rstd (a - mean(a) - xh mean(a xh)) (+ d)      dgamma = sum_rows dy xh      dbeta = sum_rows dy
//
// s is rounded before its statistics are taken, because the backward pass reads it in that form.  The variance is taken from the centred values
// in a second pass over registers: E[s^2] - mu^2 in FP32 loses a row of large mean.  All sums are FP32.
//
// A team of L threads holds a row in registers, C units of eight elements to a thread, so every tensor crosses memory once.  WIDE: rows on 16-byte
// boundaries, a thread takes eight neighbouring elements; otherwise neighbouring threads take neighbouring elements one by one.
// The column sums of the backward pass stay in registers over all rows of a team and are joined in a fixed order: over the teams of a block in shared
// memory, over the blocks by k_column_sums.  Results do not depend on timing.
#pragma once
#include <stdint.h>

#include "gws_act8.cuh"
#include "gws_sums.cuh"

namespace {

struct NormArgs {
  const uint16_t *x, *r;          // forward: input, residual (or null); backward: s
  const uint16_t *dy, *d;         // backward: gradient of y, of s past the norm (or null)
  int64_t ld_x, ld_r, ld_dy, ld_d;
  const void *weight, *bias;      // null: one, zero
  uint16_t *y, *sum;              // dense
  uint16_t* dx;
  float* stats;                   // [2, rows]: mean, rstd
  float* part;                    // backward: [blocks, 2, cols], or null
  int64_t rows, cols;
  float eps;
  int32_t f32;                    // weight and bias are FP32
};

__device__ __forceinline__ float norm_weight(const void* w, bool f32, int64_t col) {
  return f32 ? static_cast<const float*>(w)[col] : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(w)[col]) << 16);
}

// Column of a thread's element 8 c + i.
template <int L, bool WIDE>
__device__ __forceinline__ int64_t norm_col(uint32_t lane, int c, int i) {
  return WIDE ? static_cast<int64_t>(c * L + lane) * 8 + i : static_cast<int64_t>(8 * c + i) * L + lane;
}
// A thread's part of a row as it comes from memory: pairs of neighbouring elements, or one element to a word.
template <int C, bool WIDE>
struct NormWords {
  uint32_t x[WIDE ? 4 * C : 8 * C];
};
template <int L, int C, bool WIDE>
__device__ __forceinline__ void norm_load(const uint16_t* row, int64_t cols, uint32_t lane, NormWords<C, WIDE>& w) {
  if constexpr (WIDE) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = norm_col<L, WIDE>(lane, c, 0);
      const uint4 q = col < cols ? __ldg(reinterpret_cast<const uint4*>(row + col)) : make_uint4(0u, 0u, 0u, 0u);
      w.x[4 * c] = q.x; w.x[4 * c + 1] = q.y; w.x[4 * c + 2] = q.z; w.x[4 * c + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) {
      const int64_t col = norm_col<L, WIDE>(lane, 0, e);
      w.x[e] = col < cols ? static_cast<uint32_t>(__ldg(row + col)) : 0u;
    }
  }
}
template <int C, bool WIDE>
__device__ __forceinline__ float norm_value(const NormWords<C, WIDE>& w, int e) {
  if constexpr (WIDE) return (e & 1) == 0 ? bf16_lo(w.x[e / 2]) : bf16_hi(w.x[e / 2]);
  else return __uint_as_float(w.x[e] << 16);
}
template <int L, int C, bool WIDE>
__device__ __forceinline__ void norm_write(uint16_t* row, int64_t cols, uint32_t lane, const float (&v)[8 * C]) {
  if (WIDE) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = norm_col<L, WIDE>(lane, c, 0);
      if (col < cols)
        *reinterpret_cast<uint4*>(row + col) = make_uint4(pack_bf16(v[8 * c], v[8 * c + 1]), pack_bf16(v[8 * c + 2], v[8 * c + 3]), pack_bf16(v[8 * c + 4], v[8 * c + 5]),
                                                          pack_bf16(v[8 * c + 6], v[8 * c + 7]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) {
      const int64_t col = norm_col<L, WIDE>(lane, 0, e);
      if (col < cols) row[col] = static_cast<uint16_t>(pack_bf16(v[e], 0.0f));
    }
  }
}
// Eight weights (or biases) of unit c.
template <int L, bool WIDE>
__device__ __forceinline__ void norm_weights(const void* w, bool f32, float none, int64_t cols, uint32_t lane, int c, float (&v)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = none;
    return;
  }
  const int64_t col = norm_col<L, WIDE>(lane, c, 0);
  if (WIDE && f32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + col);
    const float4 a = col < cols ? __ldg(p) : make_float4(0, 0, 0, 0), b = col < cols ? __ldg(p + 1) : make_float4(0, 0, 0, 0);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else if (WIDE) {
    const uint4 q = col < cols ? __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + col)) : make_uint4(0u, 0u, 0u, 0u);
    const uint32_t p[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(p[i]); v[2 * i + 1] = bf16_hi(p[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = norm_col<L, WIDE>(lane, c, i) < cols ? norm_weight(w, f32, norm_col<L, WIDE>(lane, c, i)) : 0.0f;
  }
}

// Sums of two values over a team; every thread of the block calls it the same number of times.  `room`: [2][threads / 32], used in turn.
template <int L>
__device__ __forceinline__ float2 team_sum(float a, float b, float2* room, uint32_t& turn) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, d);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, d);
  }
  if (L == 32) return make_float2(a, b);
  constexpr uint32_t kWarps = L / 32;
  float2* mine = room + turn * (blockDim.x / 32u);
  turn ^= 1u;
  if ((threadIdx.x & 31u) == 0u) mine[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  const float2* from = mine + (threadIdx.x / L) * kWarps;
  float2 t = from[0];
#pragma unroll
  for (uint32_t w = 1; w < kWarps; ++w) { t.x += from[w].x; t.y += from[w].y; }
  return t;
}

template <int L>
constexpr uint32_t kNormThreads = L < 256 ? 256u : static_cast<uint32_t>(L);          // of a block

template <int L, int C, bool WIDE>
__global__ void __launch_bounds__(kNormThreads<L>) k_norm_fwd(const __grid_constant__ NormArgs p) {
  after_previous();
  __shared__ float2 room[2][kNormThreads<L> / 32u];
  uint32_t turn = 0;
  const uint32_t lane = threadIdx.x % L;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kNormThreads<L> / L) + threadIdx.x / L;
  if (row >= p.rows) return;               // teams of more than a warp have a block to themselves
  float s[8 * C];
  NormWords<C, WIDE> x;
  norm_load<L, C, WIDE>(p.x + row * p.ld_x, p.cols, lane, x);
  if (p.r != nullptr) {
    NormWords<C, WIDE> r;
    norm_load<L, C, WIDE>(p.r + row * p.ld_r, p.cols, lane, r);
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) s[e] = bf16_lo(pack_bf16(norm_value(x, e) + norm_value(r, e), 0.0f));
    norm_write<L, C, WIDE>(p.sum + row * p.cols, p.cols, lane, s);
  } else {
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) s[e] = norm_value(x, e);
  }
  float t = 0.0f;
#pragma unroll
  for (int e = 0; e < 8 * C; ++e) t += s[e];
  const float inv = 1.0f / static_cast<float>(p.cols), mean = team_sum<L>(t, 0.0f, room[0], turn).x * inv;
  t = 0.0f;
#pragma unroll
  for (int e = 0; e < 8 * C; ++e) {
    s[e] -= mean;
    if (norm_col<L, WIDE>(lane, e / 8, e % 8) < p.cols) t = __fmaf_rn(s[e], s[e], t);
  }
  const float rstd = rsqrtf(team_sum<L>(t, 0.0f, room[0], turn).x * inv + p.eps);
  if (lane == 0 && p.stats != nullptr) {
    p.stats[row] = mean;
    p.stats[p.rows + row] = rstd;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float w[8], b[8];
    norm_weights<L, WIDE>(p.weight, p.f32 != 0, 1.0f, p.cols, lane, c, w);
    norm_weights<L, WIDE>(p.bias, p.f32 != 0, 0.0f, p.cols, lane, c, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[8 * c + i] = __fmaf_rn(s[8 * c + i] * rstd, w[i], b[i]);
  }
  norm_write<L, C, WIDE>(p.y + row * p.cols, p.cols, lane, s);
}

// Rows of any length: a block reads its row again for each pass (from L2).
constexpr uint32_t kNormLong = 1024;
__device__ __forceinline__ float norm_element(const NormArgs& p, int64_t row, int64_t col) {
  const float x = __uint_as_float(static_cast<uint32_t>(p.x[row * p.ld_x + col]) << 16);
  return p.r == nullptr ? x : bf16_lo(pack_bf16(x + __uint_as_float(static_cast<uint32_t>(p.r[row * p.ld_r + col]) << 16), 0.0f));
}
__global__ void __launch_bounds__(kNormLong) k_norm_fwd_long(const __grid_constant__ NormArgs p) {
  after_previous();
  __shared__ float2 room[2][kNormLong / 32u];
  uint32_t turn = 0;
  const int64_t row = blockIdx.x;
  float t = 0.0f;
  for (int64_t col = threadIdx.x; col < p.cols; col += kNormLong) t += norm_element(p, row, col);
  const float inv = 1.0f / static_cast<float>(p.cols), mean = team_sum<kNormLong>(t, 0.0f, room[0], turn).x * inv;
  t = 0.0f;
  for (int64_t col = threadIdx.x; col < p.cols; col += kNormLong) {
    const float v = norm_element(p, row, col) - mean;
    t = __fmaf_rn(v, v, t);
  }
  const float rstd = rsqrtf(team_sum<kNormLong>(t, 0.0f, room[0], turn).x * inv + p.eps);
  if (threadIdx.x == 0 && p.stats != nullptr) {
    p.stats[row] = mean;
    p.stats[p.rows + row] = rstd;
  }
  for (int64_t col = threadIdx.x; col < p.cols; col += kNormLong) {
    const float s = norm_element(p, row, col), w = p.weight != nullptr ? norm_weight(p.weight, p.f32 != 0, col) : 1.0f;
    const float b = p.bias != nullptr ? norm_weight(p.bias, p.f32 != 0, col) : 0.0f;
    if (p.r != nullptr) p.sum[row * p.cols + col] = static_cast<uint16_t>(pack_bf16(s, 0.0f));
    p.y[row * p.cols + col] = static_cast<uint16_t>(pack_bf16(__fmaf_rn((s - mean) * rstd, w, b), 0.0f));
  }
}

template <int L, int C, bool WIDE>
__global__ void __launch_bounds__(kNormThreads<L>) k_norm_bwd(const __grid_constant__ NormArgs p) {
  after_previous();
  constexpr uint32_t kTeams = kNormThreads<L> / L;
  __shared__ float2 room[2][kNormThreads<L> / 32u];
  __shared__ float2 joined[kTeams > 1u ? L * C * 8u : 1u];
  __shared__ float weights[C][8][L];                     // the same for every team: out of the registers, so that the next row's words fit in
  uint32_t turn = 0;
  const uint32_t lane = threadIdx.x % L, team = threadIdx.x / L;
  const float inv = 1.0f / static_cast<float>(p.cols);
  float gw[8 * C], gb[8 * C];
#pragma unroll
  for (int e = 0; e < 8 * C; ++e) gw[e] = gb[e] = 0.0f;
  if (team == 0u) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float q[8];
      norm_weights<L, WIDE>(p.weight, p.f32 != 0, 1.0f, p.cols, lane, c, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) weights[c][i][lane] = q[i];
    }
  }
  __syncthreads();
  struct Row {
    NormWords<C, WIDE> s, dy, d;
    float mean, rstd;
  } next;
  auto fetch = [&](int64_t row, Row& r) {
    const int64_t cols = row < p.rows ? p.cols : 0;
    norm_load<L, C, WIDE>(p.x + row * p.ld_x, cols, lane, r.s);
    norm_load<L, C, WIDE>(p.dy + row * p.ld_dy, cols, lane, r.dy);
    if (p.d != nullptr) norm_load<L, C, WIDE>(p.d + row * p.ld_d, cols, lane, r.d);
    r.mean = row < p.rows ? p.stats[row] : 0.0f;
    r.rstd = row < p.rows ? p.stats[p.rows + row] : 0.0f;
  };
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kTeams;
  int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTeams;
  if (WIDE) fetch(row0 + team, next);
#pragma unroll 1
  for (; row0 < p.rows; row0 += stride) {
    Row now;
    if (WIDE) {
      now = next;
      if (row0 + stride < p.rows) fetch(row0 + stride + team, next);        // under the sums of this one
    } else {
      fetch(row0 + team, now);                                              // an element to a register: there is no room for two rows
    }
    const int64_t row = row0 + team;
    float ta = 0.0f, tb = 0.0f;
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) {
      const float xh = (norm_value(now.s, e) - now.mean) * now.rstd, dy = norm_value(now.dy, e);          // columns past the width have dy = 0
      const float a = dy * weights[e / 8][e % 8][lane];
      ta += a;
      tb = __fmaf_rn(a, xh, tb);
      gw[e] = __fmaf_rn(dy, xh, gw[e]);
      gb[e] += dy;
    }
    const float2 t = team_sum<L>(ta, tb, room[0], turn);
    if (p.dx != nullptr && row < p.rows) {
      const float ma = t.x * inv, mb = t.y * inv;
      float out[8 * C];
#pragma unroll
      for (int e = 0; e < 8 * C; ++e) {
        const float xh = (norm_value(now.s, e) - now.mean) * now.rstd, a = norm_value(now.dy, e) * weights[e / 8][e % 8][lane];
        out[e] = now.rstd * __fmaf_rn(-xh, mb, a - ma);
        if (p.d != nullptr) out[e] += norm_value(now.d, e);
      }
      norm_write<L, C, WIDE>(p.dx + row * p.cols, p.cols, lane, out);
    }
  }
  if (p.part == nullptr) return;
  if (kTeams > 1u) {
    for (uint32_t t = 0; t < kTeams; ++t) {
      if (team == t) {
#pragma unroll
        for (int e = 0; e < 8 * C; ++e) {
          float2& j = joined[e * L + lane];
          j = t == 0u ? make_float2(gw[e], gb[e]) : make_float2(j.x + gw[e], j.y + gb[e]);
        }
      }
      __syncthreads();
    }
    if (team != 0u) return;
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) { gw[e] = joined[e * L + lane].x; gb[e] = joined[e * L + lane].y; }
  }
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.cols;
#pragma unroll
  for (int e = 0; e < 8 * C; ++e) {
    const int64_t col = norm_col<L, WIDE>(lane, e / 8, e % 8);
    if (col < p.cols) {
      part[col] = gw[e];
      part[p.cols + col] = gb[e];
    }
  }
}

// Rows longer than a block holds: the gradient of s row by row, and the column sums by threads that own a column over a share of the rows.
__global__ void __launch_bounds__(kNormLong) k_norm_bwd_long(const __grid_constant__ NormArgs p) {
  after_previous();
  __shared__ float2 room[2][kNormLong / 32u];
  uint32_t turn = 0;
  const int64_t row = blockIdx.x;
  const float mean = p.stats[row], rstd = p.stats[p.rows + row], inv = 1.0f / static_cast<float>(p.cols);
  auto bf16 = [](const uint16_t* q, int64_t at) { return __uint_as_float(static_cast<uint32_t>(q[at]) << 16); };
  auto weighted = [&](int64_t col) { return bf16(p.dy, row * p.ld_dy + col) * (p.weight != nullptr ? norm_weight(p.weight, p.f32 != 0, col) : 1.0f); };
  float ta = 0.0f, tb = 0.0f;
  for (int64_t col = threadIdx.x; col < p.cols; col += kNormLong) {
    const float a = weighted(col);
    ta += a;
    tb = __fmaf_rn(a, (bf16(p.x, row * p.ld_x + col) - mean) * rstd, tb);
  }
  const float2 t = team_sum<kNormLong>(ta, tb, room[0], turn);
  const float ma = t.x * inv, mb = t.y * inv;
  for (int64_t col = threadIdx.x; col < p.cols; col += kNormLong) {
    const float v = rstd * (weighted(col) - ma - (bf16(p.x, row * p.ld_x + col) - mean) * rstd * mb);
    p.dx[row * p.cols + col] = static_cast<uint16_t>(pack_bf16(p.d != nullptr ? v + bf16(p.d, row * p.ld_d + col) : v, 0.0f));
  }
}
__global__ void __launch_bounds__(256) k_norm_columns(const __grid_constant__ NormArgs p, uint32_t shares) {
  after_previous();
  const int64_t strips = (p.cols + 255) / 256, share = blockIdx.x / strips, col = (blockIdx.x - share * strips) * 256 + threadIdx.x;
  if (col >= p.cols) return;
  const int64_t per = (p.rows + shares - 1) / shares, end = min(p.rows, (share + 1) * per);
  float gw = 0.0f, gb = 0.0f;
  for (int64_t row = share * per; row < end; ++row) {
    const float dy = __uint_as_float(static_cast<uint32_t>(p.dy[row * p.ld_dy + col]) << 16);
    const float s = __uint_as_float(static_cast<uint32_t>(p.x[row * p.ld_x + col]) << 16);
    gw = __fmaf_rn(dy, (s - p.stats[row]) * p.stats[p.rows + row], gw);
    gb += dy;
  }
  p.part[share * 2 * p.cols + col] = gw;
  p.part[(share * 2 + 1) * p.cols + col] = gb;
}

}  // namespace
