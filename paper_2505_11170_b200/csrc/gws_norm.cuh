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
// boundaries, a thread takes eight neighbouring elements; otherwise neighbouring threads take neighbouring elements one by one.  Teams are as large as the row asks for (32 to 512
// threads of 16 elements): 4096 x 5632 on 512 threads, a third of them idle, took 43 us forward, on 384 34.
// The column sums of the backward pass stay in registers over all rows of a team and are joined in a fixed order: over the teams of a block in shared
// memory, over the blocks by k_column_sums.  Results do not depend on timing.
#pragma once
#include <stdint.h>

#include "gws_act8.cuh"
#include "gws_pair.cuh"
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
// `units`: of eight elements, or elements one by one, that the row has (0: a row past the last).
template <int L, int C, bool WIDE>
__device__ __forceinline__ void norm_load(const uint16_t* row, uint32_t units, uint32_t lane, NormWords<C, WIDE>& w) {
  if constexpr (WIDE) {
    const uint4* p = reinterpret_cast<const uint4*>(row) + lane;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint4 q = lane + c * L < units ? __ldg(p + c * L) : make_uint4(0u, 0u, 0u, 0u);
      w.x[4 * c] = q.x; w.x[4 * c + 1] = q.y; w.x[4 * c + 2] = q.z; w.x[4 * c + 3] = q.w;
    }
  } else {
    const uint16_t* p = row + lane;
#pragma unroll
    for (int e = 0; e < 8 * C; ++e) w.x[e] = lane + e * L < units ? static_cast<uint32_t>(__ldg(p + e * L)) : 0u;
  }
}
// Elements 2 i and 2 i + 1.
template <int C, bool WIDE>
__device__ __forceinline__ F2 norm_pair(const NormWords<C, WIDE>& w, int i) {
  if constexpr (WIDE) return two(bf16_lo(w.x[i]), bf16_hi(w.x[i]));
  else return two(__uint_as_float(w.x[2 * i] << 16), __uint_as_float(w.x[2 * i + 1] << 16));
}
// v holds pairs of BF16.
template <int L, int C, bool WIDE>
__device__ __forceinline__ void norm_write(uint16_t* row, uint32_t units, uint32_t lane, const uint32_t (&v)[4 * C]) {
  if constexpr (WIDE) {
    uint4* p = reinterpret_cast<uint4*>(row) + lane;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (lane + c * L < units) p[c * L] = make_uint4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
  } else {
    uint16_t* p = row + lane;
#pragma unroll
    for (int e = 0; e < 8 * C; ++e)
      if (lane + e * L < units) p[e * L] = static_cast<uint16_t>(v[e / 2] >> (16 * (e & 1)));
  }
}
// Eight weights (or biases) of unit c, in pairs.
template <int L, bool WIDE>
__device__ __forceinline__ void norm_weights(const void* w, bool f32, float none, int64_t cols, uint32_t lane, int c, float4 (&v)[2]) {
  v[0] = v[1] = make_float4(none, none, none, none);
  if (w == nullptr) return;
  const int64_t col = norm_col<L, WIDE>(lane, c, 0);
  if (WIDE && f32) {
    if (col >= cols) return;
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + col);
    v[0] = __ldg(p);
    v[1] = __ldg(p + 1);
  } else if (WIDE) {
    if (col >= cols) return;
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + col));
    v[0] = make_float4(bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y));
    v[1] = make_float4(bf16_lo(q.z), bf16_hi(q.z), bf16_lo(q.w), bf16_hi(q.w));
  } else {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = norm_col<L, WIDE>(lane, c, i) < cols ? norm_weight(w, f32, norm_col<L, WIDE>(lane, c, i)) : 0.0f;
    v[0] = make_float4(t[0], t[1], t[2], t[3]);
    v[1] = make_float4(t[4], t[5], t[6], t[7]);
  }
}

// Blocks of the forward kernel that an SM holds: as many as leave a thread registers for its row and the next one.  us with a residual, one block more or less beside it: 16384 x 2048
// 46 (four: 49), x 768 18 (four: 20.5), 4096 x 3000 17.0 (three: 18.5), 4096 x 4096 22.8 (three: 23.5); elements one by one, 16384 x 1365 46 (three: 54, five: 66), x 767 29 (four:
// 32.5), 8192 x 4001 67 (three: 72), 4096 x 6001 77 (one: 116).
constexpr int norm_blocks(int team, bool wide) {
  return team > 512 ? 1 : team > 256 ? 2 : team == 256 || team == 192 || (team == 96 && !wide) ? 4 : 3;
}

// Sums of two values over a team; every thread of the team calls it the same number of times.  `room`: [2][threads / 32], used in turn.  The teams of a block wait for themselves alone
// (16384 x 1024 forward, two teams: 25.8 us when the block met, 23.7 so).
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
  if (L <= 256) asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.x / L + 1u), "n"(L) : "memory");
  else __syncthreads();
  const float2* from = mine + (threadIdx.x / L) * kWarps;
  float2 t = from[0];
#pragma unroll
  for (uint32_t w = 1; w < kWarps; ++w) { t.x += from[w].x; t.y += from[w].y; }
  return t;
}

template <int L>
constexpr uint32_t kNormThreads = L < 256 ? 256u / L * L : static_cast<uint32_t>(L);          // of a block
// Of a block of the backward kernel, whose sums over its teams are a part each: large blocks leave half of the parts (1000 x 4096 20 -> 15 us), but small teams are joined one after
// the other (300 x 768 in blocks of eight teams 6.0 us, of four 5.0).
template <int L>
constexpr uint32_t kNormBackThreads = L < 128 ? 256u / L * L : L < 512 ? 512u / L * L : static_cast<uint32_t>(L);

// Memory-bound: 2 or 4 bytes in, 2 or 4 out per element.  A team takes rows in turn, with the next row's words under way; weights stay in shared memory where the block's teams (or
// its rows) share them, and the arithmetic is on pairs (one by one, a row to a warp and
// its weights read for every row, took 41 us where this takes 28).
// 16384 x 2048: 28 us (4.8 TB/s), with a residual 46 (5.8 TB/s); 16384 x 768 with a residual 18; 16384 x 1365, elements one by one, 46 (3.9 TB/s); one row 2.
template <int L, int C, bool WIDE>
__global__ void __launch_bounds__(kNormThreads<L>, norm_blocks(L, WIDE)) k_norm_fwd(const __grid_constant__ NormArgs p) {
  after_previous();
  constexpr uint32_t kTeams = kNormThreads<L> / L;
  constexpr bool kHeld = L <= 256;
  __shared__ float2 room[2][kNormThreads<L> / 32u];
  __shared__ float4 held[kHeld ? 2 : 1][kHeld ? 2 * C : 1][kHeld ? L : 1];
  uint32_t turn = 0;
  const uint32_t lane = threadIdx.x % L, team = threadIdx.x / L;
  if (kHeld && team < 2u) {
    if (team == 0u || kTeams == 1u)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float4 q[2];
        norm_weights<L, WIDE>(p.weight, p.f32 != 0, 1.0f, p.cols, lane, c, q);
        held[0][2 * c][lane] = q[0];
        held[0][2 * c + 1][lane] = q[1];
      }
    if (team == 1u || kTeams == 1u)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float4 q[2];
        norm_weights<L, WIDE>(p.bias, p.f32 != 0, 0.0f, p.cols, lane, c, q);
        held[kHeld ? 1 : 0][2 * c][lane] = q[0];
        held[kHeld ? 1 : 0][2 * c + 1][lane] = q[1];
      }
  }
  if (kHeld) __syncthreads();
  struct Row {
    NormWords<C, WIDE> x, r;
  } next;
  const uint32_t all = static_cast<uint32_t>(WIDE ? p.cols / 8 : p.cols);
  auto fetch = [&](int64_t row, Row& to) {
    const uint32_t units = row < p.rows ? all : 0u;
    norm_load<L, C, WIDE>(p.x + row * p.ld_x, units, lane, to.x);
    if (p.r != nullptr) norm_load<L, C, WIDE>(p.r + row * p.ld_r, units, lane, to.r);
  };
  const float inv = 1.0f / static_cast<float>(p.cols);
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
      fetch(row0 + team, now);
    }
    const int64_t row = row0 + team;
    const uint32_t units = row < p.rows ? all : 0u;                                // nothing is written for rows past the last
    F2 s[4 * C], t = both(0.0f);
    uint32_t w[4 * C];
    if (p.r != nullptr) {
#pragma unroll
      for (int i = 0; i < 4 * C; ++i) {
        const F2 v = fma2(norm_pair(now.x, i), both(1.0f), norm_pair(now.r, i));
        w[i] = pack_bf16(first_of(v), second_of(v));
        s[i] = two(bf16_lo(w[i]), bf16_hi(w[i]));
      }
      norm_write<L, C, WIDE>(p.sum + row * p.cols, units, lane, w);
    } else {
#pragma unroll
      for (int i = 0; i < 4 * C; ++i) s[i] = norm_pair(now.x, i);
    }
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) t = fma2(s[i], both(1.0f), t);
    const float mean = team_sum<L>(first_of(t) + second_of(t), 0.0f, room[0], turn).x * inv;
    t = both(0.0f);
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) {
      s[i] = fma2(s[i], both(1.0f), both(-mean));
      if constexpr (WIDE) {
        if (lane + i / 4 * L >= units) s[i] = both(0.0f);                                        // outside
      } else {
        s[i] = two(lane + 2 * i * L < units ? first_of(s[i]) : 0.0f, lane + (2 * i + 1) * L < units ? second_of(s[i]) : 0.0f);
      }
      t = fma2(s[i], s[i], t);
    }
    const float rstd = rsqrtf(team_sum<L>(first_of(t) + second_of(t), 0.0f, room[0], turn).x * inv + p.eps);
    if (lane == 0 && p.stats != nullptr && row < p.rows) {
      p.stats[row] = mean;
      p.stats[p.rows + row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float4 q[2], b[2];
      if constexpr (kHeld) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          q[h] = held[0][2 * c + h][lane];
          b[h] = held[1][2 * c + h][lane];
        }
      } else {
        norm_weights<L, WIDE>(p.weight, p.f32 != 0, 1.0f, p.cols, lane, c, q);
        norm_weights<L, WIDE>(p.bias, p.f32 != 0, 0.0f, p.cols, lane, c, b);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 qh = q[i / 2], bh = b[i / 2];
        const F2 v = fma2(mul2(s[4 * c + i], both(rstd)), (i & 1) == 0 ? two(qh.x, qh.y) : two(qh.z, qh.w), (i & 1) == 0 ? two(bh.x, bh.y) : two(bh.z, bh.w));
        w[4 * c + i] = pack_bf16(first_of(v), second_of(v));
      }
    }
    norm_write<L, C, WIDE>(p.y + row * p.cols, units, lane, w);
  }
}

// Rows of any length: a block reads its row again for each pass, mostly from L2.
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

// Memory-bound: 4 or 6 bytes in, 2 out per element.  16384 x 2048: with grad_sum 45 us (6.0 TB/s), 48 with the sums of the weight's and the bias's gradients (parts in stores of
// 32 bytes, whose join is a launch; word by word 50); without the next row's loads under way 106.  4096 x 5632 41, 1000 x 4096 10.5.  16384 x 1365, elements one by one, 64.
template <int L, int C, bool WIDE>
__global__ void __launch_bounds__(kNormBackThreads<L>, L < 128 ? 2 : 1) k_norm_bwd(const __grid_constant__ NormArgs p) {
  after_previous();
  constexpr uint32_t kTeams = kNormBackThreads<L> / L;
  __shared__ float2 room[2][kNormBackThreads<L> / 32u];
  __shared__ float4 held[kTeams > 1u ? 4 * C : 2 * C][L];                      // the weights, the same for every team and row; then the sums over the teams
  uint32_t turn = 0;
  const uint32_t lane = threadIdx.x % L, team = threadIdx.x / L;
  const float inv = 1.0f / static_cast<float>(p.cols);
  F2 gw[4 * C], gb[4 * C];
#pragma unroll
  for (int i = 0; i < 4 * C; ++i) gw[i] = gb[i] = both(0.0f);
  if (team == 0u) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float4 q[2];
      norm_weights<L, WIDE>(p.weight, p.f32 != 0, 1.0f, p.cols, lane, c, q);
      held[2 * c][lane] = q[0];
      held[2 * c + 1][lane] = q[1];
    }
  }
  __syncthreads();
  auto weight = [&](int i) {
    const float4 q = held[i / 2][lane];
    return (i & 1) == 0 ? two(q.x, q.y) : two(q.z, q.w);
  };
  struct Row {
    NormWords<C, WIDE> s, dy, d;
    float mean, rstd;
  } next;
  const uint32_t all = static_cast<uint32_t>(WIDE ? p.cols / 8 : p.cols);
  auto fetch = [&](int64_t row, Row& r) {
    const uint32_t units = row < p.rows ? all : 0u;
    norm_load<L, C, WIDE>(p.x + row * p.ld_x, units, lane, r.s);
    norm_load<L, C, WIDE>(p.dy + row * p.ld_dy, units, lane, r.dy);
    if (p.d != nullptr) norm_load<L, C, WIDE>(p.d + row * p.ld_d, units, lane, r.d);
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
    // xh = s rstd - mean rstd would lose a row of large mean: the mean is taken off first
    auto centred = [&](int i) { return mul2(fma2(norm_pair(now.s, i), both(1.0f), both(-now.mean)), both(now.rstd)); };
    F2 ta = both(0.0f), tb = both(0.0f);
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) {
      const F2 xh = centred(i), dy = norm_pair(now.dy, i), a = mul2(dy, weight(i));          // columns past the width have dy = 0
      ta = fma2(a, both(1.0f), ta);
      tb = fma2(a, xh, tb);
      gw[i] = fma2(dy, xh, gw[i]);
      gb[i] = fma2(dy, both(1.0f), gb[i]);
    }
    const float2 t = team_sum<L>(first_of(ta) + second_of(ta), first_of(tb) + second_of(tb), room[0], turn);
    if (p.dx != nullptr && row < p.rows) {
      const F2 ma = both(-t.x * inv), mb = both(-t.y * inv), rstd = both(now.rstd);
      uint32_t w[4 * C];
#pragma unroll
      for (int i = 0; i < 4 * C; ++i) {
        const F2 a = fma2(norm_pair(now.dy, i), weight(i), ma);
        F2 v = mul2(fma2(centred(i), mb, a), rstd);
        if (p.d != nullptr) v = fma2(v, both(1.0f), norm_pair(now.d, i));
        w[i] = pack_bf16(first_of(v), second_of(v));
      }
      norm_write<L, C, WIDE>(p.dx + row * p.cols, all, lane, w);
    }
  }
  if (p.part == nullptr) return;
  if constexpr (kTeams > 1u) {
    __syncthreads();
    for (uint32_t t = 0; t < kTeams; ++t) {
      if (team == t) {
#pragma unroll
        for (int i = 0; i < 4 * C; ++i) {
          float4& j = held[i][lane];
          const float4 g = make_float4(first_of(gw[i]), second_of(gw[i]), first_of(gb[i]), second_of(gb[i]));
          j = t == 0u ? g : make_float4(j.x + g.x, j.y + g.y, j.z + g.z, j.w + g.w);
        }
      }
      __syncthreads();
    }
    if (team != 0u) return;
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) {
      const float4 j = held[i][lane];
      gw[i] = two(j.x, j.y);
      gb[i] = two(j.z, j.w);
    }
  }
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.cols;
  if constexpr (WIDE) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = norm_col<L, WIDE>(lane, c, 0);
      if (col >= p.cols) continue;
      V8 w, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w.x[2 * i] = __float_as_uint(first_of(gw[4 * c + i]));
        w.x[2 * i + 1] = __float_as_uint(second_of(gw[4 * c + i]));
        b.x[2 * i] = __float_as_uint(first_of(gb[4 * c + i]));
        b.x[2 * i + 1] = __float_as_uint(second_of(gb[4 * c + i]));
      }
      st32(part + col, w);
      st32(part + p.cols + col, b);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8 * C; ++e) {
    const int64_t col = norm_col<L, WIDE>(lane, e / 8, e % 8);
    if (col < p.cols) {
      part[col] = (e & 1) == 0 ? first_of(gw[e / 2]) : second_of(gw[e / 2]);
      part[p.cols + col] = (e & 1) == 0 ? first_of(gb[e / 2]) : second_of(gb[e / 2]);
    }
  }
}

// Rows longer than a block holds (backward: 8192 elements; 1024 x 16384 takes 112 us, three times the bytes of a row in registers): the gradient of s row by row, and the column sums by threads that own a column over a share of the rows.
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
