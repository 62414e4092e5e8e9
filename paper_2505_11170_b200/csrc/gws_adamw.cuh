// One AdamW step over many tensors in one launch:
//
//   g <- g * scale      m <- b1 m + (1 - b1) g      v <- b2 v + (1 - b2) g g      r = sqrt(v)
//   p <- p (1 - lr wd) - (m alpha) / (r rho + eps)        alpha = lr / (1 - b1^t),  rho = 1 / sqrt(1 - b2^t)
//
// every operation an FP32 one, rounded once, in the order written, so that the state is the same bits however the elements are split up and 8-bit
// codes are the same whichever way a value next to a border was reached.
//
// Parameters are BF16 or FP32.  Steps of a BF16 weight are mostly smaller than half its spacing and would be lost; `rest` keeps the 16 bits
// that a 32-bit weight has below the nearest BF16 number, so that p and rest together are the FP32 weight at 4 bytes, where an FP32 copy
// beside p takes 6.
//
// Moments are FP32, or 8 bits in groups of 256 consecutive elements with an FP32 unit per group and moment:
//   m   E4M3 codes, unit max|m| / 448
//   r   (not v: the square root halves the range of exponents) 4 bits of exponent and 4 of mantissa, no sign: code 16 e + f stands for
//       (1 + f / 16) 2^(e - 15) and 0 for zero, unit max r / 1.9375; a root above zero keeps a code above zero, because a v of zero under an m that
//       is not would make the next step m / eps
// The units are multiples of the largest element itself, not powers of two: where all of a group decays together, the unit decays and the codes stay,
// while with fixed units a factor of b2 = 0.95 or 0.999 (2.5 or 0.05 % of r) would be rounded away for as long as the gradient is small (half a step is 3 %).
//
// The elements of tensor i start at a multiple of 256 of arrays that all tensors share, so a group belongs to one tensor, and moments, units and rest are
// aligned whatever the parameters are.
#pragma once
#include <stdint.h>

#include "gws_act8.cuh"

namespace {

constexpr uint32_t kAdamwGroup = 256;             // elements of a group: eight to a lane
constexpr uint32_t kAdamwGroups = 16;             // groups of a block of eight warps
constexpr float kAdamwLeast = 0x1p-100f;          // a largest value below this is stored as zero

struct AdamwRec {
  void* p;
  const void* g;
  int64_t n;
  uint32_t group0, block0;        // the tensor's first group in the state, its first block in the launch
  float decay;                    // 1 - lr wd; wd where the step's scalars are on the device
  uint32_t flags;
};
enum : uint32_t { kAdamwF32 = 1u, kAdamwWide = 2u };      // FP32 tensors; both on boundaries of eight elements

struct AdamwArgs {
  uint8_t* codes;                 // 8 bits: [2, total]; FP32: moments
  float* units;
  int16_t* rest;
  int64_t total;
  const float* grad_scale;
  const float* scalars;           // alpha, rho, lr on the device, or null
  float b1, to_m, b2, to_v, eps, alpha, rho;
  int32_t n;
};
template <int CAP>
struct AdamwBatch {
  AdamwArgs a;
  AdamwRec e[CAP];
};

__device__ __forceinline__ V8 take32(const void* p) {     // memory that the same thread writes later
  V8 v;
  asm volatile("ld.global.v8.u32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v.x[0]), "=r"(v.x[1]), "=r"(v.x[2]), "=r"(v.x[3]), "=r"(v.x[4]), "=r"(v.x[5]), "=r"(v.x[6]), "=r"(v.x[7])
               : "l"(p)
               : "memory");
  return v;
}

// A lane's eight consecutive elements of a group, as FP32 bits.  `wide`: the whole group exists and lies on boundaries of eight elements; otherwise the warp reads
// (writes) neighbouring elements with neighbouring lanes and `turn` gives each lane its eight.
__device__ __forceinline__ void adamw_read(const void* p, bool f32, bool wide, int64_t left, uint32_t lane, uint32_t* turn, float (&x)[8]) {
  if (wide) {
    if (f32) {
      const V8 v = take32(static_cast<const float*>(p) + lane * 8u);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v.x[i]);
    } else {
      const uint4 v = reinterpret_cast<const uint4*>(p)[lane];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    }
    return;
  }
  uint32_t v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t at = lane + 32u * i;
    v[i] = at >= left ? 0u : f32 ? static_cast<const uint32_t*>(p)[at] : static_cast<uint32_t>(static_cast<const uint16_t*>(p)[at]) << 16;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) turn[lane + 32u * i] = v[i];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(turn[lane * 8u + i]);
  __syncwarp();
}
// x: FP32 bits, or for BF16 the number's 16 bits.
__device__ __forceinline__ void adamw_write(void* p, bool f32, bool wide, int64_t left, uint32_t lane, uint32_t* turn, const uint32_t (&x)[8]) {
  if (wide) {
    if (f32) {
      V8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.x[i] = x[i];
      st32(static_cast<float*>(p) + lane * 8u, v);
    } else {
      reinterpret_cast<uint4*>(p)[lane] = make_uint4(x[0] | (x[1] << 16), x[2] | (x[3] << 16), x[4] | (x[5] << 16), x[6] | (x[7] << 16));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) turn[lane * 8u + i] = x[i];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t at = lane + 32u * i;
    if (at >= left) continue;
    if (f32) static_cast<uint32_t*>(p)[at] = turn[at];
    else static_cast<uint16_t*>(p)[at] = static_cast<uint16_t>(turn[at]);
  }
  __syncwarp();
}

// Unit of a group from the FP32 bits of its largest magnitude; NaN where that is not finite.
__device__ __forceinline__ float adamw_unit(uint32_t top, float step) {
  if (top >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float m = __uint_as_float(top);
  return m >= kAdamwLeast ? __fmul_rn(m, step) : 0.0f;
}
__device__ __forceinline__ float adamw_inverse(float unit) { return unit > 0.0f ? __frcp_rn(unit) : 0.0f; }

__device__ __forceinline__ uint2 adamw_encode_m(const float (&m)[8], float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = encode4_e4m3(m[4 * i], m[4 * i + 1], m[4 * i + 2], m[4 * i + 3], inv);
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 adamw_encode_r(const float (&r)[8], float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t bits = __float_as_uint(__fmul_rn(r[i], inv));          // at most a little above 1.9375
    const int32_t code = static_cast<int32_t>((bits + 0x3FFFFu + ((bits >> 19) & 1u)) >> 19) - (112 << 4);
    const uint32_t c = r[i] > 0.0f && inv > 0.0f ? static_cast<uint32_t>(min(max(code, 1), 255)) : 0u;
    w[i >> 2] |= c << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void adamw_decode_m(uint2 c, float unit, float (&m)[8]) {
  float a[4], b[4];
  decode4_e4m3(c.x, unit, a);
  decode4_e4m3(c.y, unit, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) { m[i] = a[i]; m[4 + i] = b[i]; }
}
__device__ __forceinline__ void adamw_decode_r(uint2 c, float unit, float (&r)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t code = ((i < 4 ? c.x : c.y) >> (8 * (i & 3))) & 255u;
    r[i] = __fmul_rn(code != 0u ? __uint_as_float((code + (112u << 4)) << 19) : 0.0f, unit);
  }
}

// Memory-bound.  A warp takes a group, a lane eight elements of it; a block finds its tensor by bisection in the kernel parameters.
template <int FMT, int CAP>
__global__ void __launch_bounds__(256) k_adamw(const __grid_constant__ AdamwBatch<CAP> b) {
  after_previous();
  __shared__ uint32_t turns[8][kAdamwGroup];
  const AdamwArgs& a = b.a;
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.e[mid].block0 <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwRec& e = b.e[lo];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  uint32_t* turn = turns[warp];
  const bool f32 = (e.flags & kAdamwF32) != 0u, keeps = !f32 && a.rest != nullptr;
  const float scale = a.grad_scale != nullptr ? *a.grad_scale : 1.0f;
  float alpha = a.alpha, rho = a.rho, decay = e.decay;
  if (a.scalars != nullptr) {
    alpha = a.scalars[0];
    rho = a.scalars[1];
    decay = static_cast<float>(1.0 - static_cast<double>(a.scalars[2]) * static_cast<double>(decay));
  }
  const int64_t first = static_cast<int64_t>(blockIdx.x - e.block0) * kAdamwGroups;
  for (uint32_t u = warp; u < kAdamwGroups; u += 8u) {
    const int64_t at = (first + u) * kAdamwGroup, left = e.n - at;
    if (left <= 0) break;
    const bool wide = (e.flags & kAdamwWide) != 0u && left >= kAdamwGroup;
    const int64_t group = e.group0 + first + u, s = group * kAdamwGroup + lane * 8u;
    const size_t size = f32 ? 4u : 2u;
    char* pp = static_cast<char*>(e.p) + at * size;
    float p[8], g[8], m[8], v[8];
    uint4 low = make_uint4(0u, 0u, 0u, 0u);
    uint2 cm, cr;
    float um = 0.0f, ur = 0.0f;
    V8 wm, wv;
    if (FMT == GWS_ADAMW_8BIT) {
      cm = *reinterpret_cast<const uint2*>(a.codes + s);
      cr = *reinterpret_cast<const uint2*>(a.codes + a.total + s);
      um = a.units[group];
      ur = a.units[a.total / kAdamwGroup + group];
    } else {
      wm = take32(a.codes + s * 4);
      wv = take32(a.codes + (a.total + s) * 4);
    }
    if (keeps) low = *reinterpret_cast<const uint4*>(a.rest + s);
    adamw_read(static_cast<const char*>(e.g) + at * size, f32, wide, left, lane, turn, g);
    adamw_read(pp, f32, wide, left, lane, turn, p);
    if (FMT == GWS_ADAMW_8BIT) {
      adamw_decode_m(cm, um, m);
      adamw_decode_r(cr, ur, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) { m[i] = __uint_as_float(wm.x[i]); v[i] = __uint_as_float(wv.x[i]); }
    }
    if (keeps) {
      const uint32_t w[4] = {low.x, low.y, low.z, low.w};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        p[i] = __uint_as_float(__float_as_uint(p[i]) + static_cast<uint32_t>(static_cast<int32_t>(static_cast<int16_t>(w[i >> 1] >> (16 * (i & 1))))));
    }
    float r[8];
    uint32_t top_m = 0u, top_r = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float gs = a.grad_scale != nullptr ? __fmul_rn(g[i], scale) : g[i];
      m[i] = __fadd_rn(__fmul_rn(m[i], a.b1), __fmul_rn(gs, a.to_m));
      v[i] = __fadd_rn(__fmul_rn(v[i], a.b2), __fmul_rn(__fmul_rn(gs, a.to_v), gs));
      r[i] = __fsqrt_rn(v[i]);
      p[i] = __fsub_rn(__fmul_rn(p[i], decay), __fdiv_rn(__fmul_rn(m[i], alpha), __fadd_rn(__fmul_rn(r[i], rho), a.eps)));
      top_m = max(top_m, __float_as_uint(m[i]) & 0x7FFFFFFFu);
      top_r = max(top_r, __float_as_uint(r[i]) & 0x7FFFFFFFu);
    }
    if (FMT == GWS_ADAMW_8BIT) {
      um = adamw_unit(__reduce_max_sync(0xFFFFFFFFu, top_m), 1.0f / 448.0f);
      ur = adamw_unit(__reduce_max_sync(0xFFFFFFFFu, top_r), 1.0f / 1.9375f);
      // a group that is not finite has a NaN for its unit and codes of zero: it restores as NaN
      const float im = adamw_inverse(um), ir = adamw_inverse(ur);
      *reinterpret_cast<uint2*>(a.codes + s) = im > 0.0f ? adamw_encode_m(m, im) : make_uint2(0u, 0u);
      *reinterpret_cast<uint2*>(a.codes + a.total + s) = adamw_encode_r(r, ir);
      if (lane == 0) {
        a.units[group] = um;
        a.units[a.total / kAdamwGroup + group] = ur;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) { wm.x[i] = __float_as_uint(m[i]); wv.x[i] = __float_as_uint(v[i]); }
      st32(a.codes + s * 4, wm);
      st32(a.codes + (a.total + s) * 4, wv);
    }
    uint32_t out[8];
    if (f32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = __float_as_uint(p[i]);
    } else if (keeps) {
      uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i) {          // the nearest BF16 number (the larger of two as near) and what is left; a NaN as itself
        const uint32_t bits = p[i] != p[i] ? 0x7FC00000u : __float_as_uint(p[i]);
        out[i] = (bits + 0x8000u) >> 16;
        w[i >> 1] |= (bits & 0xFFFFu) << (16 * (i & 1));      // bits - (out << 16), as 16 bits
      }
      *reinterpret_cast<uint4*>(a.rest + s) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = pack_bf16(p[i], 0.0f) & 0xFFFFu;
    }
    adamw_write(pp, f32, wide, left, lane, turn, out);
  }
}

// alpha, rho and lr of a step whose count or rate is on the device.
__global__ void k_adamw_scalars(const int64_t* step_dev, const float* lr_dev, int64_t step, double lr, double b1, double b2, float* out) {
  after_previous();
  const double t = static_cast<double>(step_dev != nullptr ? *step_dev : step), rate = lr_dev != nullptr ? static_cast<double>(*lr_dev) : lr;
  out[0] = static_cast<float>(rate / (1.0 - pow(b1, t)));
  out[1] = static_cast<float>(1.0 / sqrt(1.0 - pow(b2, t)));
  out[2] = static_cast<float>(rate);
}

// What 8-bit moments stand for: m and v = r r in FP32.
__global__ void __launch_bounds__(256) k_adamw_values(const uint8_t* codes, const float* units, int64_t total, float* m, float* v) {
  after_previous();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, s = t * 8;
  if (s >= total) return;
  const int64_t group = s / kAdamwGroup;
  float x[8], r[8];
  adamw_decode_m(*reinterpret_cast<const uint2*>(codes + s), units[group], x);
  adamw_decode_r(*reinterpret_cast<const uint2*>(codes + total + s), units[total / kAdamwGroup + group], r);
  V8 a, b;
#pragma unroll
  for (int i = 0; i < 8; ++i) { a.x[i] = __float_as_uint(x[i]); b.x[i] = __float_as_uint(__fmul_rn(r[i], r[i])); }
  st32(m + s, a);
  st32(v + s, b);
}

}  // namespace
