// One AdamW step over many tensors in one launch:
//
//   g <- g * scale      m <- b1 m + (1 - b1) g      v <- b2 v + (1 - b2) g g      r = sqrt(v)
//   p <- p (1 - lr wd) - (m alpha) / (r rho + eps)        alpha = lr / (1 - b1^t),  rho = 1 / sqrt(1 - b2^t)
//
// every operation an FP32 one, rounded once, in the order written (root2 and quotient2 say with which exceptions), so that the state is the same bits however the elements are split up and 8-bit
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
#include "gws_pair.cuh"

namespace {

constexpr uint32_t kAdamwGroup = 256;             // elements of a group: eight to a lane
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
  uint32_t per;                   // groups of a block of eight warps
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

// A lane's eight consecutive elements of a parameter and of its gradient, as they come from memory.  WIDE: whole groups on boundaries of eight elements, four words of
// BF16 pairs or eight of FP32.  Otherwise the warp reads neighbouring elements with neighbouring lanes, and `turn` gives each lane its eight.
template <bool F32, bool WIDE>
struct AdamwWords {
  uint32_t x[WIDE && !F32 ? 4 : 8];
};
template <bool F32, bool WIDE>
__device__ __forceinline__ void adamw_fetch(const void* p, int64_t left, uint32_t lane, AdamwWords<F32, WIDE>& w) {
  if constexpr (WIDE && F32) {
    const V8 v = take32(static_cast<const float*>(p) + lane * 8u);
#pragma unroll
    for (int i = 0; i < 8; ++i) w.x[i] = v.x[i];
  } else if constexpr (WIDE) {
    const uint4 v = reinterpret_cast<const uint4*>(p)[lane];
    w.x[0] = v.x; w.x[1] = v.y; w.x[2] = v.z; w.x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t at = lane + 32u * i;
      w.x[i] = at >= left ? 0u : F32 ? static_cast<const uint32_t*>(p)[at] : static_cast<uint32_t>(static_cast<const uint16_t*>(p)[at]);
    }
  }
}
// The lane's own eight: words of BF16 pairs, or FP32.
template <bool F32, bool WIDE>
__device__ __forceinline__ void adamw_turn(const AdamwWords<F32, WIDE>& w, uint32_t lane, uint4* turn, uint32_t (&x)[F32 ? 8 : 4]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < (F32 ? 8 : 4); ++i) x[i] = w.x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (F32) reinterpret_cast<uint32_t*>(turn)[lane + 32 * i] = w.x[i];
      else reinterpret_cast<uint16_t*>(turn)[lane + 32 * i] = static_cast<uint16_t>(w.x[i]);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) {
      const uint4 v = turn[lane * (F32 ? 2 : 1) + i];
      x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
    }
    __syncwarp();
  }
}
template <bool F32, bool WIDE>
__device__ __forceinline__ void adamw_write(void* p, int64_t left, uint32_t lane, uint4* turn, const uint32_t (&x)[F32 ? 8 : 4]) {
  if constexpr (WIDE && F32) {
    V8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.x[i] = x[i];
    st32(static_cast<float*>(p) + lane * 8u, v);
  } else if constexpr (WIDE) {
    reinterpret_cast<uint4*>(p)[lane] = make_uint4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) turn[lane * (F32 ? 2 : 1) + i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t at = lane + 32u * i;
      if (at >= left) continue;
      if constexpr (F32) static_cast<uint32_t*>(p)[at] = reinterpret_cast<const uint32_t*>(turn)[at];
      else static_cast<uint16_t*>(p)[at] = reinterpret_cast<const uint16_t*>(turn)[at];
    }
    __syncwarp();
  }
}

// Square root and quotient to the nearest, of pairs, by the residual of an approximation (Markstein's method): with g near sqrt(v) and h near 1 / (2 sqrt(v)), g + (v - g g) h
// rounds as sqrt(v) does, and with y near 1 / d and q near n / d, q + (n - d q) y as n / d.  The reciprocal is brought to FP32's
// own precision by two steps of Newton's iteration before; for the root the device's approximation is near enough.  v in [2^-100, 2^100],
// d in [2^-40, 2^81], n up to 2^70 (or n = 1 and d in [2^-110, 2^120)); a quotient of an n below 2^-100, whose residual may be below the smallest number, or one that is itself
// below 2^-126 can be one unit of its last place off.  The method is exact where the reciprocal is; that it is exact with this one is sampled, not proven: the tests compare the
// roots of every significand in five pairs of binades, 6 10^7 random quotients and 10^7 as near to a border as they come with sqrt and /.
__device__ __forceinline__ F2 root2(F2 v) {
  float y0, y1;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(first_of(v)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(second_of(v)));
  const F2 y = two(y0, y1), g = mul2(v, y), h = mul2(y, both(-0.5f));         // h is held with its sign changed
  return fma2(two(__fmaf_rn(first_of(g), first_of(g), -first_of(v)), __fmaf_rn(second_of(g), second_of(g), -second_of(v))), h, g);
}
__device__ __forceinline__ F2 quotient2(F2 n, F2 d) {
  float y0, y1;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(first_of(d)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(second_of(d)));
  const F2 minus = mul2(d, both(-1.0f)), one = both(1.0f);
  F2 y = two(y0, y1);
  y = fma2(fma2(minus, y, one), y, y);
  y = fma2(fma2(minus, y, one), y, y);
  const F2 q = mul2(n, y);
  return fma2(fma2(minus, q, n), y, q);
}

// Unit of a group from the FP32 bits of its largest magnitude; NaN where that is not finite.
__device__ __forceinline__ float adamw_unit(uint32_t top, float step) {
  const float unit = __uint_as_float(top) >= kAdamwLeast ? __fmul_rn(__uint_as_float(top), step) : 0.0f;
  return top < 0x7F800000u ? unit : __uint_as_float(0x7FC00000u);
}

__device__ __forceinline__ uint2 adamw_encode_m(const F2 (&m)[4], float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const F2 a = mul2(m[2 * i], both(inv)), b = mul2(m[2 * i + 1], both(inv));
    w[i] = static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(first_of(a), second_of(a)), __NV_SATFINITE, __NV_E4M3)) |
           static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(first_of(b), second_of(b)), __NV_SATFINITE, __NV_E4M3)) << 16;
  }
  return make_uint2(w[0], w[1]);
}
// `small`: there may be roots of zero among them, or some below the least code's.
__device__ __forceinline__ uint2 adamw_encode_r(const F2 (&r)[4], float inv, bool small) {
  uint32_t c[8];
  // 2^19 t - fl(2^19 t - t) is t to four bits of mantissa, nearest even: 2^19 t - t has the last place that t is to be rounded to (a finer one just above a power of two,
  // where t becomes that power all the same), and 2^19 t is an even number of it where t is half way.  Above 2^-15 the code is then bits 19 to 26.  t is at most a little
  // above 1.9375.
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const F2 t = mul2(r[i], both(inv)), q = fma2(t, both(0x1p19f), mul2(t, both(-524287.0f)));
    c[2 * i] = __float_as_uint(first_of(q));
    c[2 * i + 1] = __float_as_uint(second_of(q));
  }
  if (small) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = (i & 1) == 0 ? first_of(r[i / 2]) : second_of(r[i / 2]);
      c[i] = inv > 0.0f && x > 0.0f ? max(c[i], (112u << 23) + (1u << 19)) : 0u;
    }
  }
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __byte_perm(c[2 * i], c[2 * i + 1], 0x7632) >> 3;       // codes in bytes 0 and 2
  return make_uint2(__byte_perm(w[0], w[1], 0x6420), __byte_perm(w[2], w[3], 0x6420));
}
__device__ __forceinline__ void adamw_decode_m(uint2 c, float unit, F2 (&m)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? c.x : c.y;
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>((i & 1) == 0 ? w & 0xFFFFu : w >> 16), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    m[i] = mul2(two(f.x, f.y), both(unit));
  }
}
__device__ __forceinline__ void adamw_decode_r(uint2 c, float unit, F2 (&r)[4]) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((__byte_perm(i < 4 ? c.x : c.y, 0u, 0x4440u + (i & 3)) << 19) + (112u << 23));
  const auto has_zero = [](uint32_t w) { return ((w - 0x01010101u) & ~w & 0x80808080u) != 0u; };
  if (has_zero(c.x) || has_zero(c.y)) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((((i < 4 ? c.x : c.y) >> (8 * (i & 3))) & 255u) == 0u) x[i] = 0.0f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = mul2(two(x[2 * i], x[2 * i + 1]), both(unit));
}

constexpr uint32_t kAdamwSlot = 2048u;               // bytes of a group with 8-bit moments: gradient, parameter, rest, codes
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}

struct AdamwScalars {
  float scale, alpha, rho, decay;
  bool exact;                     // eps, alpha and rho are of sizes at which root2 and quotient2 are exact
};

// Groups first + warp, first + warp + 8, ... of a tensor, `count` of them over the warps.  Addresses are the block's, plus 32 bits a lane.
template <int FMT, bool LOOSE, bool F32, bool WIDE>
__device__ __forceinline__ void adamw_run(const AdamwArgs& a, const AdamwRec& e, const AdamwScalars& k, int64_t first, uint32_t count, uint4* turn) {
  // With 8-bit moments a group is 2 KB and long arithmetic: the next one is under way meanwhile, to shared memory, which leaves the registers to more warps.
  constexpr bool kStaged = FMT == GWS_ADAMW_8BIT && !F32 && WIDE, kAhead = FMT == GWS_ADAMW_8BIT && !F32 && !WIDE && LOOSE;
  constexpr uint32_t kSize = F32 ? 4u : 2u;
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const bool keeps = !F32 && a.rest != nullptr;
  const int64_t group0 = e.group0 + first, s0 = group0 * kAdamwGroup, left0 = e.n - first * kAdamwGroup;
  constexpr uint32_t kEach = FMT == GWS_ADAMW_8BIT ? 1u : 4u;                // bytes of a moment
  char* const at_m = reinterpret_cast<char*>(a.codes) + s0 * kEach;
  char* const at_v = at_m + a.total * kEach;
  char* const at_rest = reinterpret_cast<char*>(a.rest) + s0 * 2;
  char* const at_p = static_cast<char*>(e.p) + first * (kAdamwGroup * kSize);
  const char* const at_g = static_cast<const char*>(e.g) + first * (kAdamwGroup * kSize);
  float* const at_um = a.units + group0;
  float* const at_ur = at_um + a.total / kAdamwGroup;
  struct Raw {
    AdamwWords<F32, WIDE> g, p;
    uint4 low;
    uint2 cm, cr;
    float um, ur;
    V8 m, v;
  } next;
  auto fetch = [&](uint32_t u, Raw& r) {
    const uint32_t s = u * kAdamwGroup + lane * 8u;
    if (FMT == GWS_ADAMW_8BIT) {
      r.cm = *reinterpret_cast<const uint2*>(at_m + s);
      r.cr = *reinterpret_cast<const uint2*>(at_v + s);
      r.um = at_um[u];
      r.ur = at_ur[u];
    } else {
      r.m = take32(at_m + s * 4u);
      r.v = take32(at_v + s * 4u);
    }
    r.low = make_uint4(0u, 0u, 0u, 0u);
    if (keeps) r.low = *reinterpret_cast<const uint4*>(at_rest + s * 2u);
    adamw_fetch<F32, WIDE>(at_g + u * (kAdamwGroup * kSize), left0 - u * kAdamwGroup, lane, r.g);
    adamw_fetch<F32, WIDE>(at_p + u * (kAdamwGroup * kSize), left0 - u * kAdamwGroup, lane, r.p);
  };
  uint32_t u = warp;
  uint32_t slot = 0;
  float next_um = 0.0f, next_ur = 0.0f;
  auto stage = [&](uint32_t u, uint32_t slot) {
    const uint32_t s = u * kAdamwGroup + lane * 8u, to = static_cast<uint32_t>(__cvta_generic_to_shared(turn)) + slot * kAdamwSlot + lane * 16u;
    copy_async<16>(to, at_g + s * 2u);
    copy_async<16>(to + 512u, at_p + s * 2u);
    if (keeps) copy_async<16>(to + 1024u, at_rest + s * 2u);
    copy_async<8>(to - lane * 8u + 1536u, at_m + s);
    copy_async<8>(to - lane * 8u + 1792u, at_v + s);
    next_um = at_um[u];
    next_ur = at_ur[u];
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (kStaged && u < count) stage(u, 0);
  if (kAhead && u < count) fetch(u, next);
#pragma unroll 1
  for (; u < count; u += 8) {
    Raw raw;
    if constexpr (kStaged) {
      raw.um = next_um;
      raw.ur = next_ur;
      if (u + 8u < count) {
        stage(u + 8u, slot ^ 1u);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      const uint4* from = turn + slot * (kAdamwSlot / 16u) + lane;                          // what this lane copied
      slot ^= 1u;
      const uint4 g = from[0], p = from[32];
      raw.g.x[0] = g.x; raw.g.x[1] = g.y; raw.g.x[2] = g.z; raw.g.x[3] = g.w;
      raw.p.x[0] = p.x; raw.p.x[1] = p.y; raw.p.x[2] = p.z; raw.p.x[3] = p.w;
      raw.low = keeps ? from[64] : make_uint4(0u, 0u, 0u, 0u);
      const uint2* codes = reinterpret_cast<const uint2*>(from - lane + 96) + lane;
      raw.cm = codes[0];
      raw.cr = codes[32];
    } else if constexpr (kAhead) {
      raw = next;
      if (u + 8u < count) fetch(u + 8u, next);
    } else {
      fetch(u, raw);
    }
    const uint32_t s = u * kAdamwGroup + lane * 8u;
    uint32_t gw[F32 ? 8 : 4], pw[F32 ? 8 : 4];
    adamw_turn<F32, WIDE>(raw.g, lane, turn, gw);
    adamw_turn<F32, WIDE>(raw.p, lane, turn, pw);
    const uint32_t lw[4] = {raw.low.x, raw.low.y, raw.low.z, raw.low.w};
    float p[8];
    F2 m[4], v[4], r[4];
    if (FMT == GWS_ADAMW_8BIT) {
      adamw_decode_m(raw.cm, raw.um, m);
      adamw_decode_r(raw.cr, raw.ur, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[i] = two(__uint_as_float(raw.m.x[2 * i]), __uint_as_float(raw.m.x[2 * i + 1]));
        v[i] = two(__uint_as_float(raw.v.x[2 * i]), __uint_as_float(raw.v.x[2 * i + 1]));
      }
    }
    float least = __uint_as_float(0x7F800000u), most = 0.0f, top = 0.0f;      // the last two NaN if any is
    F2 odd = both(0.0f);                                                      // zero, or NaN if a weight is not finite
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      F2 g;
      if constexpr (F32) {
        g = two(__uint_as_float(gw[2 * i]), __uint_as_float(gw[2 * i + 1]));
        p[2 * i] = __uint_as_float(pw[2 * i]);
        p[2 * i + 1] = __uint_as_float(pw[2 * i + 1]);
      } else {
        g = two(bf16_lo(gw[i]), bf16_hi(gw[i]));
        // the weight's bits, (p << 16) + rest: the upper halves are one lower where the rest is negative
        const uint32_t upper = pw[i] - ((lw[i] >> 15) & 0x00010001u);
        p[2 * i] = __uint_as_float(__byte_perm(lw[i], upper, 0x5410));
        p[2 * i + 1] = __uint_as_float(__byte_perm(lw[i], upper, 0x7632));
      }
      g = mul2(g, both(k.scale));
      m[i] = add2(mul2(m[i], both(a.b1)), mul2(g, both(a.to_m)));
      v[i] = add2(mul2(v[i], both(a.b2)), mul2(mul2(g, both(a.to_v)), g));
      least = fminf(least, fminf(first_of(v[i]), second_of(v[i])));
      most = max_nan(most, max_nan(first_of(v[i]), second_of(v[i])));
      top = max_nan(top, max_nan(fabsf(first_of(m[i])), fabsf(second_of(m[i]))));
      odd = fma2(two(p[2 * i], p[2 * i + 1]), both(0.0f), odd);
    }
    // Whether all of this lane's numbers are where root2 and quotient2 are exact; a v of zero is not.
    const bool plain = k.exact && least >= 0x1p-100f && most <= 0x1p100f && top <= 0x1p40f && first_of(odd) + second_of(odd) == 0.0f;
    uint32_t top_m = __float_as_uint(top), top_r = 0u;
    if (plain) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r[i] = root2(v[i]);
        const F2 q = quotient2(mul2(m[i], both(-k.alpha)), add2(mul2(r[i], both(k.rho)), both(a.eps)));
        const F2 w = add2(mul2(two(p[2 * i], p[2 * i + 1]), both(k.decay)), q);
        p[2 * i] = first_of(w);
        p[2 * i + 1] = second_of(w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (!F32) {                            // a zero under a negative rest, which only a parameter set from outside is: zero
          const uint32_t half = pw[i / 2] >> (16 * (i & 1)) & 0xFFFFu;
          const int32_t low = static_cast<int16_t>(lw[i / 2] >> (16 * (i & 1)));
          p[i] = __uint_as_float((half & 0x7FFFu) == 0u && low < 0 ? half << 16 : (half << 16) + static_cast<uint32_t>(low));
        }
        const float mi = (i & 1) == 0 ? first_of(m[i / 2]) : second_of(m[i / 2]), ri = __fsqrt_rn((i & 1) == 0 ? first_of(v[i / 2]) : second_of(v[i / 2]));
        r[i / 2] = (i & 1) == 0 ? two(ri, ri) : two(first_of(r[i / 2]), ri);
        p[i] = __fsub_rn(__fmul_rn(p[i], k.decay), __fdiv_rn(__fmul_rn(mi, k.alpha), __fadd_rn(__fmul_rn(ri, k.rho), a.eps)));
        if (p[i] != p[i]) p[i] = __uint_as_float(0x7FC00000u);         // which stays a NaN when it is rounded
        top_m = max(top_m, __float_as_uint(mi) & 0x7FFFFFFFu);          // a NaN is above everything
      }
    }
    if (FMT == GWS_ADAMW_8BIT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) top_r = max(top_r, max(__float_as_uint(first_of(r[i])) & 0x7FFFFFFFu, __float_as_uint(second_of(r[i])) & 0x7FFFFFFFu));
      const float um = adamw_unit(__reduce_max_sync(0xFFFFFFFFu, top_m), 1.0f / 448.0f), ur = adamw_unit(__reduce_max_sync(0xFFFFFFFFu, top_r), 1.0f / 1.9375f);
      // a group that is not finite has a NaN for its unit and codes of zero: it restores as NaN
      const F2 inverse = quotient2(both(1.0f), two(um, ur));
      const float im = um > 0.0f ? first_of(inverse) : 0.0f, ir = ur > 0.0f ? second_of(inverse) : 0.0f;
      const bool small = !plain || !(__fmul_rn(least, __fmul_rn(ir, ir)) >= 0x1.3p-30f);         // (1.0625 2^-15)^2 and some more
      *reinterpret_cast<uint2*>(at_m + s) = plain || im > 0.0f ? adamw_encode_m(m, im) : make_uint2(0u, 0u);
      *reinterpret_cast<uint2*>(at_v + s) = adamw_encode_r(r, ir, small);
      if (lane == 0) {
        at_um[u] = um;
        at_ur[u] = ur;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        raw.m.x[2 * i] = __float_as_uint(first_of(m[i]));
        raw.m.x[2 * i + 1] = __float_as_uint(second_of(m[i]));
        raw.v.x[2 * i] = __float_as_uint(first_of(v[i]));
        raw.v.x[2 * i + 1] = __float_as_uint(second_of(v[i]));
      }
      st32(at_m + s * 4u, raw.m);
      st32(at_v + s * 4u, raw.v);
    }
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) pw[i] = __float_as_uint(p[i]);
    } else if (keeps) {                      // the nearest BF16 number (the larger of two as near) and what is left
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b0 = __float_as_uint(p[2 * i]), b1 = __float_as_uint(p[2 * i + 1]);
        pw[i] = __byte_perm(b0 + 0x8000u, b1 + 0x8000u, 0x7632);
        w[i] = __byte_perm(b0, b1, 0x5410);                               // bits - (p << 16), as 16 bits
      }
      *reinterpret_cast<uint4*>(at_rest + s * 2u) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) pw[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
    }
    adamw_write<F32, WIDE>(at_p + u * (kAdamwGroup * kSize), left0 - u * kAdamwGroup, lane, turn, pw);
  }
}

// A warp takes a group, a lane eight elements of it; a block finds its tensor by bisection in the kernel parameters.  184.5 M BF16 weights with their rest: 32-bit moments 726 us, 6.6 TB/s
// (the copy rate); 8-bit moments 500 us, 5.2 TB/s of 14.06 bytes a weight: some 66 instructions a weight (roots, quotients, codes) keep the issue slots two thirds busy.  One weight at
// a time through sqrt.rn and div.rn that took 820.  Six small vectors: 2 us.
// FP32 weights: 32-bit moments 766 us (28 bytes a weight, 6.7 TB/s); 8-bit moments, whose next group is neither staged nor in registers, 575 (16.06 bytes, 5.2 TB/s).
// LOOSE: some tensors of the launch are not on boundaries of eight elements.  Groups of those take twice the loads and the registers to have the next ones under way:
// three blocks an SM, where five of the others fit (8-bit moments, 184.5 M BF16 weights: 498 us with five, 580 with three; 16.8 M unaligned: 68, 61).
template <int FMT, bool LOOSE, int CAP>
__global__ void __launch_bounds__(256, FMT == GWS_ADAMW_F32 ? 4 : LOOSE ? 3 : 5) k_adamw(const __grid_constant__ AdamwBatch<CAP> b) {
  after_previous();
  __shared__ uint4 turns[8][FMT == GWS_ADAMW_8BIT ? 2 * kAdamwSlot / 16 : kAdamwGroup / 4];
  const AdamwArgs& a = b.a;
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.e[mid].block0 <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwRec& e = b.e[lo];
  AdamwScalars k;
  k.scale = a.grad_scale != nullptr ? *a.grad_scale : 1.0f;
  k.alpha = a.alpha;
  k.rho = a.rho;
  k.decay = e.decay;
  if (a.scalars != nullptr) {
    k.alpha = a.scalars[0];
    k.rho = a.scalars[1];
    k.decay = static_cast<float>(1.0 - static_cast<double>(a.scalars[2]) * static_cast<double>(e.decay));
  }
  auto sane = [](float x, float least, float most) { return x >= least && x <= most; };
  k.exact = sane(a.eps, 0x1p-40f, 0x1p30f) && sane(k.alpha, 0x1p-30f, 0x1p30f) && sane(k.rho, 0x1p-30f, 0x1p30f);
  uint4* turn = turns[threadIdx.x >> 5];
  const int64_t first = static_cast<int64_t>(blockIdx.x - e.block0) * a.per, groups = (e.n + kAdamwGroup - 1) / kAdamwGroup, end = min(groups, first + a.per);
  const bool f32 = (e.flags & kAdamwF32) != 0u;
  int64_t wide = (e.flags & kAdamwWide) != 0u ? min(end, e.n / kAdamwGroup) : first;          // groups up to here are whole and on boundaries
  if (wide < first) wide = first;
  const uint32_t n_wide = static_cast<uint32_t>(wide - first), n_rest = static_cast<uint32_t>(end - wide);
  if (f32) {
    adamw_run<FMT, LOOSE, true, true>(a, e, k, first, n_wide, turn);
    adamw_run<FMT, LOOSE, true, false>(a, e, k, wide, n_rest, turn);
  } else {
    adamw_run<FMT, LOOSE, false, true>(a, e, k, first, n_wide, turn);
    adamw_run<FMT, LOOSE, false, false>(a, e, k, wide, n_rest, turn);
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

// What 8-bit moments stand for: m and v = r r in FP32.  Memory-bound: 184.5 M in 275 us, 6.7 TB/s.
__global__ void __launch_bounds__(256) k_adamw_values(const uint8_t* codes, const float* units, int64_t total, float* m, float* v) {
  after_previous();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, s = t * 8;
  if (s >= total) return;
  const int64_t group = s / kAdamwGroup;
  F2 x[4], r[4];
  adamw_decode_m(*reinterpret_cast<const uint2*>(codes + s), units[group], x);
  adamw_decode_r(*reinterpret_cast<const uint2*>(codes + total + s), units[total / kAdamwGroup + group], r);
  V8 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const F2 q = mul2(r[i], r[i]);
    a.x[2 * i] = __float_as_uint(first_of(x[i]));
    a.x[2 * i + 1] = __float_as_uint(second_of(x[i]));
    b.x[2 * i] = __float_as_uint(first_of(q));
    b.x[2 * i + 1] = __float_as_uint(second_of(q));
  }
  st32(m + s, a);
  st32(v + s, b);
}

}  // namespace
