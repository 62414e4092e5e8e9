// 8-bit activation checkpoints: the codec and the kernels that only move activations.
//
// A group of 32 elements along a row shares one power-of-two scale 2^(s - 127), s = max(E - emax, 0), E the biased exponent
// of the group's largest magnitude; s = 255 marks a group with a value that is not finite and restores as NaN.
//   INT8   emax 0, code c = rne(64 x / 2^(s-127)) clamped to [-127, 127], value c / 64 * 2^(s-127)
//   E4M3   emax 8, code = rne of x / 2^(s-127) onto the E4M3 grid, clamped to +-448
// Scaling by a power of two is exact, so each element is rounded once, and every restored INT8 value is a BF16 number (7 bits
// and a sign).  INT8 spaces its codes evenly: its error is at most 1/128 of the group's largest magnitude (half a step; a
// whole one where the largest itself is clamped), a third of E4M3's on normal data; E4M3 keeps small elements beside a large one.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "gws.h"

namespace {

constexpr int kGroup = 32;               // elements per scale
constexpr uint32_t kNanByte = 255u;

struct V8 { uint32_t x[8]; };            // 32 bytes

__device__ __forceinline__ V8 ld32(const void* p) {
  V8 v;
  asm volatile("ld.global.nc.v8.u32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v.x[0]), "=r"(v.x[1]), "=r"(v.x[2]), "=r"(v.x[3]), "=r"(v.x[4]), "=r"(v.x[5]), "=r"(v.x[6]), "=r"(v.x[7])
               : "l"(p));
  return v;
}
__device__ __forceinline__ void st32(void* p, const V8& v) {
  asm volatile("st.global.v8.u32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v.x[0]), "r"(v.x[1]), "r"(v.x[2]), "r"(v.x[3]),
               "r"(v.x[4]), "r"(v.x[5]), "r"(v.x[6]), "r"(v.x[7])
               : "memory");
}

// These kernels are launched programmatically: a kernel's blocks may become resident while the one before it on the stream drains, and
// touch global memory only once that one has completed.  Every kernel of this file set passes here before its first access, so
// the order along the stream holds transitively.  The next kernel may follow once this one has seen its predecessor end (as in the
// kernels of the sampling pass), so that there are never more than two of the library's kernels of a stream on the device: blocks of a
// third would hold shared memory, tensor memory and barriers without a use for them.
__device__ __forceinline__ void after_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ float bf16_lo(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// 2^(byte - 127) as a float, exactly; 2^-127 is a subnormal.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 0u ? 0x00400000u : byte == kNanByte ? 0x7FC00000u : byte << 23);
}
// 2^(127 - byte); byte = 254 gives the subnormal 2^-127.
__device__ __forceinline__ float inverse_scale_of(uint32_t byte) { return __uint_as_float(byte >= 254u ? 0x00400000u : (254u - byte) << 23); }
// 2^(byte - 133): the weight of one INT8 step, exactly (subnormal below byte 7).
__device__ __forceinline__ float step_of(uint32_t byte) {
  return __uint_as_float(byte == kNanByte ? 0x7FC00000u : byte >= 7u ? (byte - 6u) << 23 : 0x10000u << byte);
}

// Scale byte of a group from the FP32 bit pattern of its largest magnitude (NaN patterns compare above infinity).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits, int format) {
  if (top_bits >= 0x7F800000u) return kNanByte;
  const uint32_t e = top_bits >> 23, emax = format == GWS_ACT8_E4M3 ? 8u : 0u;
  return e > emax ? e - emax : 0u;
}

// Codes of four elements.  x * inv is exact (a power of two, and |x * inv| < 2); the FMA with 1.5 * 2^23 rounds 64 x once, to
// nearest even, and leaves the integer in the low byte.
__device__ __forceinline__ uint32_t encode4_int8(float a, float b, float c, float d, float inv) {
  const float magic = 12582912.0f;
  auto one = [&](float v) { return __float_as_uint(fminf(fmaxf(__fmaf_rn(v * inv, 64.0f, magic), magic - 127.0f), magic + 127.0f)); };
  return __byte_perm(__byte_perm(one(a), one(b), 0x0040), __byte_perm(one(c), one(d), 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t encode4_e4m3(float a, float b, float c, float d, float inv) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// The four values of a word of codes.  `unit` is step_of (INT8) or scale_of (E4M3) of the group's byte.
__device__ __forceinline__ void decode4_int8(uint32_t codes, float unit, float* v) {
  const uint32_t u = codes ^ 0x80808080u;        // c + 128 in every byte; 0x4B0000uu is the float 2^23 + c + 128
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540u + i)) - 8388736.0f) * unit;
}
__device__ __forceinline__ void decode4_e4m3(uint32_t codes, float unit, float* v) {
  const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes & 0xFFFFu), __NV_E4M3);
  const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes >> 16), __NV_E4M3);
  const float2 a = __half22float2(__half2(lo)), b = __half22float2(__half2(hi));
  v[0] = a.x * unit; v[1] = a.y * unit; v[2] = b.x * unit; v[3] = b.y * unit;
}

template <int FMT>
__device__ __forceinline__ float unit_of(uint32_t byte) { return FMT == GWS_ACT8_INT8 ? step_of(byte) : scale_of(byte); }
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t codes, float unit, float* v) {
  if (FMT == GWS_ACT8_INT8) decode4_int8(codes, unit, v);
  else decode4_e4m3(codes, unit, v);
}
template <int FMT>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
  return FMT == GWS_ACT8_INT8 ? encode4_int8(a, b, c, d, inv) : encode4_e4m3(a, b, c, d, inv);
}

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A whole group held by one thread.  For INT8 nearly every group needs one FMA per element: a factor of 64 * 2^(127 - byte) fits a float
// for bytes above 6, and only a largest magnitude of 255/128 or more of its power of two rounds up to 128.  The other groups (1 in 128
// on smooth data, subnormal ones, and those that hold a NaN or infinity) bring their elements into that form first.
template <int FMT>
__device__ __forceinline__ uint32_t encode_group(const float (&v)[kGroup], V8& codes) {
  float most = fabsf(v[0]);
#pragma unroll
  for (int i = 1; i < kGroup; ++i) most = max_nan(most, fabsf(v[i]));
  const uint32_t top = __float_as_uint(most), byte = scale_byte(top, FMT);
  if (FMT == GWS_ACT8_E4M3) {
    const float inv = inverse_scale_of(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) codes.x[i] = byte == kNanByte ? 0u : encode4_e4m3(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inv);
    return byte;
  }
  float x[kGroup], to64 = __uint_as_float((260u - byte) << 23);
#pragma unroll
  for (int i = 0; i < kGroup; ++i) x[i] = v[i];
  if (byte < 7u || byte == kNanByte || (top & 0x7FFFFFu) >= 0x7F0000u) {
    const float inv = inverse_scale_of(byte), lim = byte == kNanByte ? 0.0f : 127.0f / 64.0f;
    to64 = 64.0f;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) x[i] = fminf(fmaxf(v[i] * inv, -lim), lim);      // a NaN becomes -0
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = __float_as_uint(__fmaf_rn(x[4 * i + e], to64, 12582912.0f));
    codes.x[i] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
  }
  return byte;
}

struct Act8View {                 // a checkpoint in memory
  uint8_t* codes;                 // [rows, ld]
  uint8_t* scales;                // [rows, ld / 32]
  int64_t ld;                     // cols rounded up to 32
};

// ---- save / load -------------------------------------------------------------------------------------------------------
// Memory-bound: 2 bytes of activation and 1 + 1/32 of checkpoint per element.  A thread takes a whole group - two 32-byte
// accesses on the BF16 side, one on the code side, one scale byte - so the maximum needs no exchange between lanes.
// 16384 x 5632: save and load together 83.5 us, 6.7 TB/s (a plain copy moves 6.5).  One token: latency, 2.5 us each.

template <int FMT>
__global__ void __launch_bounds__(256) k_act8_save(const uint16_t* x, int64_t ldx, Act8View c, int64_t groups, uint32_t per_row) {
  after_previous();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (t >= groups) return;
  int64_t at = t * kGroup;
  if (ldx != c.ld) {
    const int64_t row = t / per_row;
    at = row * ldx + (t - row * per_row) * kGroup;
  }
  const V8 a = ld32(x + at), b = ld32(x + at + 16);
  float v[kGroup];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[2 * i] = bf16_lo(a.x[i]);
    v[2 * i + 1] = bf16_hi(a.x[i]);
    v[16 + 2 * i] = bf16_lo(b.x[i]);
    v[17 + 2 * i] = bf16_hi(b.x[i]);
  }
  V8 codes;
  c.scales[t] = static_cast<uint8_t>(encode_group<FMT>(v, codes));
  st32(c.codes + t * kGroup, codes);
}

template <int FMT>
__device__ __forceinline__ void load_group(const Act8View& c, uint16_t* x, int64_t t, int64_t at) {
  const V8 codes = ld32(c.codes + t * kGroup);
  const float unit = unit_of<FMT>(c.scales[t]);
  V8 out[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[4];
    decode4<FMT>(codes.x[i], unit, v);
    out[i >> 2].x[2 * (i & 3)] = pack_bf16(v[0], v[1]);
    out[i >> 2].x[2 * (i & 3) + 1] = pack_bf16(v[2], v[3]);
  }
  st32(x + at, out[0]);
  st32(x + at + 16, out[1]);
}
template <int FMT>
__global__ void __launch_bounds__(256) k_act8_load(Act8View c, uint16_t* x, int64_t ldx, int64_t groups, uint32_t per_row) {
  after_previous();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (t >= groups) return;
  int64_t at = t * kGroup;
  if (ldx != c.ld) {
    const int64_t row = t / per_row;
    at = row * ldx + (t - row * per_row) * kGroup;
  }
  load_group<FMT>(c, x, t, at);
}

// t / d; one 32-bit division wherever the numbers allow it (a 64-bit one is a routine of some hundred instructions).
__device__ __forceinline__ int64_t quotient(int64_t t, uint32_t d) {
  return (t >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(t) / d) : t / static_cast<int64_t>(d);
}

// The general forms: any width, row stride and 2-byte alignment of the BF16 side.
// Save: four lanes share a group, eight elements each, read one by one (a warp's reads cover 512 neighbouring bytes) and written as
// one 8-byte word of codes; columns past the width become zero codes.
template <int FMT>
__global__ void __launch_bounds__(256) k_act8_save_any(const uint16_t* x, int64_t ldx, Act8View c, int64_t quarters, uint32_t per_row, int64_t cols) {
  after_previous();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const bool real = t < quarters;
  const int64_t row = real ? quotient(t, per_row) : 0, col = real ? (t - row * per_row) * 8 : cols;
  const uint16_t* p = x + row * ldx + col;
  float v[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? __uint_as_float(static_cast<uint32_t>(p[i]) << 16) : 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
  if (!real) return;
  const uint32_t byte = scale_byte(top, FMT);
  const float inv = inverse_scale_of(byte);
  const uint2 codes = byte == kNanByte ? make_uint2(0u, 0u) : make_uint2(encode4<FMT>(v[0], v[1], v[2], v[3], inv), encode4<FMT>(v[4], v[5], v[6], v[7], inv));
  *reinterpret_cast<uint2*>(c.codes + t * 8) = codes;
  if ((t & 3) == 0) c.scales[t >> 2] = static_cast<uint8_t>(byte);
}

// Load: a warp takes a run of 256 columns of a row, a lane eight neighbouring ones, which pass through shared memory so that rows of
// any alignment are written one element at a time but side by side.
template <int FMT>
__global__ void __launch_bounds__(256) k_act8_load_any(Act8View c, uint16_t* x, int64_t ldx, int64_t runs, uint32_t runs_per_row, int64_t cols) {
  after_previous();
  __shared__ uint4 turn[8][32];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 8 + warp;
  if (t >= runs) return;
  const int64_t row = quotient(t, runs_per_row), run = (t - row * runs_per_row) * 256, at = row * c.ld + run + lane * 8;
  if (run + lane * 8 < c.ld) {
    const uint2 codes = *reinterpret_cast<const uint2*>(c.codes + at);
    const float unit = unit_of<FMT>(c.scales[at >> 5]);
    float v[8];
    decode4<FMT>(codes.x, unit, v);
    decode4<FMT>(codes.y, unit, v + 4);
    turn[warp][lane] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
  __syncwarp();
  const uint16_t* side = reinterpret_cast<const uint16_t*>(turn[warp]) + lane;
  uint16_t* to = x + row * ldx + run + lane;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (run + lane + 32 * i < cols) to[32 * i] = side[32 * i];
}

// ---- operands made ready for the tensor maps ---------------------------------------------------------------------------------
// BF16 rows brought onto 16-byte boundaries (up to three matrices: an input and both weights; a thread writes 16 bytes from eight
// reads, columns past the width are zero) and a checkpoint restored into rows of whole groups (a thread a group), in one launch, so that
// the small ones run beside each other.  2047 x 1023 and twice 2729 x 1023: 8.4 us cold, 3.7 TB/s.
struct Prep {
  const uint16_t* from[3];
  uint16_t* to[3];
  int64_t ld_from[3], cols[3];
  int64_t end[3];               // threads of the first 1, 2, 3 matrices
  uint32_t per_row[3];          // 16-byte units in a row of the copy
  uint32_t move_blocks, restore_blocks;
  Act8View kept;
  uint16_t* restored;           // [rows, ld_restored]
  int64_t ld_restored, groups;
  int32_t format;
};
__device__ __forceinline__ void move_unit(const Prep& m, int64_t t) {
  const int w = t >= m.end[1] ? 2 : t >= m.end[0] ? 1 : 0;
  if (t >= m.end[2]) return;
  const uint16_t* from = w == 0 ? m.from[0] : w == 1 ? m.from[1] : m.from[2];
  uint16_t* to = w == 0 ? m.to[0] : w == 1 ? m.to[1] : m.to[2];
  const int64_t ld = w == 0 ? m.ld_from[0] : w == 1 ? m.ld_from[1] : m.ld_from[2], cols = w == 0 ? m.cols[0] : w == 1 ? m.cols[1] : m.cols[2];
  const uint32_t per_row = w == 0 ? m.per_row[0] : w == 1 ? m.per_row[1] : m.per_row[2];
  t -= w == 0 ? 0 : w == 1 ? m.end[0] : m.end[1];
  const int64_t row = quotient(t, per_row), col = (t - row * per_row) * 8;
  const uint16_t* p = from + row * ld + col;
  uint32_t v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? p[i] : 0u;
  *reinterpret_cast<uint4*>(to + t * 8) = make_uint4(v[0] | (v[1] << 16), v[2] | (v[3] << 16), v[4] | (v[5] << 16), v[6] | (v[7] << 16));
}
// The first blocks of a launch of 256 threads; true if this block was one of them.
__device__ __forceinline__ bool prepare(const Prep& m) {
  if (blockIdx.x >= m.move_blocks + m.restore_blocks) return false;
  if (blockIdx.x < m.move_blocks) {
    move_unit(m, static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x);
    return true;
  }
  const int64_t t = static_cast<int64_t>(blockIdx.x - m.move_blocks) * 256 + threadIdx.x;
  if (t >= m.groups) return true;
  int64_t at = t * kGroup;
  if (m.ld_restored != m.kept.ld) at += quotient(t, static_cast<uint32_t>(m.kept.ld / kGroup)) * (m.ld_restored - m.kept.ld);
  if (m.format == GWS_ACT8_INT8) load_group<GWS_ACT8_INT8>(m.kept, m.restored, t, at);
  else load_group<GWS_ACT8_E4M3>(m.kept, m.restored, t, at);
  return true;
}
__global__ void __launch_bounds__(256) k_prepare(const __grid_constant__ Prep m) {
  after_previous();
  (void)prepare(m);
}

}  // namespace
