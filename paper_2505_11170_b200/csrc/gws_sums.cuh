// The join of column sums that blocks have taken over their shares of the rows.
#pragma once
#include <stdint.h>

#include "gws_act8.cuh"

namespace {

// Column sums of the parts of `outs` vectors, in order: part [parts, outs, cols] -> out[k] [cols].  A warp takes eight runs of 32 columns' parts, the warps of a
// block join theirs in order.
__global__ void __launch_bounds__(256) k_column_sums(const float* part, uint32_t parts, int64_t cols, uint32_t outs, void* out0, void* out1, int32_t f32) {
  after_previous();
  __shared__ float sums[8][32];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, strips = static_cast<uint32_t>((cols + 31) / 32), which = blockIdx.x / strips;
  const int64_t col = static_cast<int64_t>(blockIdx.x - which * strips) * 32 + lane;
  const uint32_t per = (parts + 7u) / 8u, end = min(parts, (warp + 1u) * per);
  float t = 0.0f;
  if (col < cols) {
#pragma unroll 8
    for (uint32_t k = warp * per; k < end; ++k) t += part[(static_cast<int64_t>(k) * outs + which) * cols + col];
  }
  sums[warp][lane] = t;
  __syncthreads();
  if (warp != 0u || col >= cols) return;
#pragma unroll
  for (uint32_t w = 1; w < 8u; ++w) t += sums[w][lane];
  void* out = which == 0u ? out0 : out1;
  if (out == nullptr) return;
  if (f32) static_cast<float*>(out)[col] = t;
  else static_cast<uint16_t*>(out)[col] = static_cast<uint16_t>(pack_bf16(t, 0.0f));
}

}  // namespace
