// The join of column sums that blocks have taken over their shares of the rows.
#pragma once
#include <stdint.h>

#include "gws_act8.cuh"

namespace {

// Column sums of the parts of `outs` vectors, in order: part [parts, outs, cols] -> out[k] [cols].  A warp of a block takes a run of the parts of 32 columns, and the runs are
// joined in their order.  It is latency: some 300 parts of 2 x 2048 columns (4.8 MB, out of L2) on 32 warps.
constexpr uint32_t kSumWarps = 32, kSumBatch = 10;          // loads of a warp under way: all that it has of 320 parts
__global__ void __launch_bounds__(32 * kSumWarps) k_column_sums(const float* part, uint32_t parts, int64_t cols, uint32_t outs, void* out0, void* out1, int32_t f32) {
  after_previous();
  __shared__ float sums[kSumWarps][33];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, strips = static_cast<uint32_t>((cols + 31) / 32), which = blockIdx.x / strips;
  const int64_t col = static_cast<int64_t>(blockIdx.x - which * strips) * 32 + lane;
  const uint32_t per = (parts + kSumWarps - 1u) / kSumWarps, end = min(parts, (warp + 1u) * per);
  float t = 0.0f;
  if (col < cols) {
    const float* from = part + (static_cast<int64_t>(warp) * per * outs + which) * cols + col;
    const int64_t step = static_cast<int64_t>(outs) * cols;
#pragma unroll 1
    for (uint32_t k = warp * per; k < end; k += kSumBatch) {
      float v[kSumBatch];
#pragma unroll
      for (uint32_t i = 0; i < kSumBatch; ++i, from += step) v[i] = k + i < end ? __ldg(from) : 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < kSumBatch; ++i) t += v[i];
    }
  }
  sums[warp][lane] = t;
  __syncthreads();
  if (warp != 0u) return;
  t = 0.0f;
#pragma unroll
  for (uint32_t w = 0; w < kSumWarps; ++w) t += sums[w][lane];
  void* out = which == 0u ? out0 : out1;
  if (out == nullptr || col >= cols) return;
  if (f32) static_cast<float*>(out)[col] = t;
  else static_cast<uint16_t*>(out)[col] = static_cast<uint16_t>(pack_bf16(t, 0.0f));
}

}  // namespace
