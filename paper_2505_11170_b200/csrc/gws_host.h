// Host helpers shared by the translation units of the operators around the sampling pass: argument checks, launches, SM count.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <cstring>
#include <initializer_list>

#include "gws.h"
#include "gws_internal.h"

namespace {

constexpr int64_t kMaxDim = 0x7FFFFFFFLL - 4096;
constexpr int kJobs = 256;                      // threads of the kernels that only move activations

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct Span {
  const void* p;
  int64_t bytes;
};
inline Span rows_of(const void* p, int64_t rows, int64_t cols, int64_t ld) { return {p, p == nullptr || rows == 0 || cols == 0 ? 0 : ((rows - 1) * ld + cols) * 2}; }
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.bytes > 0 && b.bytes > 0 && x < y + static_cast<uintptr_t>(b.bytes) && y < x + static_cast<uintptr_t>(a.bytes);
}
// No output may overlap an input or another output: blocks re-read inputs while others write.
inline bool clash(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
  for (const Span* a = outputs.begin(); a != outputs.end(); ++a) {
    for (const Span& b : inputs)
      if (overlap(*a, b)) return true;
    for (const Span* b = a + 1; b != outputs.end(); ++b)
      if (overlap(*a, *b)) return true;
  }
  return false;
}

inline int check_dims(int64_t a, int64_t b, int64_t c) {
  if (a < 0 || b < 0 || c < 0) return GWS_ERR_SHAPE;
  return a > kMaxDim || b > kMaxDim || c > kMaxDim ? GWS_ERR_LIMIT : GWS_OK;
}

// Every launch may become resident while the kernel before it on the stream drains (after_previous in the kernels): with ordinary
// launches calls of a few us follow each other 2 us further apart (517 tokens, 768 x 2730: 12.3 against 10.4 us a call).
template <class... P, class... A>
int launch(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t s, const char* what, const A&... args) {
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = cluster;
    attr[cfg.numAttrs].val.clusterDim.y = 1;
    attr[cfg.numAttrs++].val.clusterDim.z = 1;
  }
  const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
  if (err != cudaSuccess) { (void)cudaGetLastError(); return gws::report_cuda(err, what); }
  return gws::finish_launch(what);
}

inline unsigned blocks_for(int64_t items, int64_t per_block) { return static_cast<unsigned>((items + per_block - 1) / per_block); }

inline int sm_count() {
  static std::atomic<int> known[64];             // per device
  int dev = 0, n = 0;
  const bool current = cudaGetDevice(&dev) == cudaSuccess;
  if (current && dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) != 0) return n;
  if (!current || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 2) {
    (void)cudaGetLastError();
    return 148;
  }
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

inline bool workspace_ok(const void* p, size_t have, int64_t need) { return need == 0 || (p != nullptr && on(p, 256) && have >= static_cast<size_t>(need)); }

}  // namespace
