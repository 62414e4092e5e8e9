// Host helpers of gws_api.cu that the other translation units of the library share.
#pragma once
#include <cuda_runtime.h>

namespace gws {

// Counts a kernel launch for gws_launch_count and turns the runtime's answer into a status.
int finish_launch(const char* what);
// Records a CUDA error for gws_last_cuda_error; returns GWS_ERR_CUDA.
int report_cuda(cudaError_t err, const char* what);
// The same for an error that comes with a text of its own.
int report_text(const char* text);

}  // namespace gws
