// What the library's translation units share on the host side.
#pragma once

#include <cuda_runtime.h>

namespace sq_host {

// Records the text for squant_last_cuda_error() and returns SQUANT_ERR_CUDA.
int cuda_failed(cudaError_t e, const char *what);
// One more kernel for squant_launch_count().
void count_launch();
// Whether a kernel of the linear operators gave up a bounded wait on the current device; clears the record.
cudaError_t take_linear_status(int *status);
// Failed checks of their checked build and the first one's site; clears both.
cudaError_t take_linear_violations(unsigned *count, int *site);

}  // namespace sq_host
