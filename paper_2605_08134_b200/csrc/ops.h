// What the stand-alone operators of dare_ops.h share between their translation units.
#pragma once

#include "dare_internal.h"
#include "dare_ops.h"

namespace dare {

// rope.cu
cudaError_t launch_rope_freq_table(const dare_rope_config_t& c, float* table, long long positions, cudaStream_t st);
cudaError_t launch_rope(const dare_rope_apply_t& c, const void* x, const int* positions, const float* table, void* y, int* status,
                        cudaStream_t st);

}  // namespace dare
