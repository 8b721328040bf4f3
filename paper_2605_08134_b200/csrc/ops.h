// What the stand-alone operators of dare_ops.h share between their translation units.
//
// Their kernels are launched while the kernel in front of them may still run (launch_pdl), and any operand may be what that one writes.
// So nothing of an operand is read before pdl_wait() (the lengths in attention's merge: before its own, behind the one of the kernel in
// front), and none of it by a read-only load: those are for data that does not change while the kernel lives, and may be moved in
// front of the wait.
#pragma once

#include "dare_internal.h"
#include "dare_ops.h"

namespace dare {

// Strides that no memory reaches are refused: their products with counts stay inside 64 bits.
constexpr long long kMaxStride = 1ll << 38;
inline bool stride_ok(long long s) { return s >= 0 && s < kMaxStride; }

// Rows (stride `row`) of heads (stride `head`) of `width` elements, written by a launch: no two in one place.
inline bool places_apart(long long rows, long long row, long long heads, long long head, long long width) {
  if (rows <= 1) return heads <= 1 || head >= width;
  if (heads <= 1) return row >= width;
  return head <= row ? head >= width && row >= (heads - 1) * head + width : row >= width && head >= (rows - 1) * row + width;
}

// rope.cu
cudaError_t launch_rope_freq_table(const dare_rope_config_t& c, float* table, long long positions, cudaStream_t st);
cudaError_t launch_rope(const dare_rope_apply_t& c, const void* x, const int* positions, const float* table, void* y, int* status,
                        cudaStream_t st);

}  // namespace dare
