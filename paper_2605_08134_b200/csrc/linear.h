// y = act(x W^T + bias) + resid (dare_ops.h): what its kernels share.
#pragma once

#include "ops.h"

namespace dare {

struct LinearParams {
  const void* x;
  const void* w;
  const float* bias;         // or nullptr
  const void* resid;         // or nullptr
  void* y;
  long long x_row, w_row, resid_row, y_row;
  int rows, n, k, act;
  int tile_rows;             // rows of a tile there: a multiple of 16, at most 128
  int splits;                // float32 on the tensor cores: CTAs that share a tile's k-elements (1, 2, 4 or 8)
  int* status;
};

#ifdef __CUDACC__
// v[i] = act(v[i]); one switch for all of them.  FAST (bf16 results): exponential and quotient on the special-function unit.  __expf(x) is off
// by 2 + 1.173 |x| units at most, so SiLU and tanh GELU are right to 2^-15 of their value wherever that is no underflow, far below a
// bf16 result's rounding (with the exact ones 37 rows of 12288 outputs took 4 us longer).  1 + erf cancels for negative v: 2^-24 |v| then,
// which below v = -4.5 is more than a bf16 result's rounding (results under 2e-5); erfc would be right there, and take up to
// 35 % of a product of few k-elements (8192 x 512 x 512 13.1 / 17.7 us).  float32 has erfc, 2 % of 601 x 1024 x 1000, and no tanh,
// which cancels the same way.
template <bool FAST, int N>
__device__ __forceinline__ void activate(float (&v)[N], int act) {
  switch (act) {
    case DARE_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];                                     // (NaN stays)
      break;
    case DARE_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = FAST ? __fdividef(v[i], 1.f + __expf(-v[i])) : v[i] / (1.f + expf(-v[i]));
      break;
    case DARE_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 0.5f * v[i] * (FAST ? 1.f + erff(v[i] * 0.70710678118654752f) : erfcf(v[i] * -0.70710678118654752f));
      break;
    case DARE_ACT_GELU_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) {                        // 0.5 (1 + tanh(u)) = 1 / (1 + e^-2u)
        const float u = 0.79788456080286536f * (v[i] + 0.044715f * v[i] * v[i] * v[i]);
        v[i] = FAST ? __fdividef(v[i], 1.f + __expf(-2.f * u)) : v[i] / (1.f + expf(-2.f * u));
      }
      break;
    default: break;
  }
}
#endif

// bf16 on the tensor cores (linear_tc.cu): x, w 16-byte aligned, strides multiples of 8
cudaError_t launch_linear_tc(const LinearParams& p, cudaStream_t st);
// float32 on the tensor cores, operands in three bf16 parts (gemm_f32.cu): x, w 16-byte aligned, k and strides multiples of 4
cudaError_t launch_linear_f32(const LinearParams& p, cudaStream_t st);
// either type on the CUDA cores, any alignment (linear.cu)
cudaError_t launch_linear_simt(const LinearParams& p, bool bf16, cudaStream_t st);

}  // namespace dare
