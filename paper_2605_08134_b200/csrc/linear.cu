// y = act(x W^T + bias) + resid: the CUDA-core kernel (float32 with few rows or other alignments, bf16 whose rows TMA cannot read), and
// the C entry that chooses (dare_ops.h).
#include "linear.h"
#include "tc_ptx.cuh"

namespace dare {

using namespace ptx;

namespace {

// A warp takes kOut outputs and up to MT rows: its lanes share the k-elements, four a lane and step, and add their sums up at the end,
// halving the set of sums a lane holds at each step of the exchange.  W is read once for MT rows (blockIdx.x counts groups of rows:
// CTAs side by side take the same rows of W, which the second finds in the L2).  Every W element a lane has feeds MT multiplications
// and every x element kOut, so at 16 rows the FMA pipe and the L1 that feeds it are about even (64 cycles against 80 a step).
constexpr int kOut = 4, kWarps = 8, kThreads = kWarps * 32;

template <typename T, bool WIDE>
__device__ __forceinline__ float4 load4(const T* row, int k, int K) {
  if constexpr (WIDE) {                                    // (K a multiple of 4: all four or none)
    if (k >= K) return make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (sizeof(T) == 4) return *reinterpret_cast<const float4*>(row + k);
    else {
      const uint2 raw = *reinterpret_cast<const uint2*>(row + k);
      const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.x));
      const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.y));
      return make_float4(a.x, a.y, b.x, b.y);
    }
  }
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (k < K) v.x = (float)row[k];
  if (k + 1 < K) v.y = (float)row[k + 1];
  if (k + 2 < K) v.z = (float)row[k + 2];
  if (k + 3 < K) v.w = (float)row[k + 3];
  return v;
}

// Sums over the lanes of N values each: afterwards lane l holds max(1, N / 32) of them, the first of which is value *first.
template <int N, int O>
__device__ __forceinline__ void reduce_lanes(float* v, int* first) {
  if constexpr (O > 0) {
    const int lane = threadIdx.x & 31;
    if constexpr (N > 1) {
      const bool up = (lane & O) != 0;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float keep = up ? v[i + N / 2] : v[i], give = up ? v[i] : v[i + N / 2];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, O);
      }
      if (up) *first += N / 2;
      reduce_lanes<N / 2, O / 2>(v, first);
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], O);
      reduce_lanes<1, O / 2>(v, first);
    }
  }
}

template <typename T, int MT, bool WIDE>
__global__ void __launch_bounds__(kThreads, 2) linear_rows_kernel(const LinearParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m0 = (int)blockIdx.x * MT;
  const long long n0 = ((long long)blockIdx.y + (long long)blockIdx.z * gridDim.y) * (kWarps * kOut) + warp * kOut;
  if (n0 >= p.n) return;
  const T* x[MT];
  const T* w[kOut];
#pragma unroll
  for (int i = 0; i < MT; ++i) x[i] = reinterpret_cast<const T*>(p.x) + (long long)min(m0 + i, p.rows - 1) * p.x_row;
#pragma unroll
  for (int j = 0; j < kOut; ++j) w[j] = reinterpret_cast<const T*>(p.w) + min(n0 + j, (long long)p.n - 1) * p.w_row;
  float acc[kOut * MT];
#pragma unroll
  for (int i = 0; i < kOut * MT; ++i) acc[i] = 0.f;
#pragma unroll 2
  for (int k = lane * 4; k < p.k; k += 128) {
    float4 a[kOut];
#pragma unroll
    for (int j = 0; j < kOut; ++j) a[j] = load4<T, WIDE>(w[j], k, p.k);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float4 b = load4<T, WIDE>(x[i], k, p.k);
#pragma unroll
      for (int j = 0; j < kOut; ++j) {
        float& s = acc[i * kOut + j];
        s = fmaf(a[j].x, b.x, s);
        s = fmaf(a[j].y, b.y, s);
        s = fmaf(a[j].z, b.z, s);
        s = fmaf(a[j].w, b.w, s);
      }
    }
  }
  constexpr int N = kOut * MT, LEFT = N > 32 ? N / 32 : 1;
  int first = 0;
  reduce_lanes<N, 16>(acc, &first);
  // (fewer values than lanes: the lanes with the same ones differ in the low bits, the first of them writes)
  if (N < 32 && (lane & (32 / (N < 32 ? N : 32) - 1)) != 0) return;
  float v[LEFT];
#pragma unroll
  for (int i = 0; i < LEFT; ++i) {
    const int n = (int)n0 + (first + i) % kOut;
    v[i] = acc[i] + (p.bias && n < p.n ? p.bias[n] : 0.f);
  }
  activate(v, p.act);
#pragma unroll
  for (int i = 0; i < LEFT; ++i) {
    const int m = m0 + (first + i) / kOut, n = (int)n0 + (first + i) % kOut;
    if (m < p.rows && n < p.n) {
      if (p.resid) v[i] += (float)reinterpret_cast<const T*>(p.resid)[(long long)m * p.resid_row + n];
      reinterpret_cast<T*>(p.y)[(long long)m * p.y_row + n] = (T)v[i];
    }
  }
}

template <typename T, int MT>
cudaError_t launch_rows_as(const LinearParams& p, bool wide, cudaStream_t st) {
  const long long n_ctas = ((long long)p.n + kWarps * kOut - 1) / (kWarps * kOut), nz = (n_ctas + 65534) / 65535;
  return launch_pdl(wide ? linear_rows_kernel<T, MT, true> : linear_rows_kernel<T, MT, false>, dim3((unsigned)((p.rows + MT - 1) / MT), (unsigned)((n_ctas + nz - 1) / nz), (unsigned)nz),
                    dim3(kThreads), 0, st, 1, p);
}
template <typename T>
cudaError_t launch_rows(const LinearParams& p, cudaStream_t st) {
  const uintptr_t mask = 4 * sizeof(T) - 1;
  const bool wide = p.k % 4 == 0 && p.x_row % 4 == 0 && p.w_row % 4 == 0 && (reinterpret_cast<uintptr_t>(p.x) & mask) == 0 &&
                    (reinterpret_cast<uintptr_t>(p.w) & mask) == 0;
  if (p.rows == 1) return launch_rows_as<T, 1>(p, wide, st);
  if (p.rows == 2) return launch_rows_as<T, 2>(p, wide, st);
  if (p.rows <= 4) return launch_rows_as<T, 4>(p, wide, st);
  if (p.rows <= 8) return launch_rows_as<T, 8>(p, wide, st);
  return launch_rows_as<T, 16>(p, wide, st);
}
}  // namespace

cudaError_t launch_linear_simt(const LinearParams& p, bool bf16, cudaStream_t st) {
  return bf16 ? launch_rows<__nv_bfloat16>(p, st) : launch_rows<float>(p, st);
}

}  // namespace dare

using namespace dare;

extern "C" dare_status_t dare_linear(const dare_linear_config_t* c, const void* x, const void* w, const float* bias, const void* resid,
                                     void* y, int32_t* status, void* cuda_stream) {
  if (!c || c->struct_size != sizeof(dare_linear_config_t)) return DARE_ERR_INVALID_ARG;
  if (c->dtype != DARE_F32 && c->dtype != DARE_BF16) return DARE_ERR_INVALID_ARG;
  if (c->activation < DARE_ACT_NONE || c->activation > DARE_ACT_GELU_TANH || c->reserved != 0) return DARE_ERR_INVALID_ARG;
  if (c->rows < 0 || c->rows > (int64_t)1 << 24 || c->in_features <= 0 || c->in_features > 1 << 20 || c->out_features <= 0 ||
      c->out_features > 1 << 24 || c->rows * c->out_features > (int64_t)1 << 38)
    return DARE_ERR_SHAPE;
  if (c->x_row < 0 || c->w_row < 0 || c->resid_row < 0 || c->y_row < 0 || c->x_row >= (int64_t)1 << 38 || c->w_row >= (int64_t)1 << 38)
    return DARE_ERR_SHAPE;
  if (c->rows > 1 && c->y_row < c->out_features) return DARE_ERR_SHAPE;        // (rows of y in one place would be written twice)
  if (c->rows == 0) return DARE_OK;
  if (!x || !w || !y) return DARE_ERR_INVALID_ARG;
  if (resid == y && c->rows > 1 && c->resid_row != c->y_row) return DARE_ERR_INVALID_ARG;
  auto low = [](const void* p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; };
  const uintptr_t elem = c->dtype == DARE_BF16 ? 1u : 3u;
  if (low(x, elem) || low(w, elem) || low(resid, elem) || low(y, elem) || low(bias, 3u)) return DARE_ERR_ALIGN;

  LinearParams p = {};
  p.x = x; p.w = w; p.bias = bias; p.resid = resid; p.y = y;
  p.x_row = c->x_row; p.w_row = c->w_row; p.resid_row = c->resid_row; p.y_row = c->y_row;
  p.rows = (int)c->rows; p.n = c->out_features; p.k = c->in_features; p.act = c->activation; p.status = status;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  // a stride that 16-byte accesses can follow (one row has none); rows that repeat (stride 0) stay off the tensor maps
  auto strides = [&](int64_t rows, int64_t row, int per16) { return rows == 1 || (row > 0 && row % per16 == 0); };
  cudaError_t e;
  if (c->dtype == DARE_BF16) {
    const bool tc = !low(x, 15u) && !low(w, 15u) && strides(c->rows, c->x_row, 8) && strides(c->out_features, c->w_row, 8);
    e = tc ? launch_linear_tc(p, st) : launch_linear_simt(p, true, st);
  } else {
    const bool aligned = !low(x, 15u) && !low(w, 15u) && c->in_features % 4 == 0 && strides(c->rows, c->x_row, 4) &&
                         strides(c->out_features, c->w_row, 4);
    // CUDA cores: 80 cycles a step of 16 rows x 4 outputs x 128 elements on an SM; tensor cores: a tile of 128 rows x 64 outputs takes 4.5 us
    // and 1.1 us a block of 64 elements.
    const float here = (float)((c->rows + 15) / 16) * (float)((c->out_features + 3) / 4) * (float)((c->in_features + 127) / 128) *
                           (80.f / 1900.f / (float)kSms) + 4.f;
    const int64_t tiles = (c->rows + 127) / 128 * ((c->out_features + 63) / 64);
    const float there = (float)((tiles + kSms - 1) / kSms) * (4.5f + 1.1f * (float)((c->in_features + 63) / 64)) + 2.f;
    e = aligned && there < here ? launch_linear_f32(p, st) : launch_linear_simt(p, false, st);
  }
  if (e != cudaSuccess) { cudaGetLastError(); return DARE_ERR_CUDA; }
  return DARE_OK;
}
