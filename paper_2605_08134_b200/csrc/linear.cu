// y = act(x W^T + bias) + resid: the CUDA-core kernel (float32 with few rows or other alignments, bf16 whose rows TMA cannot read), and
// the C entry that chooses (dare_ops.h).
#include "linear.h"
#include "tc_ptx.cuh"

namespace dare {

using namespace ptx;

namespace {

// ------------------------------------------------------------------------------------------------ few rows
// At most four rows: a stream of W.  k_warps warps of a CTA take kOut outputs together; their lanes share the k-elements, VE (16 bytes of
// a row that allows it) a lane and step, and add their sums up at the end, halving the set of sums a lane holds at each step of the
// exchange.  Sums of even and odd k-elements run side by side in packed multiply-adds.  k_warps is as large as fits two
// CTAs an SM; float32 takes four at least, where that leaves each its own batch of loads.  W from the HBM, us with 1 / 2 / 4 / 8 (the pick
// in brackets), bf16, one row: 4096 x 6144 [12.4] / 13.7 / 13.4 / 14.2, 4096 x 4096 10.7 / [8.4] / 9.6 / 10.5, 1024 x 1000 3.4 / 2.6 /
// 2.4 / [2.4], three rows of 8192 x 1024 26.1 / 14.6 / 8.8 / [6.3]; float32 4096 x 6144 20.5 / 20.6 / [19.5] / 19.2, 4096 x 12288 41.0 /
// 33.9 / [33.7] / 33.8.
constexpr int kOut = 4, kWarps = 8, kThreads = kWarps * 32;

// 16 bytes as pairs
template <typename T, int VE>
__device__ __forceinline__ void widen(const uint4& raw, float2 (&v)[VE / 2]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = make_float2(__uint_as_float(raw.x), __uint_as_float(raw.y));
    v[1] = make_float2(__uint_as_float(raw.z), __uint_as_float(raw.w));
  } else {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
    for (int i = 0; i < VE / 2; ++i) v[i] = __bfloat1622float2(h[i]);
  }
}
// Four elements of a row from k on as pairs; past K: zeros.  WIDE: bf16 whose rows and length allow 8-byte accesses.
template <bool WIDE, typename T>
__device__ __forceinline__ void load_pairs(const T* row, int k, int K, float2 (&v)[2]) {
  if constexpr (WIDE) {
    if (k + 4 <= K) {
      const uint2 raw = *reinterpret_cast<const uint2*>(row + k);
      v[0] = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.x));
      v[1] = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.y));
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[i].x = k + 2 * i < K ? (float)row[k + 2 * i] : 0.f;
    v[i].y = k + 2 * i + 1 < K ? (float)row[k + 2 * i + 1] : 0.f;
  }
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

template <typename T, int MT, int VE, bool WIDE>
__global__ void __launch_bounds__(kThreads, 2) linear_rows_kernel(const LinearParams p, const int k_warps) {
  __shared__ float parts[kWarps][kOut * MT];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = warp & (k_warps - 1), group = warp / k_warps;
  const long long n0 = ((long long)blockIdx.x * (kWarps / k_warps) + group) * kOut;       // (past the end: the last output, not written)
  const T* x[MT];
  const T* w[kOut];
#pragma unroll
  for (int i = 0; i < MT; ++i) x[i] = reinterpret_cast<const T*>(p.x) + (long long)min(i, p.rows - 1) * p.x_row;
#pragma unroll
  for (int j = 0; j < kOut; ++j) w[j] = reinterpret_cast<const T*>(p.w) + min(n0 + j, (long long)p.n - 1) * p.w_row;
  constexpr int N = kOut * MT, LEFT = N > 32 ? N / 32 : 1;
  // the output this thread finishes: group of outputs, value of it; its bias and residual come beside the sums
  const int out = (int)threadIdx.x / N, value = (int)threadIdx.x % N, m = value / kOut;
  const long long n = ((long long)blockIdx.x * (kWarps / k_warps) + out) * kOut + value % kOut;
  const bool mine = out < kWarps / k_warps && m < p.rows && n < p.n;
  const float bias = mine && p.bias ? p.bias[n] : 0.f;
  const float resid = mine && p.resid ? (float)reinterpret_cast<const T*>(p.resid)[(long long)m * p.resid_row + n] : 0.f;
  float2 sums[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sums[i] = make_float2(0.f, 0.f);
  auto multiply = [&](const float2 (&a)[VE / 2], const float2 (&b)[VE / 2], int at) {
#pragma unroll
    for (int e = 0; e < VE / 2; ++e) sums[at] = __ffma2_rn(a[e], b[e], sums[at]);
  };
  if constexpr (WIDE) {
    // U steps' rows of W are asked for before the first is used, and stay as they came until then
    constexpr int U = MT <= 2 ? 4 : 2;
    const int whole = p.k / VE, stride = k_warps * 32;
    for (int c = part * 32 + lane; c < whole; c += U * stride) {
      uint4 raw[U][kOut];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < kOut; ++j) {
          raw[u][j] = make_uint4(0u, 0u, 0u, 0u);
          if (c + u * stride < whole) raw[u][j] = reinterpret_cast<const uint4*>(w[j])[c + u * stride];
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = c + u * stride;
        if (at >= whole) break;
        uint4 own[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) own[i] = reinterpret_cast<const uint4*>(x[i])[at];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          float2 b[VE / 2];
          widen<T, VE>(own[i], b);
#pragma unroll
          for (int j = 0; j < kOut; ++j) {
            float2 a[VE / 2];
            widen<T, VE>(raw[u][j], a);
            multiply(a, b, i * kOut + j);
          }
        }
      }
    }
    const int k = whole * VE + lane;                               // the last few elements
    if (part == 0 && k < p.k) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < kOut; ++j) sums[i * kOut + j].x = fmaf((float)w[j][k], (float)x[i][k], sums[i * kOut + j].x);
    }
  } else {
    for (int k = (part * 32 + lane) * VE; k < p.k; k += k_warps * 32 * VE) {
      float2 a[kOut][VE / 2];
#pragma unroll
      for (int j = 0; j < kOut; ++j) load_pairs<false>(w[j], k, p.k, a[j]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        float2 b[VE / 2];
        load_pairs<false>(x[i], k, p.k, b);
#pragma unroll
        for (int j = 0; j < kOut; ++j) multiply(a[j], b, i * kOut + j);
      }
    }
  }
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = sums[i].x + sums[i].y;
  int first = 0;
  reduce_lanes<N, 16>(acc, &first);
  // (fewer values than lanes: the lanes with the same ones differ in the low bits, the first of them writes)
  if (N >= 32 || (lane & (32 / (N < 32 ? N : 32) - 1)) == 0) {
#pragma unroll
    for (int i = 0; i < LEFT; ++i) parts[warp][first + i] = acc[i];
  }
  __syncthreads();
  if (!mine) return;
  float v[1] = {0.f};
  for (int s = 0; s < k_warps; ++s) v[0] += parts[out * k_warps + s][value];
  v[0] += bias;
  activate<sizeof(T) == 2>(v, p.act);
  reinterpret_cast<T*>(p.y)[(long long)m * p.y_row + n] = (T)(v[0] + resid);
}

template <typename T, int MT, int VE, bool WIDE>
cudaError_t launch_rows_as(const LinearParams& p, cudaStream_t st) {
  int k_warps = 1;
  while (k_warps < kWarps && (long long)p.n * k_warps * 2 <= (long long)2 * kSms * kWarps * kOut && p.k >= 2 * k_warps * 32 * VE) k_warps *= 2;
  if (sizeof(T) == 4 && WIDE && k_warps < 4 && p.k >= 16 * 32 * VE) k_warps = 4;
  const int outputs = kWarps / k_warps * kOut;
  return launch_pdl(linear_rows_kernel<T, MT, VE, WIDE>, dim3((unsigned)((p.n + outputs - 1) / outputs)), dim3(kThreads), 0, st, 1, p, k_warps);
}
template <typename T, int VE, bool WIDE>
cudaError_t launch_rows_by(const LinearParams& p, cudaStream_t st) {
  if (p.rows == 1) return launch_rows_as<T, 1, VE, WIDE>(p, st);
  if (p.rows == 2) return launch_rows_as<T, 2, VE, WIDE>(p, st);
  return launch_rows_as<T, 4, VE, WIDE>(p, st);
}

// ------------------------------------------------------------------------------------------------ tiles
// More rows: tiles of 8 RM rows x 64 outputs.  Two groups of 128 threads take every second 16 of a step's 32 k-elements; a thread owns
// RM rows x 4 outputs and reads four k-elements of each at a time.  Operands lie in shared memory row by row, three steps deep.
// Few tiles: the k-elements are split over a cluster of up to eight CTAs (blockIdx.z); each leaves its sums in shared memory and
// finishes its part of the rows from everybody's, in the order of the k-elements.  Bound by the FMA pipe and the shared-memory reads
// that feed it (RM + 8 wavefronts to 16 RM multiply-adds of a warp).
constexpr int TN = 64, TK = 32, kPitch = TK + 4, kTileStages = 3, kGroup = 128, kTileThreads = 2 * kGroup;
template <int RM>
struct Tile {
  static constexpr int BM = 8 * RM, STAGE = (BM + TN) * kPitch;                 // floats
  static constexpr int SUMS = BM * (TN + 4);
  static constexpr int FLOATS = kTileStages * STAGE > 2 * SUMS ? kTileStages * STAGE : 2 * SUMS;
  static constexpr int BYTES = FLOATS * 4;
};

template <typename T, int RM, bool WIDE>
__global__ void __launch_bounds__(kTileThreads, 2) linear_tile_kernel(const LinearParams p, const int k_part) {
  using S = Tile<RM>;
  constexpr int BM = S::BM;
  extern __shared__ __align__(16) float sm[];
  const int tid = threadIdx.x, grp = tid / kGroup, lt = tid % kGroup, tx = lt & 15, ty = lt >> 4;       // rows ty + 8 i, outputs tx + 16 j
  const int n0 = (int)blockIdx.x * TN, m0 = (int)blockIdx.y * BM, splits = (int)gridDim.z, z = (int)blockIdx.z;
  const int k0 = z * k_part, k1 = min(p.k, k0 + k_part), steps = k1 > k0 ? (k1 - k0 + TK - 1) / TK : 0;
  pdl_wait();
  pdl_launch_dependents();
  // a step's operands: rows of x, then rows of W, four k-elements a thread and chunk
  auto fetch = [&](int step) {
    constexpr int ALL = (BM + TN) * (TK / 4), N = (ALL + kTileThreads - 1) / kTileThreads;
    float* dst = sm + (step % kTileStages) * S::STAGE;
    float4 v[sizeof(T) == 4 && WIDE ? 1 : N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = tid + i * kTileThreads, r = e / (TK / 4), kk = (e % (TK / 4)) * 4, k = k0 + step * TK + kk;
      if (ALL % kTileThreads != 0 && e >= ALL) break;
      const T* row = r < BM ? reinterpret_cast<const T*>(p.x) + (long long)min(m0 + r, p.rows - 1) * p.x_row
                            : reinterpret_cast<const T*>(p.w) + (long long)min(n0 + r - BM, p.n - 1) * p.w_row;
      if constexpr (sizeof(T) == 4 && WIDE) {
        cp_async_16(smem_u32(dst + r * kPitch + kk), k < k1 ? row + k : row, k < k1 ? 16u : 0u);      // (k, k1: multiples of 4)
      } else {
        float2 h[2];
        load_pairs<WIDE>(row, k, k1, h);
        v[i] = make_float4(h[0].x, h[0].y, h[1].x, h[1].y);
      }
    }
    if constexpr (!(sizeof(T) == 4 && WIDE)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = tid + i * kTileThreads, r = e / (TK / 4), kk = (e % (TK / 4)) * 4;
        if (ALL % kTileThreads != 0 && e >= ALL) break;
        *reinterpret_cast<float4*>(dst + r * kPitch + kk) = v[i];
      }
    }
  };
  float2 acc[RM][4];                             // sums of even and of odd k-elements
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = make_float2(0.f, 0.f);
#pragma unroll
  for (int s = 0; s < kTileStages - 1; ++s) {
    if (s < steps) fetch(s);
    cp_async_commit();
  }
  for (int s = 0; s < steps; ++s) {
    cp_async_wait<kTileStages - 2>();
    __syncthreads();
    if (s + kTileStages - 1 < steps) fetch(s + kTileStages - 1);
    cp_async_commit();
    const float* xs = sm + (s % kTileStages) * S::STAGE;
    const float* ws = xs + BM * kPitch;
#pragma unroll
    for (int kk = grp * 4; kk < TK; kk += 8) {
      float4 a[RM], b[4];
#pragma unroll
      for (int i = 0; i < RM; ++i) a[i] = *reinterpret_cast<const float4*>(xs + (ty + 8 * i) * kPitch + kk);
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(ws + (tx + 16 * j) * kPitch + kk);
#pragma unroll
      for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[i][j] = __ffma2_rn(make_float2(a[i].x, a[i].y), make_float2(b[j].x, b[j].y), acc[i][j]);
          acc[i][j] = __ffma2_rn(make_float2(a[i].z, a[i].w), make_float2(b[j].z, b[j].w), acc[i][j]);
        }
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  // ---- the groups' sums over the ring, then the cluster's
  float* mine = sm + grp * S::SUMS;
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) mine[(ty + 8 * i) * (TN + 4) + tx + 16 * j] = acc[i][j].x + acc[i][j].y;
  __syncthreads();
  if (splits > 1) {
    for (int e = tid; e < BM * (TN / 4); e += kTileThreads) {
      float* at = sm + (e / (TN / 4)) * (TN + 4) + (e % (TN / 4)) * 4;
      const float4 other = *reinterpret_cast<const float4*>(at + S::SUMS);
      float4 own = *reinterpret_cast<float4*>(at);
      own.x += other.x; own.y += other.y; own.z += other.z; own.w += other.w;
      *reinterpret_cast<float4*>(at) = own;
    }
    cluster_sync_all();
  }
  const int rows_own = (BM + splits - 1) / splits, r_end = min(BM, (z + 1) * rows_own);
  for (int r = z * rows_own + tid / (TN / 4); r < r_end; r += kTileThreads / (TN / 4)) {
    const int m = m0 + r, c = (tid % (TN / 4)) * 4;
    const uint32_t at = smem_u32(sm + r * (TN + 4) + c);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (splits > 1) {
      for (int s = 0; s < splits; ++s) {
        const uint32_t from = map_to_cta(at, (uint32_t)s);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(ld_cluster_u32(from + 4 * i));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = sm[r * (TN + 4) + c + i] + sm[S::SUMS + r * (TN + 4) + c + i];
    }
    if (m < p.rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p.bias && n0 + c + i < p.n) v[i] += p.bias[n0 + c + i];
      activate<sizeof(T) == 2>(v, p.act);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + c + i;
        if (n < p.n) {
          if (p.resid) v[i] += (float)reinterpret_cast<const T*>(p.resid)[(long long)m * p.resid_row + n];
          reinterpret_cast<T*>(p.y)[(long long)m * p.y_row + n] = (T)v[i];
        }
      }
    }
  }
  if (splits > 1) cluster_sync_all();            // nobody leaves while its sums are read
}

// Splits of the k-elements: CTAs for two an SM, each with at least 128 of them.
int pick_splits(long long tiles, int k) {
  int s = 1;
  while (s < 8 && tiles * s * 2 <= 3 * kSms && k >= s * 2 * 128) s *= 2;
  return s;
}
template <typename T, int RM, bool WIDE>
cudaError_t launch_tile_as(const LinearParams& p, cudaStream_t st) {
  static std::atomic<unsigned long long> attr{0};
  auto kern = linear_tile_kernel<T, RM, WIDE>;
  if (cudaError_t e = ensure_dyn_smem(kern, Tile<RM>::BYTES, attr); e != cudaSuccess) return e;
  const unsigned nt = (unsigned)((p.n + TN - 1) / TN), mt = (unsigned)((p.rows + Tile<RM>::BM - 1) / Tile<RM>::BM);
  const int splits = pick_splits((long long)nt * mt, p.k), part = ((p.k + splits - 1) / splits + TK - 1) / TK * TK;
  // (rows over y, which stops at 65535: more of them in several launches)
  for (unsigned m = 0; m < mt; m += 65535) {
    LinearParams q = p;
    const long long r0 = (long long)m * Tile<RM>::BM;
    q.x = reinterpret_cast<const T*>(p.x) + r0 * p.x_row;
    q.y = reinterpret_cast<T*>(p.y) + r0 * p.y_row;
    if (p.resid) q.resid = reinterpret_cast<const T*>(p.resid) + r0 * p.resid_row;
    q.rows = (int)(p.rows - r0);
    const unsigned ny = mt - m < 65535 ? mt - m : 65535;
    if (ny == 65535 && mt - m > 65535) q.rows = 65535 * Tile<RM>::BM;
    if (cudaError_t e = launch_pdl(kern, dim3(nt, ny, splits), dim3(kTileThreads), Tile<RM>::BYTES, st, splits, q, part); e != cudaSuccess)
      return e;
  }
  return cudaSuccess;
}
template <typename T, bool WIDE>
cudaError_t launch_tile_by(const LinearParams& p, cudaStream_t st) {
  if (p.rows <= 8) return launch_tile_as<T, 1, WIDE>(p, st);
  if (p.rows <= 16) return launch_tile_as<T, 2, WIDE>(p, st);
  if (p.rows <= 32 || (long long)((p.rows + 63) / 64) * ((p.n + TN - 1) / TN) < kSms) return launch_tile_as<T, 4, WIDE>(p, st);
  return launch_tile_as<T, 8, WIDE>(p, st);
}

template <typename T>
cudaError_t launch_simt(const LinearParams& p, cudaStream_t st) {
  // rows that 16-byte (rows kernel) or four-element accesses can follow
  auto wide = [&](int elements) {
    const uintptr_t mask = elements * sizeof(T) - 1;
    return (p.rows == 1 || p.x_row % elements == 0) && (p.n == 1 || p.w_row % elements == 0) && (reinterpret_cast<uintptr_t>(p.x) & mask) == 0 &&
           (reinterpret_cast<uintptr_t>(p.w) & mask) == 0;
  };
  constexpr int VE = 16 / sizeof(T);
  if (p.rows <= 4) return wide(VE) ? launch_rows_by<T, VE, true>(p, st) : launch_rows_by<T, 4, false>(p, st);
  return wide(4) && p.k % 4 == 0 ? launch_tile_by<T, true>(p, st) : launch_tile_by<T, false>(p, st);
}
}  // namespace

cudaError_t launch_linear_simt(const LinearParams& p, bool bf16, cudaStream_t st) {
  return bf16 ? launch_simt<__nv_bfloat16>(p, st) : launch_simt<float>(p, st);
}

}  // namespace dare

using namespace dare;

namespace {
// bf16, up to four rows, of a W that is not large: CUDA cores / tensor cores, W from the HBM, us: one row of 1024 x 1000 2.4 / 3.9, 8192 x 1024
// 5.3 / 7.6 (four 6.3 / 7.7), 4096 x 4096 8.4 / 9.5 (two 8.9 / 9.6), 4096 x 5000 11.4 / 10.4 (two 12.2 / 10.5), 4096 x 6144 12.4 / 11.9,
// 4096 x 12288 23.8 / 18.9; three of 4096 x 3000 10.3 / 8.6, four of 4096 x 2560 10.1 / 7.6.
bool rows_on_cuda_cores(const LinearParams& p) {
  const long long size = (long long)p.n * p.k;
  return (p.rows <= 2 && size <= 18 << 20) || (p.rows <= 4 && size <= 9 << 20);
}
}  // namespace

extern "C" dare_status_t dare_linear(const dare_linear_config_t* c, const void* x, const void* w, const float* bias, const void* resid,
                                     void* y, int32_t* status, void* cuda_stream) {
  if (!c || c->struct_size != sizeof(dare_linear_config_t)) return DARE_ERR_INVALID_ARG;
  if (c->dtype != DARE_F32 && c->dtype != DARE_BF16) return DARE_ERR_INVALID_ARG;
  if (c->activation < DARE_ACT_NONE || c->activation > DARE_ACT_GELU_TANH || c->reserved != 0) return DARE_ERR_INVALID_ARG;
  if (c->rows < 0 || c->rows > (int64_t)1 << 24 || c->in_features <= 0 || c->in_features > 1 << 20 || c->out_features <= 0 ||
      c->out_features > 1 << 24 || c->rows * c->out_features > (int64_t)1 << 38)
    return DARE_ERR_SHAPE;
  if (!stride_ok(c->x_row) || !stride_ok(c->w_row) || !stride_ok(c->resid_row) || !stride_ok(c->y_row)) return DARE_ERR_SHAPE;
  if (c->rows > 1 && c->y_row < c->out_features) return DARE_ERR_SHAPE;        // (rows of y in one place would be written twice)
  if (c->rows == 0) return DARE_OK;
  if (!x || !w || !y) return DARE_ERR_INVALID_ARG;
  if (resid == y && c->rows > 1 && c->resid_row != c->y_row) return DARE_ERR_INVALID_ARG;
  auto low = [](const void* p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; };
  const uintptr_t elem = c->dtype == DARE_BF16 ? 1u : 3u;
  if (low(x, elem) || low(w, elem) || low(resid, elem) || low(y, elem) || low(bias, 3u) || low(status, 3u)) return DARE_ERR_ALIGN;

  LinearParams p = {};
  p.x = x; p.w = w; p.bias = bias; p.resid = resid; p.y = y;
  p.x_row = c->x_row; p.w_row = c->w_row; p.resid_row = c->resid_row; p.y_row = c->y_row;
  p.rows = (int)c->rows; p.n = c->out_features; p.k = c->in_features; p.act = c->activation; p.status = status;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  // a stride that 16-byte accesses can follow (one row has none); rows that overlap stay off the tensor maps
  auto strides = [&](int64_t rows, int64_t row, int per16) { return rows == 1 || (row >= c->in_features && row % per16 == 0); };
  cudaError_t e;
  if (c->dtype == DARE_BF16) {
    const bool tc = !low(x, 15u) && !low(w, 15u) && strides(c->rows, c->x_row, 8) && strides(c->out_features, c->w_row, 8);
    e = tc && !rows_on_cuda_cores(p) ? launch_linear_tc(p, st) : launch_linear_simt(p, true, st);
  } else {
    const bool aligned = !low(x, 15u) && !low(w, 15u) && c->in_features % 4 == 0 && strides(c->rows, c->x_row, 4) &&
                         strides(c->out_features, c->w_row, 4);
    // What each takes, us.  Tensor cores: tiles of up to 128 rows x 64 outputs, one an SM at a time, a block of 64 k-elements 0.62 and
    // 0.0041 a row, shared by a cluster of up to eight (of which kClusters fit beside one another).  601 x 1024 x 1000, 128 rows a tile
    // 24.4, 80 rows 21.3, 64 34.4; 128 x 8192 x 1000: one CTA a tile 148, four 42, eight 48, four and 64 rows 34.5; 64 x 4096 x 4096 60.4,
    // two 34.7.  CUDA cores: an SM does about 50 multiply-adds a cycle and a launch takes 6 at least; few rows 1.5 times that: 8 x 2048
    // x 2048 9.7 (tensor cores 11.2), 16 x 4096 x 4096 30.6 (29.3), 64 77.
    constexpr int kClusters[4] = {kSms, 72, 32, 14};
    const int blocks = (c->in_features + 63) / 64, all_rows = (int)((c->rows + 15) / 16) * 16;
    float there = 1e30f;
    for (int rows = all_rows < 128 ? all_rows : 128; rows >= 16; rows -= 16) {
      const int64_t tiles = (c->rows + rows - 1) / rows * ((c->out_features + 63) / 64);
      for (int i = 0; i < 4 && 1 << i <= blocks; ++i) {
        const float block = fmaxf(0.72f, 0.62f + 0.0041f * (float)rows);
        const float us = 1.2f + (float)((tiles + kClusters[i] - 1) / kClusters[i]) *
                                    ((i ? 5.5f : 4.3f) + block * (float)((blocks + (1 << i) - 1) >> i));
        if (us < there) { there = us; p.splits = 1 << i; p.tile_rows = rows; }
      }
    }
    const int64_t simt_rows = c->rows <= 8 ? 12 : (c->rows <= 16 ? 24 : (c->rows + 31) / 32 * 32);
    const float here = 6.f + (float)simt_rows * (float)c->out_features * (float)c->in_features / (50.f * 1900.f * (float)kSms);
    e = aligned && p.rows > 4 && there < here ? launch_linear_f32(p, st) : launch_linear_simt(p, false, st);
  }
  if (e != cudaSuccess) { cudaGetLastError(); return DARE_ERR_CUDA; }
  return DARE_OK;
}
