// Rotary positions: the table of cosines and sines (scaled for long contexts), and its application to the heads of tokens
// (dare_ops.h).  Both are streams: a table is written once, heads are read once and written once.
#include <math.h>

#include "ops.h"
#include "tc_ptx.cuh"

namespace dare {

using namespace ptx;

namespace {

// ------------------------------------------------------------------------------------------------ table
constexpr int kMaxPairs = 128;
struct Frequencies {
  double f[kMaxPairs];       // angle a position of every pair
};
// A thread fills kRun consecutive positions of one pair.  cos and sin of p f come from one sincos in fp64 at the run's first position
// and a rotation by f for each next one, (c, s) <- (c cos f - s sin f, s cos f + c sin f): each multiplication adds at most
// 2^-52, so kRun of them stay 2^-24 of an fp32 rounding away from mattering, for an eighth of the sincos calls, which were
// all of the kernel's time.
constexpr int kRun = 16;
__global__ void __launch_bounds__(128) rope_freq_table_kernel(const Frequencies fr, float2* __restrict__ table, const long long positions,
                                                              const int pairs, const double magnitude) {
  pdl_wait();
  pdl_launch_dependents();
  const int per_cta = (int)blockDim.x / pairs;                    // runs side by side
  const int run = (int)threadIdx.x / pairs, j = (int)threadIdx.x - run * pairs;
  const long long p0 = ((long long)blockIdx.x * per_cta + run) * kRun;
  if (run >= per_cta || p0 >= positions) return;
  double c, s, cf, sf;
  sincos((double)p0 * fr.f[j], &s, &c);
  sincos(fr.f[j], &sf, &cf);
  c *= magnitude;
  s *= magnitude;
  float2* dst = table + (size_t)p0 * pairs + j;
  const int n = positions - p0 < kRun ? (int)(positions - p0) : kRun;
  for (int i = 0; i < n; ++i, dst += pairs) {
    *dst = make_float2((float)c, (float)s);
    const double cn = c * cf - s * sf;
    s = s * cf + c * sf;
    c = cn;
  }
}

// ------------------------------------------------------------------------------------------------ application
// A thread takes one unit of kHeads heads of a token (the table's entries are read once for them; their loads are in flight
// together).  Units of a head, VEC elements (16 bytes, or one pair where widths, strides or addresses do not allow that):
//   HALF         VEC elements of the first half of the rotated part and their partners in the second
//   INTERLEAVED  VEC elements = VEC / 2 pairs
// and behind them units of VEC elements that are copied (none in place).
constexpr int kHeads = 4, kThreads = 256;

// VEC elements, kept as they were read until they are used: a unit's heads are all on their way while the position and then the
// table's row are.
template <typename T, int VEC>
struct Chunk {
  static constexpr bool kWide = VEC * sizeof(T) == 16;
  union {
    uint4 vec;
    T el[VEC];
  };
  __device__ __forceinline__ Chunk() {}
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kWide) {
      vec = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) el[i] = p[i];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kWide) {
      *reinterpret_cast<uint4*>(p) = vec;
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) p[i] = el[i];
    }
  }
  __device__ __forceinline__ void get(float (&v)[VEC]) const {
    if constexpr (kWide && sizeof(T) == 2) {
      const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&vec);
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) {
        const float2 f = __bfloat1622float2(h[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = (float)el[i];
    }
  }
  __device__ __forceinline__ void put(const float (&v)[VEC]) {
    if constexpr (kWide && sizeof(T) == 2) {
      vec = pack8_bf16(v);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) el[i] = (T)v[i];
    }
  }
};

struct RopeParams {
  const void* x;
  void* y;
  const int* positions;
  const float2* table;
  int* status;
  long long tokens, table_positions, x_token, x_head, y_token, y_head;
  int heads, pairs, rotary, head_dim, pos_begin, transpose;
  int turn_units, units, chunks;       // of a head: units that turn, all units; chunks of kHeads heads
  int tokens_per_cta;
};

template <typename T, int VEC, bool HALF>
__global__ void __launch_bounds__(kThreads, 3) rope_kernel(const RopeParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int per_token = p.units * p.chunks;
  const long long t0 = (long long)blockIdx.x * p.tokens_per_cta;
  for (int w = (int)threadIdx.x; w < p.tokens_per_cta * per_token; w += kThreads) {
    const int tl = w / per_token, rest = w - tl * per_token, chunk = rest / p.units, u = rest - chunk * p.units;
    const long long t = t0 + tl;
    if (t >= p.tokens) return;
    const long long pos = p.positions ? (long long)p.positions[t] : p.pos_begin + t;
    const int h0 = chunk * kHeads, n = min(kHeads, p.heads - h0);
    const T* x = reinterpret_cast<const T*>(p.x) + t * p.x_token + h0 * p.x_head;
    T* y = reinterpret_cast<T*>(p.y) + t * p.y_token + h0 * p.y_head;
    const bool turns = u < p.turn_units;
    // a unit's elements: e .. and, of a half-split pair, its partners pairs further on
    const int e = turns ? u * VEC : p.rotary + (u - p.turn_units) * VEC;
    const bool whole = Chunk<T, VEC>::kWide || e + VEC <= p.head_dim;        // (a copied part may end in one element)
    Chunk<T, VEC> a[kHeads], b[HALF ? kHeads : 1];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (i < n) {
        if (whole) a[i].load(x + i * p.x_head + e);
        else a[i].el[0] = x[i * p.x_head + e];
        if (HALF && turns) b[HALF ? i : 0].load(x + i * p.x_head + p.pairs + e);
      }
    if (pos < 0 || pos >= p.table_positions) {
      flag_device_check(p.status);
      continue;
    }
    if (!turns) {
#pragma unroll
      for (int i = 0; i < kHeads; ++i)
        if (i < n) {
          if (whole) a[i].store(y + i * p.y_head + e);
          else y[i * p.y_head + e] = a[i].el[0];
        }
      continue;
    }
    constexpr int PAIRS = HALF ? VEC : VEC / 2;                              // pairs of a unit
    const float2* tab = p.table + pos * p.pairs + u * PAIRS;
    const float sign = p.transpose ? -1.f : 1.f;
    float2 cs[PAIRS];
#pragma unroll
    for (int k = 0; k < PAIRS; ++k) {
      cs[k] = tab[k];
      cs[k].y *= sign;
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (i < n) {
        float va[VEC];
        a[i].get(va);
        if constexpr (HALF) {
          float vb[VEC];
          b[i].get(vb);
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float s = va[k], r = vb[k];
            va[k] = s * cs[k].x - r * cs[k].y;
            vb[k] = r * cs[k].x + s * cs[k].y;
          }
          b[i].put(vb);
          b[i].store(y + i * p.y_head + p.pairs + e);
        } else {
#pragma unroll
          for (int k = 0; k < PAIRS; ++k) {
            const float s = va[2 * k], r = va[2 * k + 1];
            va[2 * k] = s * cs[k].x - r * cs[k].y;
            va[2 * k + 1] = r * cs[k].x + s * cs[k].y;
          }
        }
        a[i].put(va);
        a[i].store(y + i * p.y_head + e);
      }
  }
}

template <typename T, int VEC, bool HALF>
cudaError_t launch_rope_as(RopeParams p, cudaStream_t st) {
  p.turn_units = HALF ? p.pairs / VEC : p.rotary / VEC;
  const bool in_place = p.x == p.y;
  p.units = p.turn_units + (in_place ? 0 : (p.head_dim - p.rotary + VEC - 1) / VEC);
  p.chunks = (p.heads + kHeads - 1) / kHeads;
  const long long per_token = (long long)p.units * p.chunks;
  p.tokens_per_cta = per_token >= kThreads ? 1 : (int)(kThreads / per_token);
  const long long grid = (p.tokens + p.tokens_per_cta - 1) / p.tokens_per_cta;
  return launch_pdl(rope_kernel<T, VEC, HALF>, dim3((unsigned)grid), dim3(kThreads), 0, st, 1, p);
}

template <typename T>
cudaError_t launch_rope_type(const RopeParams& p, bool half, cudaStream_t st) {
  constexpr int V = 16 / sizeof(T);
  auto whole = [](long long v) { return v % V == 0; };
  const bool wide = whole(half ? p.pairs : p.rotary) && whole(p.head_dim - p.rotary) && whole(p.x_token) && whole(p.x_head) &&
                    whole(p.y_token) && whole(p.y_head) && (reinterpret_cast<uintptr_t>(p.x) & 15u) == 0 &&
                    (reinterpret_cast<uintptr_t>(p.y) & 15u) == 0;
  if (half) return wide ? launch_rope_as<T, V, true>(p, st) : launch_rope_as<T, 1, true>(p, st);
  return wide ? launch_rope_as<T, V, false>(p, st) : launch_rope_as<T, 2, false>(p, st);
}

}  // namespace

cudaError_t launch_rope_freq_table(const dare_rope_config_t& c, float* table, long long positions, cudaStream_t st) {
  const double kTwoPi = 6.283185307179586476925286766559;
  const int r = c.rotary_dim, pairs = r / 2;
  const double theta = c.scaling == DARE_ROPE_SCALE_BASE ? c.theta * pow(c.factor, (double)r / (double)(r - 2)) : c.theta;
  Frequencies fr;
  double first = 0., last = 0.;
  if (c.scaling == DARE_ROPE_SCALE_INDEX) {
    auto index_of = [&](double turns) { return (double)r * log((double)c.trained / (kTwoPi * turns)) / (2. * log(theta)); };
    first = fmax(floor(index_of(c.high)), 0.);
    last = fmin(ceil(index_of(c.low)), (double)(r - 1));
  }
  for (int j = 0; j < pairs; ++j) {
    double f = pow(theta, -2. * (double)j / (double)r), keep = 1.;
    if (c.scaling == DARE_ROPE_SCALE_LINEAR) keep = 0.;
    if (c.scaling == DARE_ROPE_SCALE_TURNS) keep = ((double)c.trained * f / kTwoPi - c.low) / (c.high - c.low);
    if (c.scaling == DARE_ROPE_SCALE_INDEX) keep = 1. - ((double)j - first) / fmax(last - first, 1e-3);
    keep = fmin(fmax(keep, 0.), 1.);
    fr.f[j] = keep >= 1. ? f : keep * f + (1. - keep) * f / c.factor;
  }
  const int per_cta = 128 / pairs;
  const long long runs = (positions + kRun - 1) / kRun;
  return launch_pdl(rope_freq_table_kernel, dim3((unsigned)((runs + per_cta - 1) / per_cta)), dim3(128), 0, st, 1, fr,
                    reinterpret_cast<float2*>(table), positions, pairs, c.magnitude);
}

cudaError_t launch_rope(const dare_rope_apply_t& c, const void* x, const int* positions, const float* table, void* y, int* status,
                        cudaStream_t st) {
  if (c.tokens == 0 || c.heads == 0) return cudaSuccess;
  RopeParams p = {};
  p.x = x; p.y = y; p.positions = positions; p.table = reinterpret_cast<const float2*>(table); p.status = status;
  p.tokens = c.tokens; p.table_positions = c.table_positions;
  p.x_token = c.x_token; p.x_head = c.x_head; p.y_token = c.y_token; p.y_head = c.y_head;
  p.heads = c.heads; p.pairs = c.rotary_dim / 2; p.rotary = c.rotary_dim; p.head_dim = c.head_dim;
  p.pos_begin = c.pos_begin; p.transpose = c.transpose;
  return c.dtype == DARE_BF16 ? launch_rope_type<__nv_bfloat16>(p, c.layout == DARE_ROPE_HALF, st)
                              : launch_rope_type<float>(p, c.layout == DARE_ROPE_HALF, st);
}

}  // namespace dare

using namespace dare;

extern "C" {

dare_status_t dare_rope_table(const dare_rope_config_t* c, float* table, int64_t positions, void* cuda_stream) {
  if (!c || c->struct_size != sizeof(dare_rope_config_t)) return DARE_ERR_INVALID_ARG;
  if (c->scaling < DARE_ROPE_SCALE_NONE || c->scaling > DARE_ROPE_SCALE_INDEX) return DARE_ERR_INVALID_ARG;
  if (!(c->theta > 0.) || !isfinite(c->theta) || !isfinite(c->magnitude)) return DARE_ERR_INVALID_ARG;
  if (c->scaling != DARE_ROPE_SCALE_NONE && (!(c->factor >= 1.) || !isfinite(c->factor))) return DARE_ERR_INVALID_ARG;
  if (c->rotary_dim <= 0 || c->rotary_dim % 2 != 0 || c->rotary_dim > 2 * kMaxPairs) return DARE_ERR_SHAPE;
  if (c->scaling == DARE_ROPE_SCALE_BASE && c->rotary_dim == 2) return DARE_ERR_SHAPE;
  if (c->scaling == DARE_ROPE_SCALE_TURNS || c->scaling == DARE_ROPE_SCALE_INDEX) {
    if (c->trained <= 0 || !(c->low > 0.) || !(c->high > c->low) || !isfinite(c->high)) return DARE_ERR_INVALID_ARG;
    if (c->scaling == DARE_ROPE_SCALE_INDEX && !(c->theta > 1.)) return DARE_ERR_INVALID_ARG;
  }
  if (positions < 0 || positions > (int64_t)1 << 24) return DARE_ERR_SHAPE;
  if (positions == 0) return DARE_OK;
  if (!table) return DARE_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(table) & 7u) != 0) return DARE_ERR_ALIGN;
  if (launch_rope_freq_table(*c, table, positions, (cudaStream_t)cuda_stream) != cudaSuccess) { cudaGetLastError(); return DARE_ERR_CUDA; }
  return DARE_OK;
}

dare_status_t dare_rope(const dare_rope_apply_t* c, const void* x, const int32_t* positions, const float* table, void* y,
                        int32_t* status, void* cuda_stream) {
  if (!c || c->struct_size != sizeof(dare_rope_apply_t)) return DARE_ERR_INVALID_ARG;
  if (c->dtype != DARE_F32 && c->dtype != DARE_BF16) return DARE_ERR_INVALID_ARG;
  if (c->layout != DARE_ROPE_HALF && c->layout != DARE_ROPE_INTERLEAVED) return DARE_ERR_INVALID_ARG;
  if (c->transpose != 0 && c->transpose != 1) return DARE_ERR_INVALID_ARG;
  if (c->tokens < 0 || c->tokens > (int64_t)1 << 30 || c->heads < 0 || c->heads > 65536 || c->head_dim <= 0 || c->head_dim > 65536)
    return DARE_ERR_SHAPE;
  if (c->rotary_dim <= 0 || c->rotary_dim % 2 != 0 || c->rotary_dim > 2 * kMaxPairs || c->rotary_dim > c->head_dim) return DARE_ERR_SHAPE;
  if (c->table_positions < 0) return DARE_ERR_SHAPE;
  if (c->tokens == 0 || c->heads == 0) return DARE_OK;
  if (!x || !y || !table) return DARE_ERR_INVALID_ARG;
  if (!stride_ok(c->x_token) || !stride_ok(c->x_head) || !stride_ok(c->y_token) || !stride_ok(c->y_head)) return DARE_ERR_SHAPE;
  if (!places_apart(c->tokens, c->y_token, c->heads, c->y_head, c->head_dim)) return DARE_ERR_SHAPE;
  if (x == y && ((c->tokens > 1 && c->x_token != c->y_token) || (c->heads > 1 && c->x_head != c->y_head))) return DARE_ERR_INVALID_ARG;
  const uintptr_t mask = c->dtype == DARE_BF16 ? 1u : 3u;
  if ((reinterpret_cast<uintptr_t>(x) & mask) || (reinterpret_cast<uintptr_t>(y) & mask) || (reinterpret_cast<uintptr_t>(table) & 7u) ||
      (reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(status) & 3u))
    return DARE_ERR_ALIGN;
  if (launch_rope(*c, x, positions, table, y, status, (cudaStream_t)cuda_stream) != cudaSuccess) { cudaGetLastError(); return DARE_ERR_CUDA; }
  return DARE_OK;
}

}  // extern "C"
