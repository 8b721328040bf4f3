// Attention over packed sequences: the CUDA-core kernel (float32, head widths and alignments that the tensor-core kernel does not
// take) and the merge of the shares' partial results (attn_packed.h).
#include "attn_packed.h"
#include "tc_ptx.cuh"

namespace dare {

using namespace ptx;

namespace {

// ------------------------------------------------------------------------------------------------ CUDA cores
// A CTA walks the segments of its share with tiles of 32 rows; four groups of 128 threads take every fourth block of BKV keys and
// are merged at the end of a segment.  A thread owns 4 rows: scores of BKV / 16 keys each, then HD / 16 columns of the output each;
// the 16 lanes of a half-warp share their rows, so the softmax is shuffles and the weights pass through shared memory inside the
// half-warp.  Everything in fp32.  Bound by the FMA pipe and the shared-memory reads that feed it (8 16-byte reads to 64 FMAs).
constexpr int BQ = kSimtRows, KG = 4, GROUP = 128, kThreads = KG * GROUP;
template <int HD>
struct Sm {
  static constexpr int BKV = HD == 256 ? 16 : (HD == 128 ? 32 : 64), JN = BKV / 16;
  static constexpr int KP = HD + 4, PP = BKV + 4;                         // pitches (floats)
  static constexpr int VW = HD >= 64 ? 4 : 2, NC = HD / (16 * VW);        // a lane's columns: NC vectors of VW
  static constexpr int BUF = BKV * KP + BKV * HD;
  static constexpr int Q_OFF = 0, P_OFF = BQ * KP, KV_OFF = P_OFF + KG * BQ * PP, FLOATS = KV_OFF + KG * BUF;
  static constexpr int BYTES = FLOATS * 4;
  static_assert(BYTES <= 226 * 1024 && BQ * HD + 2 * BQ <= BUF, "shared memory; a group's result over its buffer");
};

// four elements of a row as fp32
template <typename T>
__device__ __forceinline__ float4 load4(const T* src, bool wide) {
  if constexpr (sizeof(T) == 4) {
    if (wide) return __ldcg(reinterpret_cast<const float4*>(src));
    return make_float4(src[0], src[1], src[2], src[3]);
  } else {
    if (wide) {
      const uint2 raw = __ldcg(reinterpret_cast<const uint2*>(src));
      const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.x));
      const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.y));
      return make_float4(a.x, a.y, b.x, b.y);
    }
    return make_float4((float)src[0], (float)src[1], (float)src[2], (float)src[3]);
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads, 1) packed_simt_kernel(const PackedParams p, const bool wide) {
  using S = Sm<HD>;
  constexpr int BKV = S::BKV, JN = S::JN, KP = S::KP, PP = S::PP, VW = S::VW, NC = S::NC;
  extern __shared__ __align__(16) float sm[];
  __shared__ Place pl_sh;
  __shared__ long long share_sh[2];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x, grp = tid / GROUP, lt = tid % GROUP, tx = lt & 15, ty = lt >> 4;      // rows ty + 8 i
  float* qs = sm + S::Q_OFF;
  float* ps = sm + S::P_OFF + grp * BQ * PP;
  float* ks = sm + S::KV_OFF + grp * S::BUF;
  float* vs = ks + BKV * KP;
  const T* q = reinterpret_cast<const T*>(p.q);
  const T* kg = reinterpret_cast<const T*>(p.k);
  const T* vg = reinterpret_cast<const T*>(p.v);
  if (tid < 32) {
    long long total = 0;
    const long long per = share_units<BQ>(p, &total), begin = (long long)blockIdx.x * per;
    if (tid == 0) {
      share_sh[0] = begin;
      share_sh[1] = begin + per < total ? begin + per : total;
    }
  }
  __syncthreads();
  const long long share_begin = share_sh[0], share_end = share_sh[1];
  for (long long u = share_begin; u < share_end;) {
    if (tid < 32) {
      Place pl;
      if (find_place<BQ, true>(p, u, &pl, nullptr) && tid == 0) pl_sh = pl;
    }
    __syncthreads();
    const Place pl = pl_sh;
    const int row0 = pl.tile * BQ, rows = (int)min((long long)BQ, (long long)pl.s.nq * p.group - row0);
    const long long pair_end = pl.first + pl.units, end = pair_end < share_end ? pair_end : share_end;
    const bool whole = u == pl.first && end == pair_end;
    const int slot = whole ? -1 : 2 * (int)blockIdx.x + (pl.first <= share_begin ? 0 : 1);
    const int last_seen = keys_seen(p, pl.s, (row0 + rows - 1) / p.group);
    const int key0 = (int)(u - pl.first) * kUnitKeys, key1 = min(last_seen, (int)min((end - pl.first) * kUnitKeys, 0x7fffffffll));
    for (int i = tid; i < BQ * (HD / 4); i += kThreads) {
      const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < rows) {
        const RowAt at = row_at(p, pl, row0 + r);
        x = load4(q + (long long)(pl.s.q0 + at.query) * p.q_token + at.head * p.q_head + d, wide);
      }
      *reinterpret_cast<float4*>(qs + r * KP + d) = x;
    }
    int seen[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) seen[i] = keys_seen(p, pl.s, row_at(p, pl, row0 + min(ty + 8 * i, rows - 1)).query);
    float m[4], l[4], acc[4][NC * VW];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int e = 0; e < NC * VW; ++e) acc[i][e] = 0.f;
    }
    __syncthreads();
    for (int kb = key0 + grp * BKV; kb < key1; kb += KG * BKV) {
      const int keys = min(BKV, key1 - kb);
      for (int i = lt; i < BKV * (HD / 4); i += GROUP) {
        const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (r < keys) {
          const long long row = (long long)pl.s.k0 + kb + r;
          a = load4(kg + row * p.k_token + pl.h * p.k_head + d, wide);
          b = load4(vg + row * p.v_token + pl.h * p.v_head + d, wide);
        }
        *reinterpret_cast<float4*>(ks + r * KP + d) = a;
        *reinterpret_cast<float4*>(vs + r * HD + d) = b;
      }
      asm volatile("bar.sync %0, %1;" ::"r"(1 + grp), "n"(GROUP) : "memory");
      float s[4][JN];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < JN; ++j) s[i][j] = 0.f;
#pragma unroll 4
      for (int d = 0; d < HD; d += 4) {
        float4 a[4], b[JN];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(qs + (ty + 8 * i) * KP + d);
#pragma unroll
        for (int j = 0; j < JN; ++j) b[j] = *reinterpret_cast<const float4*>(ks + (tx + 16 * j) * KP + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < JN; ++j) {
            s[i][j] = fmaf(a[i].x, b[j].x, s[i][j]);
            s[i][j] = fmaf(a[i].y, b[j].y, s[i][j]);
            s[i][j] = fmaf(a[i].z, b[j].z, s[i][j]);
            s[i][j] = fmaf(a[i].w, b[j].w, s[i][j]);
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < JN; ++j) {
          s[i][j] = kb + tx + 16 * j < min(seen[i], key1) ? s[i][j] * p.scale_log2 : -INFINITY;
          top = fmaxf(top, s[i][j]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float m_new = fmaxf(m[i], top), base = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2f(m[i] - base);                          // (nothing yet: 2^-inf = 0)
        m[i] = m_new;
        l[i] *= alpha;
#pragma unroll
        for (int e = 0; e < NC * VW; ++e) acc[i][e] *= alpha;
#pragma unroll
        for (int j = 0; j < JN; ++j) {
          const float w = exp2f(s[i][j] - base);
          l[i] += w;                                                     // (this lane's keys; the lanes are added up at the end)
          ps[(ty + 8 * i) * PP + tx + 16 * j] = w;
        }
      }
      __syncwarp();
#pragma unroll 2
      for (int j = 0; j < BKV; j += 4) {
        float4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(ps + (ty + 8 * i) * PP + j);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float v[NC * VW];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const float* src = vs + (j + jj) * HD + c * 16 * VW + tx * VW;
#pragma unroll
            for (int e = 0; e < VW; e += 2) {
              const float2 t = *reinterpret_cast<const float2*>(src + e);
              v[c * VW + e] = t.x;
              v[c * VW + e + 1] = t.y;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float wj = jj == 0 ? w[i].x : (jj == 1 ? w[i].y : (jj == 2 ? w[i].z : w[i].w));
#pragma unroll
            for (int e = 0; e < NC * VW; ++e) acc[i][e] = fmaf(wj, v[e], acc[i][e]);
          }
        }
      }
      asm volatile("bar.sync %0, %1;" ::"r"(1 + grp), "n"(GROUP) : "memory");
    }
    // ---- the groups' results over their buffers, merged by everybody
    float* res = ks;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
      const int r = ty + 8 * i;
      if (tx == 0) {
        res[BQ * HD + r] = m[i];
        res[BQ * HD + BQ + r] = l[i];
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < VW; ++e) res[r * HD + c * 16 * VW + tx * VW + e] = acc[i][c * VW + e];
    }
    __syncthreads();
    for (int i = tid; i < rows * (HD / 4); i += kThreads) {
      const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int g = 0; g < KG; ++g) top = fmaxf(top, sm[S::KV_OFF + g * S::BUF + BQ * HD + r]);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll
      for (int g = 0; g < KG; ++g) {
        const float* src = sm + S::KV_OFF + g * S::BUF;
        const float mg = src[BQ * HD + r], w = mg == -INFINITY ? 0.f : exp2f(mg - top);
        const float4 a = *reinterpret_cast<const float4*>(src + r * HD + d);
        o.x = fmaf(a.x, w, o.x); o.y = fmaf(a.y, w, o.y); o.z = fmaf(a.z, w, o.z); o.w = fmaf(a.w, w, o.w);
        sum = fmaf(src[BQ * HD + BQ + r], w, sum);
      }
      if (slot >= 0) {
        *reinterpret_cast<float4*>(p.part_o + ((size_t)slot * BQ + r) * HD + d) = o;
        if (d == 0) p.part_ml[(size_t)slot * BQ + r] = make_float2(top, sum);
      } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const RowAt at = row_at(p, pl, row0 + r);
        T* dst = reinterpret_cast<T*>(p.o) + (long long)(pl.s.q0 + at.query) * p.o_token + at.head * p.o_head + d;
        dst[0] = (T)(o.x * inv); dst[1] = (T)(o.y * inv); dst[2] = (T)(o.z * inv); dst[3] = (T)(o.w * inv);
        if (p.lse && d == 0)
          p.lse[(long long)(pl.s.q0 + at.query) * p.n_heads + at.head] = sum == 0.f ? -INFINITY : top * 0.69314718055994531f + logf(sum);
      }
    }
    u = end;
    __syncthreads();
  }
}

template <typename T, int HD>
cudaError_t launch_simt_as(const PackedParams& p, cudaStream_t st) {
  static std::atomic<unsigned long long> attr{0};
  auto kern = packed_simt_kernel<T, HD>;
  if (cudaError_t e = ensure_dyn_smem(kern, Sm<HD>::BYTES, attr); e != cudaSuccess) return e;
  auto whole = [](long long v) { return v % 4 == 0; };
  const uintptr_t mask = 4 * sizeof(T) - 1;
  auto at = [&](const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & mask) == 0; };
  const bool wide = whole(p.q_token) && whole(p.q_head) && whole(p.k_token) && whole(p.k_head) && whole(p.v_token) && whole(p.v_head) &&
                    at(p.q) && at(p.k) && at(p.v);
  return launch_pdl(kern, dim3((unsigned)p.n_ctas), dim3(kThreads), Sm<HD>::BYTES, st, 1, p, wide);
}

// ------------------------------------------------------------------------------------------------ merge
// o = sum_c 2^(m_c - m) o_c / sum_c 2^(m_c - m) l_c over the shares that hold keys of the row's pair, in the order of the keys (so the
// result does not depend on which CTA was first).  One CTA a pair; a thread has four columns of a row.  A pair that lies in one
// share was written by it.
template <typename T, int HD, int ROWS>
__global__ void __launch_bounds__(256) packed_combine_kernel(const PackedParams p) {
  __shared__ Place pl_sh;
  __shared__ long long per_sh;
  __shared__ int more_sh;
  pdl_wait();
  pdl_launch_dependents();
  if (threadIdx.x < 32) {
    // (blockIdx.x counts pairs: looked up by pair, the unit it begins at by its place among the units)
    long long total = 0, base_units = 0, base_pairs = 0;
    const int lane = threadIdx.x;
    const long long per = share_units<ROWS>(p, &total), u = blockIdx.x;
    bool found = false;
    for (int b0 = 0; b0 < p.batch && !found; b0 += 32) {
      const int b = b0 + lane;
      SeqGeom s{0, 0, 0, 0};
      if (b < p.batch) s = seq_geom(p, b);
      const long long pairs = (((long long)s.nq * p.group + ROWS - 1) / ROWS) * p.kv_heads;
      const int units = max(1, (s.n + kUnitKeys - 1) / kUnitKeys);
      long long inc = pairs, inc_u = pairs * units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, inc, o), w = __shfl_up_sync(0xffffffffu, inc_u, o);
        if (lane >= o) { inc += v; inc_u += w; }
      }
      const unsigned hit = __ballot_sync(0xffffffffu, u < base_pairs + inc);
      if (hit != 0u) {
        const int src = __ffs((int)hit) - 1;
        const long long pair = u - (base_pairs + __shfl_sync(0xffffffffu, inc - pairs, src));
        const long long first = base_units + __shfl_sync(0xffffffffu, inc_u - pairs * units, src) +
                                pair * __shfl_sync(0xffffffffu, units, src);
        Place pl;
        find_place<ROWS, true>(p, first, &pl, nullptr);
        if (lane == 0) { pl_sh = pl; per_sh = per; }
        found = true;
      }
      base_pairs += __shfl_sync(0xffffffffu, inc, 31);
      base_units += __shfl_sync(0xffffffffu, inc_u, 31);
    }
    if (lane == 0) more_sh = found ? 1 : 0;
  }
  __syncthreads();
  if (!more_sh) return;
  const Place pl = pl_sh;
  const long long per = per_sh;
  const int c0 = (int)(pl.first / per), c1 = (int)((pl.first + pl.units - 1) / per);
  if (c0 == c1) return;
  const int row0 = pl.tile * ROWS, rows = (int)min((long long)ROWS, (long long)pl.s.nq * p.group - row0);
  // the first share's part is the last of that CTA (unless the share begins with this pair), the others' their first
  auto slot_of = [&](int c) { return 2 * c + (c == c0 && pl.first > c0 * per ? 1 : 0); };
  for (int i = threadIdx.x; i < rows * (HD / 4); i += 256) {
    const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
    float top = -INFINITY;
#pragma unroll 8
    for (int c = c0; c <= c1; ++c) top = fmaxf(top, __ldcg(p.part_ml + (size_t)slot_of(c) * ROWS + r).x);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int c = c0; c <= c1; ++c) {
      const size_t at = (size_t)slot_of(c) * ROWS + r;
      const float2 ml = __ldcg(p.part_ml + at);
      const float4 a = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * HD + d));
      const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top);
      o.x = fmaf(a.x, w, o.x); o.y = fmaf(a.y, w, o.y); o.z = fmaf(a.z, w, o.z); o.w = fmaf(a.w, w, o.w);
      sum = fmaf(ml.y, w, sum);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const RowAt at = row_at(p, pl, row0 + r);
    T* dst = reinterpret_cast<T*>(p.o) + (long long)(pl.s.q0 + at.query) * p.o_token + at.head * p.o_head + d;
    dst[0] = (T)(o.x * inv); dst[1] = (T)(o.y * inv); dst[2] = (T)(o.z * inv); dst[3] = (T)(o.w * inv);
    if (p.lse && d == 0)
      p.lse[(long long)(pl.s.q0 + at.query) * p.n_heads + at.head] = sum == 0.f ? -INFINITY : top * 0.69314718055994531f + logf(sum);
  }
}
template <typename T, int HD, int ROWS>
cudaError_t launch_combine_as(const PackedParams& p, cudaStream_t st) {
  const long long pairs = ((p.q_rows * p.group) / ROWS + p.batch) * p.kv_heads;
  return launch_pdl(packed_combine_kernel<T, HD, ROWS>, dim3((unsigned)pairs), dim3(256), 0, st, 1, p);
}
}  // namespace

cudaError_t launch_packed_simt(const PackedParams& p, int head_dim, bool bf16, cudaStream_t st) {
  switch (head_dim) {
    case 32: return bf16 ? launch_simt_as<__nv_bfloat16, 32>(p, st) : launch_simt_as<float, 32>(p, st);
    case 64: return bf16 ? launch_simt_as<__nv_bfloat16, 64>(p, st) : launch_simt_as<float, 64>(p, st);
    case 128: return bf16 ? launch_simt_as<__nv_bfloat16, 128>(p, st) : launch_simt_as<float, 128>(p, st);
    default: return bf16 ? launch_simt_as<__nv_bfloat16, 256>(p, st) : launch_simt_as<float, 256>(p, st);
  }
}

cudaError_t launch_packed_combine(const PackedParams& p, int head_dim, int bq, bool bf16, cudaStream_t st) {
  if (bq == kTcRows)
    return head_dim == 128 ? launch_combine_as<__nv_bfloat16, 128, kTcRows>(p, st) : launch_combine_as<__nv_bfloat16, 64, kTcRows>(p, st);
  switch (head_dim) {
    case 32: return bf16 ? launch_combine_as<__nv_bfloat16, 32, kSimtRows>(p, st) : launch_combine_as<float, 32, kSimtRows>(p, st);
    case 64: return bf16 ? launch_combine_as<__nv_bfloat16, 64, kSimtRows>(p, st) : launch_combine_as<float, 64, kSimtRows>(p, st);
    case 128: return bf16 ? launch_combine_as<__nv_bfloat16, 128, kSimtRows>(p, st) : launch_combine_as<float, 128, kSimtRows>(p, st);
    default: return bf16 ? launch_combine_as<__nv_bfloat16, 256, kSimtRows>(p, st) : launch_combine_as<float, 256, kSimtRows>(p, st);
  }
}

}  // namespace dare
