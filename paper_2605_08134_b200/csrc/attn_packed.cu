// Attention over packed sequences: the CUDA-core kernel (float32, head widths and alignments that the tensor-core kernel does not
// take) and the merge of the shares' partial results (attn_packed.h).
#include "attn_packed.h"
#include "tc_ptx.cuh"

namespace dare {

using namespace ptx;

namespace {

// ------------------------------------------------------------------------------------------------ CUDA cores
// A CTA walks the segments of its share with tiles of 32 rows (8 where the sequences have no more, as in decoding: a thread then has one
// row instead of four); two groups of 128 threads take every second block of BKV keys and
// are merged at the end of a segment.  A thread owns 4 (1) rows: scores of BKV / 16 keys each, then HD / 16 columns of the output each;
// the 16 lanes of a half-warp share their rows, so the softmax is shuffles and the weights pass through shared memory inside the
// half-warp.  Two CTAs an SM, so that one multiplies while the other is between two segments.  Everything in fp32.  Bound by the FMA pipe and the shared-memory reads that feed it (8 16-byte reads to 64 FMAs).
constexpr int KG = 2, GROUP = 128, kThreads = KG * GROUP;
template <int HD, int BQ>
struct Sm {
  static constexpr int BKV = HD == 256 ? 16 : (HD == 128 ? 32 : 64), JN = BKV / 16;
  static constexpr int KP = HD + 4, PP = BKV + 4;                         // pitches (floats)
  static constexpr int VW = HD >= 64 ? 4 : 2, NC = HD / (16 * VW);        // a lane's columns: NC vectors of VW
  static constexpr int BUF = BKV * KP + BKV * HD;
  static constexpr int Q_OFF = 0, P_OFF = BQ * KP, KV_OFF = P_OFF + KG * BQ * PP, FLOATS = KV_OFF + KG * BUF;
  static constexpr int BYTES = FLOATS * 4;
  static_assert(BYTES <= 112 * 1024 && BQ * HD + 2 * BQ <= BUF, "shared memory; a group's result over its buffer");
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

template <typename T, int HD, int BQ>
__global__ void __launch_bounds__(kThreads, 2) packed_simt_kernel(const PackedParams p, const bool wide) {
  using S = Sm<HD, BQ>;
  constexpr int RI = BQ / 8;                                                // rows of a thread
  constexpr int BKV = S::BKV, JN = S::JN, KP = S::KP, PP = S::PP, VW = S::VW, NC = S::NC;
  extern __shared__ __align__(16) float sm[];
  __shared__ Place pl_sh;
  __shared__ unsigned share_sh[2];
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
  Line<BQ, true> line(p);                        // (used by warp 0)
  if (tid < 32) {
    const unsigned total = line.total(), per = share_units(p, total), begin = blockIdx.x * per;
    if (tid == 0) {
      share_sh[0] = begin;
      share_sh[1] = min(begin + per, total);
    }
  }
  __syncthreads();
  const unsigned share_begin = share_sh[0], share_end = share_sh[1];
  for (unsigned u = share_begin; u < share_end;) {
    if (tid < 32) {
      Place pl;
      if (line.find(u, &pl) && tid == 0) pl_sh = pl;
    }
    __syncthreads();
    const Place pl = pl_sh;
    const int row0 = pl.tile * BQ, rows = min(BQ, pl.s.nq * p.group - row0);
    const TileRows tr = tile_rows(p, row0);
    const Part part = part_of(pl, u, share_begin, share_end, (int)blockIdx.x);
    if (part.k1 == 0) break;                     // (the share ends before the pair's keys begin)
    const int slot = part.slot;
    const int last_seen = keys_seen(p, pl.s, row_at(p, tr, 0, rows - 1).query);
    const int key0 = (int)(part.k0 << p.unit_shift), key1 = min(last_seen, (int)(part.k1 << p.unit_shift));
    for (int i = tid; i < BQ * (HD / 4); i += kThreads) {
      const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < rows) {
        const RowAt at = row_at(p, tr, pl.h, r);
        x = load4(q + (long long)(pl.s.q0 + at.query) * p.q_token + at.head * p.q_head + d, wide);
      }
      *reinterpret_cast<float4*>(qs + r * KP + d) = x;
    }
    int seen[RI];
#pragma unroll
    for (int i = 0; i < RI; ++i) seen[i] = keys_seen(p, pl.s, row_at(p, tr, 0, min(ty + 8 * i, rows - 1)).query);
    float m[RI], l[RI];
    float2 acc[RI][NC * VW / 2];
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int e = 0; e < NC * VW / 2; ++e) acc[i][e] = make_float2(0.f, 0.f);
    }
    __syncthreads();
    // A group's next keys come while it multiplies weights and values, its next values while it works out scores (float32: asynchronous
    // copies, two groups of them in flight).
    auto fetch = [&](float* dst, int pitch, const T* src, long long token, long long head, int kb) {
      constexpr int N = BKV * (HD / 4) / GROUP;
      const T* base = src + (long long)pl.s.k0 * token + pl.h * head;
      float4 x[sizeof(T) == 4 ? 1 : N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = lt + i * GROUP, r = e / (HD / 4), d = (e % (HD / 4)) * 4;
        const bool there = kb + r < key1;                 // (else zeros: what lies there may be anything)
        const T* at = base + (there ? (long long)(kb + r) * token + d : 0);
        if constexpr (sizeof(T) == 4) {
          if (wide) cp_async_16(smem_u32(dst + r * pitch + d), at, there ? 16u : 0u);
          else *reinterpret_cast<float4*>(dst + r * pitch + d) = there ? load4(at, false) : make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
          x[i] = there ? load4(at, wide) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      if constexpr (sizeof(T) != 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int e = lt + i * GROUP, r = e / (HD / 4), d = (e % (HD / 4)) * 4;
          *reinterpret_cast<float4*>(dst + r * pitch + d) = x[i];
        }
      }
      cp_async_commit();
    };
    auto fetch_k = [&](int kb) { if (kb < key1) fetch(ks, KP, kg, p.k_token, p.k_head, kb); else cp_async_commit(); };
    auto fetch_v = [&](int kb) { if (kb < key1) fetch(vs, HD, vg, p.v_token, p.v_head, kb); else cp_async_commit(); };
    auto group_sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + grp), "n"(GROUP) : "memory"); };
    fetch_k(key0 + grp * BKV);
    fetch_v(key0 + grp * BKV);
    for (int kb = key0 + grp * BKV; kb < key1; kb += KG * BKV) {
      cp_async_wait<1>();                                 // the keys are here
      group_sync();
      float2 s2[RI][JN];                                   // sums over even and over odd elements
#pragma unroll
      for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < JN; ++j) s2[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
      for (int d = 0; d < HD; d += 4) {
        float4 a[RI], b[JN];
#pragma unroll
        for (int i = 0; i < RI; ++i) a[i] = *reinterpret_cast<const float4*>(qs + (ty + 8 * i) * KP + d);
#pragma unroll
        for (int j = 0; j < JN; ++j) b[j] = *reinterpret_cast<const float4*>(ks + (tx + 16 * j) * KP + d);
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
          for (int j = 0; j < JN; ++j) {
            s2[i][j] = __ffma2_rn(make_float2(a[i].x, a[i].y), make_float2(b[j].x, b[j].y), s2[i][j]);
            s2[i][j] = __ffma2_rn(make_float2(a[i].z, a[i].w), make_float2(b[j].z, b[j].w), s2[i][j]);
          }
      }
      group_sync();                                       // everybody is through with the keys
      fetch_k(kb + KG * BKV);
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        float top = -INFINITY, s[JN];
#pragma unroll
        for (int j = 0; j < JN; ++j) {
          s[j] = kb + tx + 16 * j < min(seen[i], key1) ? (s2[i][j].x + s2[i][j].y) * p.scale_log2 : -INFINITY;
          top = fmaxf(top, s[j]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float m_new = fmaxf(m[i], top), base = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2f(m[i] - base);                          // (nothing yet: 2^-inf = 0)
        m[i] = m_new;
        l[i] *= alpha;
#pragma unroll
        for (int e = 0; e < NC * VW / 2; ++e) acc[i][e] = __fmul2_rn(acc[i][e], make_float2(alpha, alpha));
#pragma unroll
        for (int j = 0; j < JN; ++j) {
          const float w = exp2f(s[j] - base);
          l[i] += w;                                                     // (this lane's keys; the lanes are added up at the end)
          ps[(ty + 8 * i) * PP + tx + 16 * j] = w;
        }
      }
      cp_async_wait<1>();                                 // the values are here
      group_sync();
#pragma unroll 2
      for (int j = 0; j < BKV; j += 4) {
        float4 w[RI];
#pragma unroll
        for (int i = 0; i < RI; ++i) w[i] = *reinterpret_cast<const float4*>(ps + (ty + 8 * i) * PP + j);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float2 v[NC * VW / 2];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const float* src = vs + (j + jj) * HD + c * 16 * VW + tx * VW;
            if constexpr (VW == 4) *reinterpret_cast<float4*>(v + 2 * c) = *reinterpret_cast<const float4*>(src);
            else v[c] = *reinterpret_cast<const float2*>(src);
          }
#pragma unroll
          for (int i = 0; i < RI; ++i) {
            const float wj = jj == 0 ? w[i].x : (jj == 1 ? w[i].y : (jj == 2 ? w[i].z : w[i].w));
#pragma unroll
            for (int e = 0; e < NC * VW / 2; ++e) acc[i][e] = __ffma2_rn(make_float2(wj, wj), v[e], acc[i][e]);
          }
        }
      }
      group_sync();                                       // everybody is through with the values
      fetch_v(kb + KG * BKV);
    }
    cp_async_wait<0>();
    // ---- the groups' results over their buffers, merged by everybody
    float* res = ks;
#pragma unroll
    for (int i = 0; i < RI; ++i) {
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
        for (int e = 0; e < VW / 2; ++e)
          *reinterpret_cast<float2*>(res + r * HD + c * 16 * VW + tx * VW + 2 * e) = acc[i][c * (VW / 2) + e];
    }
    __syncthreads();
    // (a warp has 4 rows x 32 columns at a time: whole sectors of the slot, whose rows lie side by side, and of the output)
    for (int i = tid; i < (rows + 3) / 4 * HD; i += kThreads) {
      const int chunk = i >> 5, r = chunk / (HD / 32) * 4 + ((i >> 3) & 3), d = chunk % (HD / 32) * 32 + (i & 7) * 4;
      if (r >= rows) continue;
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
        reinterpret_cast<float4*>(p.part_o)[((size_t)slot * (HD / 4) + d / 4) * BQ + r] = o;
        if (d == 0) p.part_ml[(size_t)slot * BQ + r] = make_float2(top, sum);
      } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const RowAt at = row_at(p, tr, pl.h, r);
        T* dst = reinterpret_cast<T*>(p.o) + (long long)(pl.s.q0 + at.query) * p.o_token + at.head * p.o_head + d;
        dst[0] = (T)(o.x * inv); dst[1] = (T)(o.y * inv); dst[2] = (T)(o.z * inv); dst[3] = (T)(o.w * inv);
        if (p.lse && d == 0)
          p.lse[(long long)(pl.s.q0 + at.query) * p.n_heads + at.head] = sum == 0.f ? -INFINITY : top * 0.69314718055994531f + logf(sum);
      }
    }
    u = part.end;
    __syncthreads();
  }
}

template <typename T, int HD, int BQ>
cudaError_t launch_simt_as(const PackedParams& p, cudaStream_t st) {
  static std::atomic<unsigned long long> attr{0};
  auto kern = packed_simt_kernel<T, HD, BQ>;
  if (cudaError_t e = ensure_dyn_smem(kern, Sm<HD, BQ>::BYTES, attr); e != cudaSuccess) return e;
  auto whole = [](long long v) { return v % 4 == 0; };
  const uintptr_t mask = 4 * sizeof(T) - 1;
  auto at = [&](const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & mask) == 0; };
  const bool wide = whole(p.q_token) && whole(p.q_head) && whole(p.k_token) && whole(p.k_head) && whole(p.v_token) && whole(p.v_head) &&
                    at(p.q) && at(p.k) && at(p.v);
  return launch_pdl(kern, dim3((unsigned)p.n_ctas), dim3(kThreads), Sm<HD, BQ>::BYTES, st, 1, p, wide);
}

// ------------------------------------------------------------------------------------------------ merge
// o = sum_c 2^(m_c - m) o_c / sum_c 2^(m_c - m) l_c over the shares that hold keys of the row's pair, in the order of the keys (so the
// result does not depend on which CTA was first).  blockIdx.x is a cut between two shares; the CTAs of the first cut in a pair merge it,
// a warp kItems times 4 rows x 32 columns.  CTAs of two warps: the first 148 fit beside the CTAs of the kernel before, look their
// cut up there and only wait for its end (CTAs of 256 threads that did so afterwards, each with 8 rows of a pair, were 8 us behind it).
constexpr int kCombineThreads = 64, kItems = 2;
template <typename T, int HD, int ROWS>
__global__ void __launch_bounds__(kCombineThreads, 18) packed_combine_kernel(const PackedParams p) {
  __shared__ Place pl_sh;
  __shared__ unsigned per_sh;
  __shared__ int more_sh;
  // (the lengths are inputs: complete before the kernel in front let this one start)
  if (threadIdx.x < 32) {
    Line<ROWS, true, true> line(p);
    const unsigned total = line.total(), per = share_units(p, total), cut = (blockIdx.x + 1) * per;
    Place pl;
    const bool found = cut < total && line.find(cut, &pl) && pl.first < cut && pl.first >= cut - per;
    if (threadIdx.x == 0) { pl_sh = pl; per_sh = per; more_sh = found ? 1 : 0; }
  }
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  if (!more_sh) return;
  const Place pl = pl_sh;
  const unsigned per = per_sh;
  const int c0 = (int)blockIdx.x, c1 = (int)((pl.first + pl.units - 1) / per);
  const int row0 = pl.tile * ROWS, rows = min(ROWS, pl.s.nq * p.group - row0);
  const TileRows tr = tile_rows(p, row0);
  // the first share's part is the last of that CTA, the others' their first
  auto slot_of = [&](int c) { return c == c0 ? 2 * c + 1 : 2 * c; };
  // a warp takes 4 rows x 32 columns at a time: whole 32-byte sectors of the slots and of the output
  constexpr int COLS = HD / 32;
  const int chunks = (rows + 3) / 4 * COLS, lane = (int)threadIdx.x & 31;
  const int chunk0 = ((int)blockIdx.y * (kCombineThreads / 32) + ((int)threadIdx.x >> 5)) * kItems;
  if (chunk0 >= chunks) return;
  int r[kItems], d[kItems];                      // (past the end: the last row again, not written)
  float top[kItems], sum[kItems];
  float4 o[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int chunk = chunk0 + i;
    r[i] = min(chunk / COLS * 4 + (lane >> 3), rows - 1);
    d[i] = (chunk % COLS) * 32 + (lane & 7) * 4;
    top[i] = -INFINITY;
    sum[i] = 0.f;
    o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 2
  for (int c = c0; c <= c1; ++c)
#pragma unroll
    for (int i = 0; i < kItems; ++i) top[i] = fmaxf(top[i], __ldcg(p.part_ml + (size_t)slot_of(c) * ROWS + r[i]).x);
#pragma unroll 2
  for (int c = c0; c <= c1; ++c)
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const size_t at = (size_t)slot_of(c) * ROWS + r[i];
      const float2 ml = __ldcg(p.part_ml + at);
      const float4 a = __ldcg(reinterpret_cast<const float4*>(p.part_o) + ((size_t)slot_of(c) * (HD / 4) + d[i] / 4) * ROWS + r[i]);
      const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top[i]);
      o[i].x = fmaf(a.x, w, o[i].x); o[i].y = fmaf(a.y, w, o[i].y); o[i].z = fmaf(a.z, w, o[i].z); o[i].w = fmaf(a.w, w, o[i].w);
      sum[i] = fmaf(ml.y, w, sum[i]);
    }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    if ((chunk0 + i) / COLS * 4 + (lane >> 3) >= rows) break;
    const float inv = sum[i] == 0.f ? 0.f : 1.f / sum[i];
    const RowAt at = row_at(p, tr, pl.h, r[i]);
    T* dst = reinterpret_cast<T*>(p.o) + (long long)(pl.s.q0 + at.query) * p.o_token + at.head * p.o_head + d[i];
    dst[0] = (T)(o[i].x * inv); dst[1] = (T)(o[i].y * inv); dst[2] = (T)(o[i].z * inv); dst[3] = (T)(o[i].w * inv);
    if (p.lse && d[i] == 0)
      p.lse[(long long)(pl.s.q0 + at.query) * p.n_heads + at.head] = sum[i] == 0.f ? -INFINITY : top[i] * 0.69314718055994531f + logf(sum[i]);
  }
}
template <typename T, int HD, int ROWS>
cudaError_t launch_combine_as(const PackedParams& p, cudaStream_t st) {
  // (no tile has more rows than there are)
  constexpr int per_cta = kCombineThreads / 32 * kItems;
  const long long all = p.q_rows * p.group, chunks = ((all < ROWS ? all : ROWS) + 3) / 4 * (HD / 32);
  return launch_pdl(packed_combine_kernel<T, HD, ROWS>, dim3((unsigned)(p.n_ctas - 1), (unsigned)((chunks + per_cta - 1) / per_cta)),
                    dim3(kCombineThreads), 0, st, 1, p);
}

template <typename T, int BQ>
cudaError_t launch_simt_hd(const PackedParams& p, int head_dim, cudaStream_t st) {
  switch (head_dim) {
    case 32: return launch_simt_as<T, 32, BQ>(p, st);
    case 64: return launch_simt_as<T, 64, BQ>(p, st);
    case 128: return launch_simt_as<T, 128, BQ>(p, st);
    default: return launch_simt_as<T, 256, BQ>(p, st);
  }
}
template <typename T, int BQ>
cudaError_t launch_combine_hd(const PackedParams& p, int head_dim, cudaStream_t st) {
  switch (head_dim) {
    case 32: return launch_combine_as<T, 32, BQ>(p, st);
    case 64: return launch_combine_as<T, 64, BQ>(p, st);
    case 128: return launch_combine_as<T, 128, BQ>(p, st);
    default: return launch_combine_as<T, 256, BQ>(p, st);
  }
}
}  // namespace

cudaError_t launch_packed_simt(const PackedParams& p, int head_dim, int bq, bool bf16, cudaStream_t st) {
  if (bq == kSimtRows) return bf16 ? launch_simt_hd<__nv_bfloat16, kSimtRows>(p, head_dim, st) : launch_simt_hd<float, kSimtRows>(p, head_dim, st);
  return bf16 ? launch_simt_hd<__nv_bfloat16, kSimtFewRows>(p, head_dim, st) : launch_simt_hd<float, kSimtFewRows>(p, head_dim, st);
}

cudaError_t launch_packed_combine(const PackedParams& p, int head_dim, int bq, bool bf16, cudaStream_t st) {
  if (bq == kTcRows)
    return head_dim == 128 ? launch_combine_as<__nv_bfloat16, 128, kTcRows>(p, st) : launch_combine_as<__nv_bfloat16, 64, kTcRows>(p, st);
  if (bq == kSimtRows)
    return bf16 ? launch_combine_hd<__nv_bfloat16, kSimtRows>(p, head_dim, st) : launch_combine_hd<float, kSimtRows>(p, head_dim, st);
  return bf16 ? launch_combine_hd<__nv_bfloat16, kSimtFewRows>(p, head_dim, st) : launch_combine_hd<float, kSimtFewRows>(p, head_dim, st);
}

}  // namespace dare
