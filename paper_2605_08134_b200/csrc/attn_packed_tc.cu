// Attention over packed sequences on tcgen05 tensor cores: bf16, head_dim 128 or 64, fp32 softmax (attn_packed.h: rows, pairs, tiles and
// shares).  Both forms have the same parts; this file has the one for few rows (shares), attn_packed_tiles.cu the one for many.
//   TMA       K and V blocks (64-column boxes, 128-byte swizzle) into rings
//   issuers   one lane of a warp for each of two streams: S = Q K^T into a score buffer of tensor memory, O += P V with P read from
//             tensor memory
//   softmax   four warps a stream, thread <-> row: scores from tensor memory, maximum, 2^x, P as bf16 back over the scores; O is rescaled
//             in place only when a row's maximum grew by more than 2^8
// P is one bf16 part with heads of 128: its rounding (2^-8 of a weight at most) leaves the output 1.3 to 1.4 times as far from exact as
// storing it as bf16 does; a second part would be half as much tensor work again.  With heads of 64 it is two parts, 16 bits, as in the
// layer's own attention: the output is as near to exact as its storage is (1.66e-3 relative; one part: 2.3e-3).  The second part
// takes 10 % (a block of 160 over 2500 keys) to 30 % (prompts) of a call's time.
// Shares: a CTA has 128 rows and its streams take its blocks of 64 keys in turn, so that few rows (a decoding step has n_heads /
// n_kv_heads of them) still keep 192 KB of keys and values on their way; the streams' results are merged as two parts of a key
// split.  Two score buffers a stream: the next block's scores are there when the softmax is through with one.  The producers know a
// share's segments themselves and run ahead into the next one while the rest of the CTA finishes.
//   warps 0, 1 TMA; 2, 3 issuers; 4-11 softmax
// Bound by the HBM with many keys (16 tokens over up to 16k keys each: 650 MB in 111 us, 0.89 of the copy peak); with few by the way of a
// segment: look-up 1.7 us, rows 0.8, first scores 0.6, a unit of 128 keys 0.7, rows out 0.8 to 1.5, merge 2.5.
#include "attn_packed_tc.cuh"
#include "tc.h"

namespace dare {

using namespace ptx;

namespace {

using namespace packed_tc;

constexpr int BK = 64, kWorkers = 320;                   // keys a block; workers: all threads but the producers

template <int HD>
struct Smem {
  static constexpr int Q_BYTES = BQ * HD * 2, KV_BYTES = BK * HD * 2;
  static constexpr int RING = 6;                         // blocks of K and of V: half of them a stream
  static constexpr int Q_OFF = 0;
  static constexpr int K_OFF = Q_OFF + Q_BYTES;
  static constexpr int V_OFF = K_OFF + RING * KV_BYTES;
  static constexpr int BAR_OFF = V_OFF + RING * KV_BYTES;
  static constexpr int TOTAL = one_cta_per_sm(BAR_OFF + 512 + 1024);
  static_assert(TOTAL <= 232448, "shared memory of one CTA");
};

// The segment of a share that begins at unit u; *end: unit behind it.  By a warp.
typedef Line<BQ, true> WorkLine;
__device__ __forceinline__ bool segment_at(WorkLine& line, unsigned u, unsigned share_begin, unsigned share_end, Segment* g, unsigned* end) {
  const PackedParams& p = line.p;
  if (!line.find(u, &g->pl)) return false;
  const int row0 = g->pl.tile * BQ;
  g->at = tile_rows(p, row0);
  g->rows = min(BQ, g->pl.s.nq * p.group - row0);
  const Part part = part_of(g->pl, u, share_begin, share_end, (int)blockIdx.x);
  const int shift = p.unit_shift - 6;                                        // (blocks of 64 keys)
  *end = part.end;
  g->blk0 = (int)(part.k0 << shift);
  g->seen = row_sees(p, *g, g->rows - 1);
  g->n_blk = max(0, min((g->seen + BK - 1) / BK, (int)(part.k1 << shift)) - g->blk0);
  g->slot = part.slot;
  g->none = part.k1 == 0;
  return true;
}

}  // namespace

template <int HD>
__global__ void __launch_bounds__(kThreads, 1)
packed_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PackedParams p) {
  using S = Smem<HD>;
  constexpr int RING = S::RING / 2;                            // blocks of a stream's ring
  constexpr int UPR = HD / 8;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);    // [S::RING]
  uint64_t* k_empty = k_full + S::RING;
  uint64_t* v_full = k_empty + S::RING;
  uint64_t* v_empty = v_full + S::RING;
  uint64_t* s_full = v_empty + S::RING;                        // [2 streams][2 score buffers]
  uint64_t* p_full = s_full + 4;
  uint64_t* o_full = p_full + 4;                               // [2 streams][2]: product j signals o_full[stream][j & 1]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_full + 4);
  __shared__ Segment seg_sh;
  __shared__ int seg_more;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::RING; ++i) {
      mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s_full[i], 1); mbar_init(&o_full[i], 1); mbar_init(&p_full[i], kSoftmaxThreads / 64);
    }
    fence_mbar_init();
    prefetch_tmap(&tm_k);
    prefetch_tmap(&tm_v);
  }
  if (warp == 2) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_launch_dependents();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  // this CTA's part of the launch's line of units
  unsigned share_begin = 0, share_end = 0;
  auto find_share = [&](WorkLine& line) {
    const unsigned total = line.total(), per = share_units(p, total);
    share_begin = blockIdx.x * per;
    share_end = min(share_begin + per, total);
  };

  const int st = warp < 4 ? (warp & 1) : ((warp - 4) >> 2);                  // stream
  if (warp < 2) {
    // ---- producers
    WorkLine line(p);
    find_share(line);
    Segment g;
    unsigned u = share_begin, next;
    uint32_t cnt = 0;
    for (; u < share_end && segment_at(line, u, share_begin, share_end, &g, &next); u = next) {
      const int n = (g.n_blk - st + 1) / 2;
      for (int j = 0; j < n; ++j, ++cnt) {
        const int slot = st * RING + (int)(cnt % RING);
        const uint32_t freed = ((cnt / RING) & 1) ^ 1;
        const int row = g.pl.s.k0 + (g.blk0 + 2 * j + st) * BK;
        mbar_wait(&k_empty[slot], freed, p.status);
        if (elect_one()) load_block<HD, BK>(smem + S::K_OFF + slot * S::KV_BYTES, &tm_k, p.k_head_inner, g.pl.h, row, &k_full[slot]);
        __syncwarp();
        mbar_wait(&v_empty[slot], freed, p.status);
        if (elect_one()) load_block<HD, BK>(smem + S::V_OFF + slot * S::KV_BYTES, &tm_v, p.v_head_inner, g.pl.h, row, &v_full[slot]);
        __syncwarp();
      }
    }
  } else {
    const uint32_t tmem_s = tmem_base + st * 2 * BK, tmem_o = tmem_base + 4 * BK + st * HD;
    // (warp 2 looks the segments up; the others get them through shared memory)
    WorkLine line(p);
    if (warp == 2) find_share(line);
    unsigned u = share_begin, next = 0;
    uint32_t cnt = 0;                        // blocks of this stream so far: score buffer cnt & 1
    for (;;) {
      // everybody is through with the segment before: its Q tile, its accumulators
      asm volatile("bar.sync 2, %0;" ::"n"(kWorkers) : "memory");
      if (warp == 2) {
        Segment g;
        bool more = u < share_end && segment_at(line, u, share_begin, share_end, &g, &next);
        more = more && !g.none;                                      // (nothing follows then)
        u = next;
        if (lane == 0) {
          seg_more = more ? 1 : 0;
          if (more) seg_sh = g;
        }
      }
      asm volatile("bar.sync 2, %0;" ::"n"(kWorkers) : "memory");
      if (!seg_more) break;
      const Segment g = seg_sh;
      // ---- Q rows -> shared memory, K-major, 128-byte swizzle
      {
        constexpr int UNITS = BQ * UPR, QU = (UNITS + kWorkers - 1) / kWorkers;
        const int u0 = (int)threadIdx.x - 64;
        const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q);
        uint4 qv[QU];
#pragma unroll
        for (int i = 0; i < QU; ++i) {
          const int w = u0 + i * kWorkers, r = w / UPR, unit = w % UPR;
          qv[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < g.rows) {
            const RowAt at = row_at(p, g.at, g.pl.h, r);
            qv[i] = __ldcg(reinterpret_cast<const uint4*>(q + (long long)(g.pl.s.q0 + at.query) * p.q_token + at.head * p.q_head + unit * 8));
          }
        }
#pragma unroll
        for (int i = 0; i < QU; ++i) {
          const int w = u0 + i * kWorkers, r = w / UPR, unit = w % UPR;
          if (w < UNITS)
            *reinterpret_cast<uint4*>(smem + S::Q_OFF + (unit >> 3) * (BQ * 128) + r * 128 + (((unit & 7) ^ (r & 7)) << 4)) = qv[i];
        }
        fence_proxy_async_smem();
      }
      asm volatile("bar.sync 2, %0;" ::"n"(kWorkers) : "memory");

      const int rows = g.rows;
      const int n_st = (g.n_blk - st + 1) / 2;          // blocks of this stream
      if (warp < 4) {
        // ---- issuer of this stream's products
        constexpr uint32_t idesc_qk = idesc_bf16(BQ, BK, false), idesc_pv = idesc_bf16(BQ, HD, true);
        const uint64_t q_desc = smem_desc_k_sw128(smem_u32(smem + S::Q_OFF));
        const uint64_t k_desc0 = smem_desc_k_sw128(smem_u32(smem + S::K_OFF));
        const uint64_t v_desc0 = smem_desc_mn_sw128(smem_u32(smem + S::V_OFF), BK * 128);
        const int ring0 = st * RING;
        auto issue_qk = [&](int j) {
          const uint32_t sc = cnt + j, sb = sc & 1;
          const int slot = ring0 + (int)(sc % RING);
          mbar_wait(&k_full[slot], (sc / RING) & 1, p.status);
          tc_fence_after();
          if (elect_one()) {
            const uint64_t k_desc = k_desc0 + (uint64_t)(slot * (S::KV_BYTES >> 4));
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk)
              umma_ss(tmem_s + sb * BK, q_desc + (((kk >> 2) * (BQ * 128) + (kk & 3) * 32) >> 4),
                      k_desc + (((kk >> 2) * (BK * 128) + (kk & 3) * 32) >> 4), idesc_qk, kk != 0 ? 1u : 0u);
            umma_commit(&s_full[2 * st + sb]);
            umma_commit(&k_empty[slot]);
          }
          __syncwarp();
        };
        if (n_st > 0) issue_qk(0);
        if (n_st > 1) issue_qk(1);
        for (int j = 0; j < n_st; ++j) {
          const uint32_t sc = cnt + j, sb = sc & 1;
          const int slot = ring0 + (int)(sc % RING);
          mbar_poll(&p_full[2 * st + sb], (sc >> 1) & 1, p.status);          // P(j) has replaced S(j)
          mbar_wait(&v_full[slot], (sc / RING) & 1, p.status);
          const int keys = g.seen - (g.blk0 + 2 * j + st) * BK;              // (at least one: the block is one that is seen)
          if (keys < BK) zero_values<HD, BK>(smem + S::V_OFF + slot * S::KV_BYTES, keys, lane);
          tc_fence_after();
          if (elect_one()) {
            const uint64_t v_desc = v_desc0 + (uint64_t)(slot * (S::KV_BYTES >> 4));
#pragma unroll
            for (int ks = 0; ks < BK / 16; ++ks) {
              umma_ts(tmem_o, tmem_s + sb * BK + ks * 8, v_desc + ((ks * (16 * 128)) >> 4), idesc_pv, (j | ks) != 0 ? 1u : 0u);
              if (kSplitP<HD>) umma_ts(tmem_o, tmem_s + sb * BK + 32 + ks * 8, v_desc + ((ks * (16 * 128)) >> 4), idesc_pv, 1u);
            }
            umma_commit(&o_full[2 * st + sb]);
            umma_commit(&v_empty[slot]);
          }
          __syncwarp();
          if (j + 2 < n_st) issue_qk(j + 2);          // (in issue order behind the product that reads P(j))
        }
      } else {
        // ---- softmax of this stream's rows
        const int quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
        const float c = p.scale_log2;
        const bool warp_has_rows = quarter * 32 < rows;
        const RowAt at = row_at(p, g.at, g.pl.h, min(r, rows - 1));
        const int seen = keys_seen(p, g.pl.s, at.query);
        float m = -INFINITY, l = 0.f;               // maximum the exponentials are taken against; sum against it
        for (int j = 0; j < n_st; ++j) {
          const uint32_t sc = cnt + j, sb = sc & 1, sbuf = tmem_s + sb * BK + lane_addr;
          mbar_poll(&s_full[2 * st + sb], (sc >> 1) & 1, p.status);
          tc_fence_after();
          if (!warp_has_rows) {                     // rows of no query: only hand the block on
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[2 * st + sb]);
            continue;
          }
          const int keys = seen - (g.blk0 + 2 * j + st) * BK;     // of the block that this row sees
          float v[BK];
          tmem_ld_32x32_nowait(sbuf, v);
          tmem_ld_32x32_nowait(sbuf + 32, v + 32);
          tmem_ld_wait();
          if (__any_sync(0xffffffffu, keys < BK)) {
#pragma unroll
            for (int i = 0; i < BK; ++i)
              if (i >= keys) v[i] = -INFINITY;
          }
          float mx4[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) mx4[k] = fmaxf(v[k], v[4 + k]);
#pragma unroll
          for (int i = 8; i < BK; i += 8) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mx4[k] = fmax3(mx4[k], v[i + k], v[i + 4 + k]);
          }
          const float m_new = fmax3(m, fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
          if (j == 0) {
            m = m_new;
          } else {
            const bool grow = (m_new - m) * c > kRescaleStep;        // (-inf to -inf: NaN, no)
            if (__any_sync(0xffffffffu, grow)) {
              const float alpha = grow ? fast_exp2((m - m_new) * c) : 1.f;
              if (grow) { m = m_new; l *= alpha; }
              mbar_wait(&o_full[2 * st + (sb ^ 1)], ((sc - 1) >> 1) & 1, p.status);     // product j - 1 has been added
              tc_fence_after();
#pragma unroll 1
              for (int ch = 0; ch < HD / 32; ++ch) {
                float o[32];
                tmem_ld_32x32(tmem_o + lane_addr + ch * 32, o);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= alpha;
                tmem_st_32x32(tmem_o + lane_addr + ch * 32, o);
              }
            }
          }
          const float mc = m == -INFINITY ? 0.f : m * c;             // (nothing seen yet: 2^-inf = 0, not 2^NaN)
          const float2 c2 = make_float2(c, c), nmc2 = make_float2(-mc, -mc);
          float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          float pk[BK / 2], pl[kSplitP<HD> ? BK / 2 : 1];
#pragma unroll
          for (int i = 0; i < BK; i += 2) {
            float2 e = __ffma2_rn(make_float2(v[i], v[i + 1]), c2, nmc2);
            e.x = fast_exp2(e.x);
            e.y = fast_exp2(e.y);
            sum2[(i >> 1) & 1] = __fadd2_rn(sum2[(i >> 1) & 1], e);
            pack_weights<kSplitP<HD>>(e, pk[i >> 1], pl[kSplitP<HD> ? i >> 1 : 0]);
          }
          tmem_st_32x32_nowait(sbuf, pk);
          if constexpr (kSplitP<HD>) tmem_st_32x32_nowait(sbuf + 32, pl);
          tmem_st_wait();
          l += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_full[2 * st + sb]);
        }
        for (int j = max(0, n_st - 2); j < n_st; ++j)                // the last two products
          mbar_wait(&o_full[2 * st + ((cnt + j) & 1)], ((cnt + j) >> 1) & 1, p.status);
        tc_fence_after();

        auto out_row = [&](int row) {
          const RowAt w = row_at(p, g.at, g.pl.h, row);
          return reinterpret_cast<__nv_bfloat16*>(p.o) + (long long)(g.pl.s.q0 + w.query) * p.o_token + w.head * p.o_head;
        };
        float* lse = p.lse ? p.lse + (long long)(g.pl.s.q0 + at.query) * p.n_heads + at.head : nullptr;
        {
          // ---- merge the two streams: thread (stream, row) finishes its half of the row's columns.  The statistics and the finished
          // rows go where the Q tile was: both streams' last products are complete behind the first barrier.
          constexpr int HC = HD / 2;
          float2* stat = reinterpret_cast<float2*>(smem + S::Q_OFF + 8 * 32 * HC * 2 - 2 * BQ * sizeof(float2));
          asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory");
          stat[st * BQ + r] = make_float2(m, l);
          tc_fence_before();
          asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory");
          tc_fence_after();
          const float2 other = stat[(st ^ 1) * BQ + r];
          asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory");          // (the staging may lie over the statistics)
          if (warp_has_rows) {
            const int n_other = g.n_blk - n_st;
            const float m_all = fmaxf(m, other.x);
            const float w_mine = m == -INFINITY ? 0.f : fast_exp2((m - m_all) * c);
            const float w_other = other.x == -INFINITY ? 0.f : fast_exp2((other.x - m_all) * c);
            const float l_row = w_mine * l + w_other * other.y;
            const float inv = g.slot >= 0 ? 1.f : (l_row == 0.f ? 0.f : 1.f / l_row);
            const uint32_t t_mine = tmem_o + lane_addr + st * HC;
            const uint32_t t_other = tmem_base + 4 * BK + (st ^ 1) * HD + lane_addr + st * HC;
            uint8_t* stage = smem + S::Q_OFF + (warp - 4) * (32 * HC * 2);
            float4* part = reinterpret_cast<float4*>(p.part_o) + ((size_t)max(g.slot, 0) * (HD / 4) + st * (HC / 4)) * BQ + r;
#pragma unroll 1
            for (int ch = 0; ch < HC / 32; ++ch) {
              float o[32], a[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = 0.f;
              if (n_st > 0) {
                tmem_ld_32x32(t_mine + ch * 32, a);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = a[i] * w_mine;
              }
              if (n_other > 0) {
                tmem_ld_32x32(t_other + ch * 32, a);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = fmaf(a[i], w_other, o[i]);
              }
              if (g.slot >= 0) {
                if (r < rows) {
#pragma unroll
                  for (int q4 = 0; q4 < 8; ++q4) part[(ch * 8 + q4) * BQ] = make_float4(o[4 * q4], o[4 * q4 + 1], o[4 * q4 + 2], o[4 * q4 + 3]);
                }
              } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= inv;
                stage_row<HC>(stage, lane, ch * 32, o);
              }
            }
            if (g.slot < 0) store_rows<HC>(stage, lane, rows - quarter * 32, [&](int row) { return out_row(quarter * 32 + row) + st * HC; });
            if (st == 0 && r < rows) {
              if (g.slot >= 0) p.part_ml[(size_t)g.slot * BQ + r] = make_float2(m_all * c, l_row);
              else if (lse) *lse = l_row == 0.f ? -INFINITY : (m_all * c) * 0.69314718055994531f + logf(l_row);
            }
          }
          tc_fence_before();
        }
      }
      cnt += n_st;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) tmem_dealloc(tmem_base, kTmemCols);
}

// [rows][heads][head_dim] with any strides as a tensor map of boxes 64 columns x `keys` rows of one head; the dimension with the
// smaller stride comes first.  A dimension of one entry has no stride of its own.
bool make_head_map(CUtensorMap* m, const void* base, int head_dim, uint64_t heads, uint64_t rows, long long head_stride, long long row_stride,
                   int keys, int* head_inner) {
  if (heads == 1) head_stride = head_dim;
  if (rows == 1) row_stride = head_stride * (long long)heads;
  *head_inner = head_stride <= row_stride ? 1 : 0;
  return make_map_3d(m, base, head_dim, *head_inner ? heads : rows, *head_inner ? rows : heads, *head_inner ? head_stride : row_stride,
                     *head_inner ? row_stride : head_stride, *head_inner ? 1 : keys, *head_inner ? keys : 1);
}

template <int HD>
static cudaError_t launch_shares(PackedParams p, cudaStream_t st) {
  static std::atomic<unsigned long long> attr{0};
  auto kern = packed_tc_kernel<HD>;
  if (cudaError_t e = ensure_dyn_smem(kern, Smem<HD>::TOTAL, attr); e != cudaSuccess) return e;
  CUtensorMap mk, mv;
  if (!make_head_map(&mk, p.k, HD, p.kv_heads, p.k_rows, p.k_head, p.k_token, BK, &p.k_head_inner) ||
      !make_head_map(&mv, p.v, HD, p.kv_heads, p.k_rows, p.v_head, p.v_token, BK, &p.v_head_inner))
    return cudaErrorInvalidValue;
  return launch_pdl(kern, dim3((unsigned)p.n_ctas), dim3(kThreads), Smem<HD>::TOTAL, st, 1, mk, mv, p);
}

cudaError_t launch_packed_tc(const PackedParams& p, int head_dim, bool tiles, cudaStream_t st) {
  if (tiles) return launch_packed_tiles(p, head_dim, st);
  return head_dim == 128 ? launch_shares<128>(p, st) : launch_shares<64>(p, st);
}

}  // namespace dare
