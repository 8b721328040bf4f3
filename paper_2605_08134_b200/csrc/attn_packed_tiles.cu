// Packed attention on tensor cores, the form for many rows (attn_packed.h): a CTA has 256 rows of a pair, two streams of 128 (see
// attn_packed_tc.cu for what they share with the form for few), and all keys that they see.
// Key blocks of 128, brought in once for both streams.  A stream has one score buffer of 128 columns (N = 128: the tensor pipe runs at
// two thirds of its rate at 64), so its products and its softmax take turns; the other stream's fill the gaps.  P goes back over
// the scores in two halves of 64 keys, each handed over as soon as it is there.  The scores of block j + 1 come behind the products of
// block j in issue order, so that whoever sees them knows that O is complete up to block j.
#include "attn_packed_tc.cuh"
#include "tc.h"

namespace dare {

using namespace packed_tc;

namespace {
constexpr int TK = 128;                        // keys a block
template <int HD>
struct TileSmem {
  static constexpr int Q_BYTES = BQ * HD * 2, KV_BYTES = TK * HD * 2, RING = 2;
  static constexpr int K_OFF = 2 * Q_BYTES, V_OFF = K_OFF + RING * KV_BYTES, BAR_OFF = V_OFF + RING * KV_BYTES;
  static constexpr int TOTAL = one_cta_per_sm(BAR_OFF + 256 + 1024);
  static_assert(TOTAL <= 232448, "shared memory of one CTA");
};
template <int N>
struct Const { static constexpr int value = N; };
template <int N>
__device__ __forceinline__ void set_registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void set_registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// CTA u's pair.  By a warp.
__device__ __forceinline__ bool tile_segment(Line<2 * BQ, false>& line, unsigned u, Segment* g) {
  const PackedParams& p = line.p;
  if (!line.find(u, &g->pl)) return false;
  const int row0 = g->pl.tile * (2 * BQ);
  g->at = tile_rows(p, row0);
  g->rows = min(2 * BQ, g->pl.s.nq * p.group - row0);
  g->blk0 = 0;
  g->seen = row_sees(p, *g, g->rows - 1);
  g->n_blk = (g->seen + TK - 1) / TK;
  g->slot = -1;
  g->none = false;
  return true;
}
__device__ __forceinline__ int stream_rows(const Segment& g, int st) { return max(0, min(BQ, g.rows - st * BQ)); }
}  // namespace

template <int HD>
__global__ void __launch_bounds__(kThreads, 1)
packed_tiles_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PackedParams p) {
  using S = TileSmem<HD>;
  constexpr int UPR = HD / 8;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);    // [2]
  uint64_t* k_empty = k_full + 2;
  uint64_t* v_full = k_empty + 2;
  uint64_t* v_empty = v_full + 2;
  uint64_t* s_full = v_empty + 2;              // [2 streams]
  uint64_t* p_full = s_full + 2;               // [2 streams][2 halves]
  uint64_t* o_full = p_full + 4;               // [2 streams]: the last product
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_full + 2);
  __shared__ Segment seg_sh;
  __shared__ int seg_more;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 2); mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 2);
      mbar_init(&s_full[i], 1); mbar_init(&o_full[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&p_full[i], kSoftmaxThreads / 64);
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
  if (warp == 1) {
    Line<2 * BQ, false> line(p);
    Segment g;
    const bool more = tile_segment(line, blockIdx.x, &g);
    if (lane == 0) {
      seg_more = more ? 1 : 0;
      if (more) seg_sh = g;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (seg_more) {
    const Segment g = seg_sh;
    auto load_kv = [&](int i) {
      const int slot = i & 1, row = g.pl.s.k0 + i * TK;
      load_block<HD, TK>(smem + S::K_OFF + slot * S::KV_BYTES, &tm_k, p.k_head_inner, g.pl.h, row, &k_full[slot]);
      load_block<HD, TK>(smem + S::V_OFF + slot * S::KV_BYTES, &tm_v, p.v_head_inner, g.pl.h, row, &v_full[slot]);
    };
    if (threadIdx.x == 0)
      for (int i = 0; i < 2 && i < g.n_blk; ++i) load_kv(i);
    // ---- Q rows -> shared memory, K-major, 128-byte swizzle
    if (warp != 0) {
      constexpr int kGather = kThreads - 32, QU = (2 * BQ * UPR + kGather - 1) / kGather;
      const int u0 = (int)threadIdx.x - 32;
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q);
      uint4 qv[QU];
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int w = u0 + i * kGather, r = w / UPR, unit = w % UPR;
        qv[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < g.rows) {
          const RowAt at = row_at(p, g.at, g.pl.h, r);
          qv[i] = __ldcg(reinterpret_cast<const uint4*>(q + (long long)(g.pl.s.q0 + at.query) * p.q_token + at.head * p.q_head + unit * 8));
        }
      }
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int w = u0 + i * kGather, r = w / UPR, unit = w % UPR, rt = r & (BQ - 1);
        if (r < 2 * BQ)
          *reinterpret_cast<uint4*>(smem + (r / BQ) * S::Q_BYTES + (unit >> 3) * (BQ * 128) + rt * 128 + (((unit & 7) ^ (rt & 7)) << 4)) = qv[i];
      }
      fence_proxy_async_smem();
    }
    __syncthreads();

    const int st = warp < 4 ? (warp & 1) : ((warp - 4) >> 2);            // stream
    const int rows = stream_rows(g, st);
    const int n_st = rows > 0 ? min(g.n_blk, (row_sees(p, g, st * BQ + rows - 1) + TK - 1) / TK) : 0;
    const uint32_t tmem_s = tmem_base + st * TK, tmem_o = tmem_base + 2 * TK + st * HD;
    if (warp < 4) {
      set_registers_down<40>();
      if (warp == 0) {
        for (int i = 2; i < g.n_blk; ++i) {
          const int slot = i & 1;
          mbar_wait(&k_empty[slot], ((i >> 1) & 1) ^ 1, p.status);
          mbar_wait(&v_empty[slot], ((i >> 1) & 1) ^ 1, p.status);
          if (elect_one()) load_kv(i);
          __syncwarp();
        }
      } else if (warp >= 2) {
        constexpr uint32_t idesc_qk = idesc_bf16(BQ, TK, false), idesc_pv = idesc_bf16(BQ, HD, true);
        const uint64_t q_desc = smem_desc_k_sw128(smem_u32(smem + st * S::Q_BYTES));
        const uint64_t k_desc0 = smem_desc_k_sw128(smem_u32(smem + S::K_OFF));
        const uint64_t v_desc0 = smem_desc_mn_sw128(smem_u32(smem + S::V_OFF), TK * 128);
        auto issue_qk = [&](int j) {
          const int slot = j & 1;
          mbar_wait(&k_full[slot], (j >> 1) & 1, p.status);
          tc_fence_after();
          if (elect_one()) {
            const uint64_t k_desc = k_desc0 + (uint64_t)(slot * (S::KV_BYTES >> 4));
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk)
              umma_ss(tmem_s, q_desc + (((kk >> 2) * (BQ * 128) + (kk & 3) * 32) >> 4),
                      k_desc + (((kk >> 2) * (TK * 128) + (kk & 3) * 32) >> 4), idesc_qk, kk != 0 ? 1u : 0u);
            umma_commit(&s_full[st]);
            umma_commit(&k_empty[slot]);
          }
          __syncwarp();
        };
        if (n_st > 0) issue_qk(0);
        for (int j = 0; j < n_st; ++j) {
          const int slot = j & 1;
          mbar_wait(&v_full[slot], (j >> 1) & 1, p.status);
          const int keys = g.seen - j * TK;          // (of the tile: the streams share the block, both may write the same zeros)
          if (keys < TK) zero_values<HD, TK>(smem + S::V_OFF + slot * S::KV_BYTES, keys, lane);
          const uint64_t v_desc = v_desc0 + (uint64_t)(slot * (S::KV_BYTES >> 4));
#pragma unroll
          for (int h = 0; h < 2; ++h) {                                   // 64 keys of P each
            mbar_poll(&p_full[2 * st + h], j & 1, p.status);
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < 4; ++ks) {
                const uint64_t v16 = v_desc + (((h * 4 + ks) * (16 * 128)) >> 4);
                umma_ts(tmem_o, tmem_s + h * 32 + ks * 8, v16, idesc_pv, (j | h | ks) != 0 ? 1u : 0u);
                if (kSplitP<HD>) umma_ts(tmem_o, tmem_s + 64 + h * 32 + ks * 8, v16, idesc_pv, 1u);
              }
              if (h == 1) {
                umma_commit(&v_empty[slot]);
                if (j == n_st - 1) umma_commit(&o_full[st]);
              }
            }
            __syncwarp();
          }
          if (j + 1 < n_st) issue_qk(j + 1);
        }
        for (int j = n_st; j < g.n_blk; ++j) {        // blocks that only the other stream's rows see
          const int slot = j & 1;
          mbar_wait(&k_full[slot], (j >> 1) & 1, p.status);
          if (elect_one()) mbar_arrive(&k_empty[slot]);
          __syncwarp();
          mbar_wait(&v_full[slot], (j >> 1) & 1, p.status);
          if (elect_one()) mbar_arrive(&v_empty[slot]);
          __syncwarp();
        }
      }
    } else {
      set_registers_up<232>();
      const int quarter = warp & 3, r = quarter * 32 + lane;
      const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
      const float c = p.scale_log2;
      const bool warp_has_rows = quarter * 32 < rows;
      const RowAt at = row_at(p, g.at, g.pl.h, st * BQ + min(r, max(rows - 1, 0)));
      const int seen = keys_seen(p, g.pl.s, at.query);
      float m = -INFINITY, l = 0.f;
      // The two warps of a scheduler, one of each stream, take turns at the exponentials: side by side they take as long as one after
      // the other, but then both streams' products come at the same time too, and neither unit has anything to do meanwhile.
      // Barrier 1 + quarter: stream 0's turn, 5 + quarter: stream 1's.
      const int turns = max(g.n_blk, 1);
      auto take_turn = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + 4 * st + quarter) : "memory"); };
      auto pass_turn = [&](int j) {
        if (st == 0 || j + 1 < turns) asm volatile("bar.arrive %0, 64;" ::"r"(1 + 4 * (st ^ 1) + quarter) : "memory");
      };
      if (st == 1) asm volatile("bar.arrive %0, 64;" ::"r"(1 + quarter) : "memory");
      for (int j = 0; j < n_st; ++j) {
        mbar_poll(&s_full[st], j & 1, p.status);
        tc_fence_after();
        if (!warp_has_rows) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) { mbar_arrive(&p_full[2 * st]); mbar_arrive(&p_full[2 * st + 1]); }
          take_turn();
          pass_turn(j);
          continue;
        }
        const uint32_t sbuf = tmem_s + lane_addr;
        float v[TK];
#pragma unroll
        for (int i = 0; i < TK; i += 32) tmem_ld_32x32_nowait(sbuf + i, v + i);
        tmem_ld_wait();
        const int keys = seen - j * TK;
        if (__any_sync(0xffffffffu, keys < TK)) {
#pragma unroll
          for (int i = 0; i < TK; ++i)
            if (i >= keys) v[i] = -INFINITY;
        }
        auto row_max = [&]() {
          float mx4[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) mx4[k] = fmaxf(v[k], v[4 + k]);
#pragma unroll
          for (int i = 8; i < TK; i += 8) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mx4[k] = fmax3(mx4[k], v[i + k], v[i + 4 + k]);
          }
          return fmax3(m, fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        };
        if (j == 0) m = row_max();
        // The exponentials are taken against the maximum of the blocks before, so that they need not wait for this one's; only if it
        // has grown by more than 2^8 (any smaller growth changes nothing in exact arithmetic) are the first half's taken again.
        float2 sum2[2];
        float pk[16], pl[kSplitP<HD> ? 16 : 1];
        auto exponentials = [&](auto part) {                               // of 32 keys
          constexpr int k0 = decltype(part)::value * 32;
          const float mc = m == -INFINITY ? 0.f : m * c;                   // (nothing seen yet: 2^-inf = 0, not 2^NaN)
          const float2 c2 = make_float2(c, c), nmc2 = make_float2(-mc, -mc);
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float2 e = __ffma2_rn(make_float2(v[k0 + i], v[k0 + i + 1]), c2, nmc2);
            e.x = fast_exp2(e.x);
            e.y = fast_exp2(e.y);
            sum2[(i >> 1) & 1] = __fadd2_rn(sum2[(i >> 1) & 1], e);
            pack_weights<kSplitP<HD>>(e, pk[i >> 1], pl[kSplitP<HD> ? i >> 1 : 0]);
          }
        };
        auto store_p = [&](int part) {
          tmem_st_32x16_nowait(sbuf + part * 16, pk);
          if constexpr (kSplitP<HD>) tmem_st_32x16_nowait(sbuf + 64 + part * 16, pl);
        };
        auto hand_over = [&](int h) {
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_full[2 * st + h]);
        };
        take_turn();
#pragma unroll 1
        for (;;) {
          sum2[0] = sum2[1] = make_float2(0.f, 0.f);
          exponentials(Const<0>{});
          store_p(0);
          exponentials(Const<1>{});
          store_p(1);
          const float m_new = row_max();
          const bool grow = (m_new - m) * c > kRescaleStep;                // (-inf to -inf: NaN, no)
          if (!__any_sync(0xffffffffu, grow)) break;
          const float alpha = grow ? fast_exp2((m - m_new) * c) : 1.f;
          if (grow) { m = m_new; l *= alpha; }
          if (j > 0) {
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
        exponentials(Const<2>{});
        hand_over(0);                                                      // (the stores have landed meanwhile)
        store_p(2);
        exponentials(Const<3>{});
        pass_turn(j);
        store_p(3);
        hand_over(1);
        l += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
      }
      for (int j = n_st; j < turns; ++j) {
        take_turn();
        pass_turn(j);
      }
      if (n_st > 0) mbar_wait(&o_full[st], 0, p.status);
      tc_fence_after();
      if (warp_has_rows) {
        // (over this warp's rows of the stream's Q tile: its last score product is complete)
        uint8_t* stage = smem + st * S::Q_BYTES + quarter * (32 * HD * 2);
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
        for (int ch = 0; ch < HD / 32; ++ch) {
          float o[32];
          if (n_st > 0) {
            tmem_ld_32x32(tmem_o + lane_addr + ch * 32, o);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] *= inv;
          stage_row<HD>(stage, lane, ch * 32, o);
        }
        const int first = st * BQ + quarter * 32;
        store_rows<HD>(stage, lane, rows - quarter * 32, [&](int row) {
          const RowAt w = row_at(p, g.at, g.pl.h, first + row);
          return reinterpret_cast<__nv_bfloat16*>(p.o) + (long long)(g.pl.s.q0 + w.query) * p.o_token + w.head * p.o_head;
        });
        if (p.lse && r < rows)
          p.lse[(long long)(g.pl.s.q0 + at.query) * p.n_heads + at.head] = l == 0.f ? -INFINITY : (m * c) * 0.69314718055994531f + logf(l);
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) tmem_dealloc(tmem_base, kTmemCols);
}

template <int HD>
static cudaError_t launch_tiles(PackedParams p, cudaStream_t st) {
  static std::atomic<unsigned long long> attr{0};
  auto kern = packed_tiles_kernel<HD>;
  if (cudaError_t e = ensure_dyn_smem(kern, TileSmem<HD>::TOTAL, attr); e != cudaSuccess) return e;
  CUtensorMap mk, mv;
  if (!make_head_map(&mk, p.k, HD, p.kv_heads, p.k_rows, p.k_head, p.k_token, TK, &p.k_head_inner) ||
      !make_head_map(&mv, p.v, HD, p.kv_heads, p.k_rows, p.v_head, p.v_token, TK, &p.v_head_inner))
    return cudaErrorInvalidValue;
  // as many CTAs as there can be pairs (a sequence's last tile may be partly filled); those behind the last one leave
  const long long grid = ((p.q_rows * p.group) / (2 * BQ) + p.batch) * p.kv_heads;
  return launch_pdl(kern, dim3((unsigned)grid), dim3(kThreads), TileSmem<HD>::TOTAL, st, 1, mk, mv, p);
}
cudaError_t launch_packed_tiles(const PackedParams& p, int head_dim, cudaStream_t st) {
  return head_dim == 128 ? launch_tiles<128>(p, st) : launch_tiles<64>(p, st);
}

}  // namespace dare
