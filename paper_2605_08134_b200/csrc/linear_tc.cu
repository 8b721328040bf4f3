// y = act(x W^T + bias) + resid in bf16 on tcgen05 tensor cores, any number of rows and outputs (dare_ops.h).
// Persistent: a CTA (or a pair of CTAs sharing M = 256 MMAs, cta_group::2) walks output tiles of 128 (256) rows x `width` columns, the
// finishing pass of a tile running beside the next one's main loop.  The width is not fixed: it is what the launch rule below
// finds cheapest, a multiple of 16 up to 256; where there are few tiles, the rule may share a tile's k-elements between CTAs (the
// second kernel).  Of few rows only those there are come into shared memory (the MMA's other rows read whatever follows, and nobody
// reads their results), which leaves up to 12 stages of W on their way.
//   warp 0     TMA producer: rows of x and of W, 128 k-elements a stage in two boxes of 64 columns each (256 bytes of a row of W come
//              from one place of the HBM at a time); rows, columns and k-elements past the end are zeros
//   warp 1     MMA issuer (of a pair: the even CTA's), two accumulators of up to 256 columns of tensor memory in turn
//   warps 2-9  finishing pass, two warps a lane quarter, thread <-> row, 32 columns at a time: bias, activation, residual, store
#include "linear.h"
#include "tc.h"
#include "tc_ptx.cuh"

namespace dare {

using namespace ptx;

namespace {
constexpr int BM = 128, BK = 128, kFinish = 8, kThreads = (2 + kFinish) * 32;
constexpr int kRing = 192 * 1024, kMaxStages = 12;
constexpr int HALF_X = BM * 128;                           // 128 rows of 64 k-elements, what an MMA reads as its rows of x ...
constexpr int BIAS_OFFSET = kRing + HALF_X;                // ... from where a stage's begin, however few it has
constexpr int kBiasCols = 128;                             // a finishing warp's columns of the widest tile
constexpr int BAR_OFFSET = BIAS_OFFSET + kFinish * kBiasCols * 4;
constexpr int SMEM_TOTAL = BAR_OFFSET + 512 + 1024;
static_assert(SMEM_TOTAL <= 227 * 1024 && (2 * kMaxStages + 4) * 8 + 4 <= 512, "shared memory of one CTA");
constexpr int kGroupBytes = 24 << 20;                      // column tiles are walked in groups of this much of W, as in gemm_persist.cu

struct TileWalk {
  int width, x_rows;          // columns of a tile; rows of x a stage holds
  int n_tiles, m_units;       // column tiles; row tiles (PAIR: pairs of them)
  int n_group;
  int wide_y;                 // y (and resid) by 16 bytes
};

template <bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
linear_tc_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const LinearParams p,
                 const TileWalk t) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + BAR_OFFSET);
  uint64_t* empty_bar = full_bar + kMaxStages;
  uint64_t* acc_full = empty_bar + kMaxStages;       // [2]
  uint64_t* acc_empty = acc_full + 2;                // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int pr = PAIR ? (int)cluster_ctarank() : 0;
  const int walker = PAIR ? (int)blockIdx.x / 2 : (int)blockIdx.x, n_walkers = PAIR ? (int)gridDim.x / 2 : (int)gridDim.x;
  const int w_rows = PAIR ? t.width / 2 : t.width, x_bytes = t.x_rows * BK * 2, w_bytes = w_rows * BK * 2, stage_bytes = x_bytes + w_bytes;
  const int stages = min(kMaxStages, kRing / stage_bytes), KB = (p.k + BK - 1) / BK, k16 = (p.k + 15) / 16 * 16;
  const int total = t.n_tiles * t.m_units;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], PAIR ? 2 * kFinish : kFinish); }
    fence_mbar_init();
    prefetch_tmap(&tm_x);
    prefetch_tmap(&tm_w);
  }
  if (warp == 1) {
    if (PAIR) { tmem_alloc2(tmem_slot, 512); tmem_relinquish2(); }
    else { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
  }
  tc_fence_before();
  __syncthreads();
  uint32_t tmem_base;
  if (PAIR) {
    cluster_sync_all();              // both CTAs have their barriers and tensor memory before either touches the other's
    tc_fence_after();
    tmem_base = ld_cluster_u32(map_to_cta(smem_u32(tmem_slot), 0));
  } else {
    tc_fence_after();
    tmem_base = *tmem_slot;
  }
  pdl_wait();
  pdl_launch_dependents();

  auto tile_of = [&](int u, int* m0, int* n0) {
    int width = t.n_tiles, nt0 = 0, r = u;
    if (t.n_group < t.n_tiles) {
      const int in_group = t.n_group * t.m_units, grp = u / in_group;
      r = u - grp * in_group;
      nt0 = grp * t.n_group;
      width = min(t.n_group, t.n_tiles - nt0);
    }
    const int mu = r / width;
    *m0 = (PAIR ? 2 * mu + pr : mu) * BM;
    *n0 = (nt0 + r - mu * width) * t.width;
  };
  if (warp == 0) {
    uint32_t it = 0;
    for (int u = walker; u < total; u += n_walkers) {
      int m0, n0;
      tile_of(u, &m0, &n0);
      for (int kb = 0; kb < KB; ++kb, ++it) {
        const int s = it % stages;
        mbar_wait(&empty_bar[s], ((it / stages) & 1) ^ 1, p.status);
        if (elect_one()) {
          uint8_t* dst = smem + s * stage_bytes;
          const uint32_t fb = PAIR ? map_to_cta(smem_u32(&full_bar[s]), 0) : 0;
          // (PAIR: the bytes of both CTAs are counted on the even one's barrier)
          if (!PAIR) mbar_arrive_expect_tx(&full_bar[s], (uint32_t)stage_bytes);
          else if (pr == 0) mbar_arrive_expect_tx(&full_bar[s], 2u * stage_bytes);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int k0 = kb * BK + h * 64;
            if (PAIR) {
              tma_load_2d_pair(dst + h * (x_bytes / 2), &tm_x, k0, m0, fb);
              tma_load_2d_pair(dst + x_bytes + h * (w_bytes / 2), &tm_w, k0, n0 + pr * w_rows, fb);
            } else {
              tma_load_2d(dst + h * (x_bytes / 2), &tm_x, k0, m0, &full_bar[s]);
              tma_load_2d(dst + x_bytes + h * (w_bytes / 2), &tm_w, k0, n0, &full_bar[s]);
            }
          }
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    if (pr == 0) {
      const uint32_t idesc = idesc_bf16(PAIR ? 2 * BM : BM, t.width);
      uint32_t it = 0, tcount = 0;
      for (int u = walker; u < total; u += n_walkers, ++tcount) {
        const uint32_t buf = tcount & 1, d_tmem = tmem_base + buf * 256;
        mbar_wait(&acc_empty[buf], ((tcount >> 1) & 1) ^ 1, p.status);
        tc_fence_after();
        for (int kb = 0; kb < KB; ++kb, ++it) {
          const int s = it % stages;
          mbar_poll(&full_bar[s], (it / stages) & 1, p.status);
          tc_fence_after();
          if (elect_one()) {
            const uint32_t at = smem_u32(smem + s * stage_bytes);
            const uint64_t a = smem_desc_k_sw128(at), b = smem_desc_k_sw128(at + x_bytes);
            const int steps = min(BK, k16 - kb * BK) / 16;          // (the last block's k-elements past the end are not there)
#pragma unroll
            for (int k = 0; k < BK / 16; ++k) {
              if (k >= steps) break;
              const uint64_t ak = a + (k >> 2) * (uint32_t)(x_bytes >> 5) + 2 * (k & 3), bk = b + (k >> 2) * (uint32_t)(w_bytes >> 5) + 2 * (k & 3);
              if (PAIR) umma2_ss(d_tmem, ak, bk, idesc, (kb | k) != 0 ? 1u : 0u);
              else umma_ss(d_tmem, ak, bk, idesc, (kb | k) != 0 ? 1u : 0u);
            }
            if (PAIR) {
              umma2_commit(map_to_cta(smem_u32(&empty_bar[s]), 0));
              umma2_commit(map_to_cta(smem_u32(&empty_bar[s]), 1));
              if (kb == KB - 1) {
                umma2_commit(map_to_cta(smem_u32(&acc_full[buf]), 0));
                umma2_commit(map_to_cta(smem_u32(&acc_full[buf]), 1));
              }
            } else {
              umma_commit(&empty_bar[s]);
              if (kb == KB - 1) umma_commit(&acc_full[buf]);
            }
          }
          __syncwarp();
        }
      }
    }
  } else {
    const int q = warp & 3, sub = (warp - 2) >> 2;
    uint32_t tcount = 0;
    for (int u = walker; u < total; u += n_walkers, ++tcount) {
      int m0, n0;
      tile_of(u, &m0, &n0);
      const uint32_t buf = tcount & 1;
      // (the warp's part of the bias while the tile is multiplied: read where it is used, it held every 32 columns up for 0.7 us)
      const int cols = min(t.width, p.n - n0);
      float* bias_sh = reinterpret_cast<float*>(smem + BIAS_OFFSET) + (warp - 2) * kBiasCols;
      if (p.bias) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kBiasCols; i += 32) {
          const int e = i + lane, run = t.wide_y ? 31 : 15;          // the warps of a quarter take runs of 32 (16) columns in turn
          const int c = 2 * (e & ~run) + sub * (run + 1) + (e & run);
          if (c < cols) bias_sh[e] = p.bias[n0 + c];
        }
        __syncwarp();
      }
      uint8_t* stg = smem + kRing + (warp - 2) * 2048;
      const int pr8 = lane >> 2, unit = lane & 3, rows = p.rows - (m0 + q * 32);
      const long long piece = (long long)(m0 + q * 32 + pr8);
      __nv_bfloat16* yp = reinterpret_cast<__nv_bfloat16*>(p.y) + piece * p.y_row + n0 + unit * 8;
      const __nv_bfloat16* rp = p.resid ? reinterpret_cast<const __nv_bfloat16*>(p.resid) + piece * p.resid_row + n0 + unit * 8 : nullptr;
      uint4 rs[4];                   // of 32 rows x 32 columns of resid; the next ones come while these are used
      auto load_resid = [&](int c) {
        if (rp == nullptr || !t.wide_y || c + 32 > cols) return;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i * 8 + pr8 < rows) rs[i] = *reinterpret_cast<const uint4*>(rp + c + i * 8 * p.resid_row);
      };
      load_resid(sub * 32);
      mbar_wait(&acc_full[buf], (tcount >> 1) & 1, p.status);
      tc_fence_after();
      const uint32_t t_lane = tmem_base + buf * 256 + ((uint32_t)(q * 32) << 16);
      const int row = m0 + q * 32 + lane;
      const bool warp_has_rows = m0 + q * 32 < p.rows;
      __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(p.y) + (long long)row * p.y_row + n0;
      const __nv_bfloat16* resid = p.resid ? reinterpret_cast<const __nv_bfloat16*>(p.resid) + (long long)row * p.resid_row + n0 : nullptr;
      if (warp_has_rows && t.wide_y) {
        // 32 rows x 32 columns at a time between the threads' rows and whole 64-byte pieces of y and resid, through 2 KB of shared
        // memory (past the ring; 16-byte units swizzled by row).  Stores straight from the threads' rows touch 32 lines each.
        auto place = [&](int r, int u) { return reinterpret_cast<uint4*>(stg + r * 64 + ((u ^ ((r >> 1) & 3)) << 4)); };
#pragma unroll 1
        for (int c = sub * 32; c < cols; c += 64) {
          const bool full = c + 32 <= cols;
          float v[32];
          tmem_ld_32x32_nowait(t_lane + c, v);
          tmem_ld_wait();
          if (p.bias) {
            const float4* b = reinterpret_cast<const float4*>(bias_sh + ((c >> 1) & ~31));        // (columns past the end: anything)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 f = b[i];
              v[4 * i] += f.x; v[4 * i + 1] += f.y; v[4 * i + 2] += f.z; v[4 * i + 3] += f.w;
            }
          }
          activate<true>(v, p.act);
          if (full) {
            if (resid) {
#pragma unroll
              for (int i = 0; i < 4; ++i) *place(i * 8 + pr8, unit) = rs[i];
              load_resid(c + 64);
              __syncwarp();
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint4 raw = *place(lane, i);
                const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float2 f = __bfloat1622float2(h[e]);
                  v[8 * i + 2 * e] += f.x;
                  v[8 * i + 2 * e + 1] += f.y;
                }
              }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) *place(lane, i) = pack8_bf16(v + 8 * i);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i * 8 + pr8 < rows) *reinterpret_cast<uint4*>(yp + c + i * 8 * p.y_row) = *place(i * 8 + pr8, unit);
          } else if (row < p.rows) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c + i < cols) {
                float o = v[i];
                if (resid) o += __bfloat162float(resid[c + i]);
                y[c + i] = __float2bfloat16_rn(o);
              }
          }
          __syncwarp();
        }
      } else if (warp_has_rows) {
        // Rows of y or resid that are not on the 16-byte grid: 16 columns at a time through 2 KB of shared memory (the rows that the
        // last stage's MMA reads past its own; units of 16 bytes swizzled by row), from where half a warp takes a row: 2-byte
        // stores of 32 rows at a time took as long as the main loop (3080 x 6400 x 1899: 111 us, 64 so).
        float* stg_f = reinterpret_cast<float*>(stg);
        const int lr = lane >> 4, lc = lane & 15;
#pragma unroll 1
        for (int c = sub * 16; c < cols; c += 32) {
          float v[16];
          tmem_ld_32x16_nowait(t_lane + c, v);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<float4*>(stg_f + lane * 16 + ((i ^ ((lane >> 1) & 3)) << 2)) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          __syncwarp();
          const bool there = c + lc < cols;
          const float bias = p.bias ? bias_sh[((c >> 1) & ~15) + lc] : 0.f;
          float o[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = 2 * i + lr;
            o[i] = stg_f[r * 16 + ((((lc >> 2) ^ ((r >> 1) & 3)) << 2) | (lc & 3))] + bias;
          }
          activate<true>(o, p.act);
          const long long row0 = m0 + q * 32 + lr;
          const __nv_bfloat16* rp = reinterpret_cast<const __nv_bfloat16*>(p.resid) + (p.resid ? row0 * p.resid_row + n0 + c + lc : 0);
          __nv_bfloat16* yp = reinterpret_cast<__nv_bfloat16*>(p.y) + row0 * p.y_row + n0 + c + lc;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (there && 2 * i + lr < rows) {
              if (p.resid) o[i] += __bfloat162float(rp[2 * i * p.resid_row]);
              yp[2 * i * p.y_row] = __float2bfloat16_rn(o[i]);
            }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) mbar_arrive_cluster(map_to_cta(smem_u32(&acc_empty[buf]), 0));
        else mbar_arrive(&acc_empty[buf]);
      }
    }
  }
  tc_fence_before();
  if (PAIR) cluster_sync_relaxed(); else __syncthreads();      // nobody frees tensor memory its partner's MMAs may still use
  if (warp == 1) {
    if (PAIR) tmem_dealloc2(*tmem_slot, 512);
    else tmem_dealloc(*tmem_slot, 512);
  }
}

// ------------------------------------------------------------------------------------------------ few tiles
// A tile's k-blocks shared by a cluster of S CTAs (blockIdx.z), one tile a cluster: tiles stay wide (an SM brings in 128 rows of x for a
// tile however narrow it is) and every SM still has work.  Each CTA leaves its sums in shared memory, over the ring, and finishes its
// part of the tile from everybody's, in the order of the k-elements.  Warps 0 and 1 as above, all warps finish.
template <int S>
__global__ void __launch_bounds__(kThreads, 1)
linear_split_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const LinearParams p,
                    const TileWalk t) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + BAR_OFFSET);
  uint64_t* empty_bar = full_bar + kMaxStages;
  uint64_t* acc_full = empty_bar + kMaxStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 4);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int x_bytes = t.x_rows * BK * 2, w_bytes = t.width * BK * 2, stage_bytes = x_bytes + w_bytes;
  const int stages = min(kMaxStages, kRing / stage_bytes), all = (p.k + BK - 1) / BK, k16 = (p.k + 15) / 16 * 16;
  const int z = (int)blockIdx.z, kb0 = z * all / S, kb1 = (z + 1) * all / S;
  const int n0 = (int)blockIdx.x * t.width, m0 = (int)blockIdx.y * BM;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
    mbar_init(acc_full, 1);
    fence_mbar_init();
    prefetch_tmap(&tm_x);
    prefetch_tmap(&tm_w);
  }
  if (warp == 1) { tmem_alloc(tmem_slot, 256); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();
  // What a thread finishes: eight columns of a row at a time.  Bias and residual of its first eight come beside the main loop.
  const int rows = min(BM, p.rows - m0), eights = t.width / 8, items = rows * eights, first = z * items / S, last = (z + 1) * items / S;
  float bias[8];
  uint4 rs;
  auto fetch = [&](int e) {
    const int r = e / eights, n = n0 + (e - r * eights) * 8;
    if (e >= last || n >= p.n) return;
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 8; ++i) bias[i] = p.bias[min(n + i, p.n - 1)];
    }
    if (p.resid && t.wide_y && n + 8 <= p.n)
      rs = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.resid) + (long long)(m0 + r) * p.resid_row + n);
  };
  if (warp == 0) {
    for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
      const int s = it % stages;
      mbar_wait(&empty_bar[s], ((it / stages) & 1) ^ 1, p.status);
      if (elect_one()) {
        uint8_t* dst = smem + s * stage_bytes;
        mbar_arrive_expect_tx(&full_bar[s], (uint32_t)stage_bytes);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k0 = kb * BK + h * 64;
          tma_load_2d(dst + h * (x_bytes / 2), &tm_x, k0, m0, &full_bar[s]);
          tma_load_2d(dst + x_bytes + h * (w_bytes / 2), &tm_w, k0, n0, &full_bar[s]);
        }
      }
      __syncwarp();
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_bf16(BM, t.width);
    for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
      const int s = it % stages;
      mbar_poll(&full_bar[s], (it / stages) & 1, p.status);
      tc_fence_after();
      if (elect_one()) {
        const uint32_t at = smem_u32(smem + s * stage_bytes);
        const uint64_t a = smem_desc_k_sw128(at), b = smem_desc_k_sw128(at + x_bytes);
        const int steps = min(BK, k16 - kb * BK) / 16;
#pragma unroll
        for (int k = 0; k < BK / 16; ++k) {
          if (k >= steps) break;
          umma_ss(tmem_base, a + (k >> 2) * (uint32_t)(x_bytes >> 5) + 2 * (k & 3), b + (k >> 2) * (uint32_t)(w_bytes >> 5) + 2 * (k & 3), idesc,
                  (it | k) != 0 ? 1u : 0u);
        }
        umma_commit(&empty_bar[s]);
        if (kb == kb1 - 1) umma_commit(acc_full);
      }
      __syncwarp();
    }
  }
  __syncwarp();
  fetch(first + (int)threadIdx.x);
  // ---- tensor memory -> shared memory (idle: every MMA is complete, so every load is), thread <-> row
  float* tile = reinterpret_cast<float*>(smem);
  const int pitch = t.width + 4;
  if (warp >= 2) {
    const int q = warp & 3, sub = (warp - 2) >> 2;
    mbar_wait(acc_full, 0, p.status);
    tc_fence_after();
    if (q * 32 < rows) {
      float* dst = tile + (q * 32 + lane) * pitch;
#pragma unroll 2
      for (int c = sub * 16; c < t.width; c += 32) {
        float v[16];
        tmem_ld_32x16_nowait(tmem_base + ((uint32_t)(q * 32) << 16) + c, v);
        tmem_ld_wait();
        if (q * 32 + lane < rows) {
#pragma unroll
          for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(dst + c + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) tmem_dealloc(tmem_base, 256);
  // ---- eight columns a thread
  for (int e = first + (int)threadIdx.x; e < last; e += kThreads) {
    const int r = e / eights, c = (e - r * eights) * 8;
    const uint32_t at = smem_u32(tile + r * pitch + c);
    float4 a[S], b[S];                // (all of them on their way at once)
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const uint32_t from = map_to_cta(at, (uint32_t)s);
      a[s] = ld_cluster_f4(from);
      b[s] = ld_cluster_f4(from + 16);
    }
    float v[8] = {};
#pragma unroll
    for (int s = 0; s < S; ++s) {
      v[0] += a[s].x; v[1] += a[s].y; v[2] += a[s].z; v[3] += a[s].w;
      v[4] += b[s].x; v[5] += b[s].y; v[6] += b[s].z; v[7] += b[s].w;
    }
    const int cols = p.n - (n0 + c);
    if (cols <= 0) continue;
    if (e != first + (int)threadIdx.x) fetch(e);
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += bias[i];
    }
    activate<true>(v, p.act);
    const long long row = m0 + r;
    __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(p.y) + row * p.y_row + n0 + c;
    const __nv_bfloat16* resid = p.resid ? reinterpret_cast<const __nv_bfloat16*>(p.resid) + row * p.resid_row + n0 + c : nullptr;
    if (t.wide_y && cols >= 8) {
      if (resid) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&rs);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = __bfloat1622float2(h[i]);
          v[2 * i] += f.x;
          v[2 * i + 1] += f.y;
        }
      }
      *reinterpret_cast<uint4*>(y) = pack8_bf16(v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < cols) y[i] = __float2bfloat16_rn(resid ? v[i] + __bfloat162float(resid[i]) : v[i]);
    }
  }
  __syncwarp();
  cluster_sync_all();                // nobody leaves while its sums are read
}

// Tile width and form: waves of tiles times what a k-block takes an SM (the tensor pipe's cycles, or the operand bytes
// at 64 a cycle), plus the finishing pass of the last tile.  us by width, p: pairs, the pick in brackets:
//   37 rows of 4096 x 12288   48 27.7, 64 28.5, [96 21.3], 128 21.9, 160 23.6, 192 24.2, 256 32.5
//   256 of 4096 x 4096        64 15.8, 96 18.3, 128 19.1, [p64 15.0], p96 16.0, p128 16.3, p256 24.7
//   256 of 4096 x 12288       96 35.9, 192 33.8, p96 30.9, p160 41.0, [p192 28.1], p224 29.5, p256 30.9
//   512 of 4096 x 4096        96 30.7, 128 19.2, p96 25.3, [p128 16.9], p160 21.2, p256 25.0
//   2048 of 4096 x 4096       128 64.5, 256 59.6, p128 53.6, p160 52.1, p224 59.0, [p256 49.2]
// At the ten sizes timed (8 to 2048 rows) the pick was the fastest or within 0.4 us of it.
struct Form { int pair, width, splits; };
Form pick_form(int rows, int n, int k) {
  const int m_tiles = (rows + BM - 1) / BM, KB = (k + BK - 1) / BK, x_rows = rows < BM ? (rows + 7) / 8 * 8 : BM;
  Form best{0, 16, 1};
  float least = 1e30f, best_block = 0.f;
  for (int pair = 0; pair <= (m_tiles > 1 ? 1 : 0); ++pair)
    for (int width = pair ? 32 : 16; width <= 256; width += pair ? 32 : 16) {
      const int units = (n + width - 1) / width * (pair ? (m_tiles + 1) / 2 : m_tiles), slots = pair ? kSms / 2 : kSms;
      const float waves = (float)((units + slots - 1) / slots);
      const float mma = 8.f * fmaxf(48.f, 129.f * (float)width / 256.f);
      const float feed = (float)(x_rows + (pair ? width / 2 : width)) * (float)(BK * 2) / 64.f;
      const float block = waves * fmaxf(mma, feed), cycles = block * (float)KB + 6.f * (float)width;
      if (cycles < least) { least = cycles; best = Form{pair, width, 1}; best_block = fmaxf(block, 590.f * waves); }
    }
  // Shared k-elements: what that takes in us, the larger of the SMs' and the memory's time and a fifth of the other, against the same for
  // the tile found above (where a block of k-elements takes 590 cycles at least).  A tile's own time is 3.2 us and 0.2 us a 1000
  // elements of it.  Whole tiles / two / four / eight CTAs a tile, the pick in brackets:
  //   8 rows of 12288 x 4096   35.7 / 24.1 / [19.8] / 24.8       64 of 8192 x 1000   25.2 / 14.9 / 10.1 / [9.2]
  //   100 of 10000 x 200       30.2 / 17.3 / 10.3 / [7.6]        128 of 12288 x 512  36.8 / 20.8 / 12.9 / [10.3]
  //   512 of 8192 x 1024       22.8 / 18.0 / [15.9] / 38.2       256 of 4096 x 4096  [14.9] / 14.5 / 20.7
  //   1024 of 1024 x 1024      [6.6] / 8.5 / 14.1                16 of 4096 x 6144   16.6 / 12.5 / [12.5] / 18.0
  // Of 22 such sizes the pick was at most 10 % behind the fastest.  (More tiles than clusters that fit beside one another: two waves.)
  if ((long long)m_tiles * ((n + 255) / 256) > 2 * kSms) return best;
  constexpr int kClusters[3] = {72, 32, 14};
  const float memory = 2.f * ((float)rows * (float)k + (float)n * (float)k + (float)rows * (float)n) / 6.5e6f;
  auto both = [](float a, float b) { return fmaxf(a, b) + 0.2f * fminf(a, b); };
  float least_us = both((best_block * (float)KB + 6.f * (float)best.width) / 1900.f + 4.f, memory + 4.f);
  for (int i = 0; i < 3 && 2 << i <= KB; ++i)
    for (int width = 16; width <= 256 && width < n + 16; width += 16) {
      const int tiles = m_tiles * ((n + width - 1) / width);
      const float block = fmaxf(590.f, fmaxf(8.f * 129.f * (float)width / 256.f, (float)(x_rows + width) * (float)(BK * 2) / 64.f)) / 1900.f;
      const float own = 0.0002f * (float)(x_rows * width);
      const float us = both((float)((tiles + kClusters[i] - 1) / kClusters[i]) * ((float)((KB + (2 << i) - 1) >> (i + 1)) * block + 3.2f + own),
                            memory + 3.2f + 0.5f * own);
      if (us < least_us) { least_us = us; best = Form{0, width, 2 << i}; }
    }
  return best;
}
}  // namespace

template <int S>
static cudaError_t launch_split(const CUtensorMap& mx, const CUtensorMap& mw, const LinearParams& p, const TileWalk& t, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  if (cudaError_t e = ensure_dyn_smem(linear_split_kernel<S>, SMEM_TOTAL, done); e != cudaSuccess) return e;
  return launch_pdl(linear_split_kernel<S>, dim3((unsigned)t.n_tiles, (unsigned)t.m_units, S), dim3(kThreads), SMEM_TOTAL, st, S, mx, mw, p, t);
}
cudaError_t launch_linear_tc(const LinearParams& p, cudaStream_t st) {
  const Form f = pick_form(p.rows, p.n, p.k);
  const int m_tiles = (p.rows + BM - 1) / BM;
  TileWalk t = {};
  t.width = f.width;
  t.x_rows = !f.pair && p.rows < BM ? (p.rows + 7) / 8 * 8 : BM;
  t.n_tiles = (p.n + f.width - 1) / f.width;
  t.m_units = f.pair ? (m_tiles + 1) / 2 : m_tiles;
  const long long tile_bytes = (long long)f.width * p.k * 2;
  t.n_group = (int)(kGroupBytes / tile_bytes > 0 ? kGroupBytes / tile_bytes : 1);
  auto aligned = [](const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; };
  t.wide_y = aligned(p.y) && p.y_row % 8 == 0 && (!p.resid || (aligned(p.resid) && p.resid_row % 8 == 0));
  // (one row, one output: no stride of its own)
  const uint64_t k8 = ((uint64_t)p.k + 7) / 8 * 8;
  CUtensorMap mx, mw;
  if (!make_map_strided(&mx, p.x, p.rows, p.k, p.rows == 1 ? k8 : p.x_row, t.x_rows) ||
      !make_map_strided(&mw, p.w, p.n, p.k, p.n == 1 ? k8 : p.w_row, f.pair ? f.width / 2 : f.width))
    return cudaErrorInvalidValue;
  if (f.splits == 2) return launch_split<2>(mx, mw, p, t, st);
  if (f.splits == 4) return launch_split<4>(mx, mw, p, t, st);
  if (f.splits == 8) return launch_split<8>(mx, mw, p, t, st);
  const long long units = (long long)t.n_tiles * t.m_units;
  static std::atomic<unsigned long long> done1{0}, done2{0};
  if (f.pair) {
    if (cudaError_t e = ensure_dyn_smem(linear_tc_kernel<true>, SMEM_TOTAL, done2); e != cudaSuccess) return e;
    return launch_pdl_xz(linear_tc_kernel<true>, dim3(2 * (unsigned)(units < kSms / 2 ? units : kSms / 2)), dim3(kThreads), SMEM_TOTAL, st,
                         2, 1, mx, mw, p, t);
  }
  if (cudaError_t e = ensure_dyn_smem(linear_tc_kernel<false>, SMEM_TOTAL, done1); e != cudaSuccess) return e;
  return launch_pdl(linear_tc_kernel<false>, dim3((unsigned)(units < kSms ? units : kSms)), dim3(kThreads), SMEM_TOTAL, st, 1, mx, mw, p, t);
}

}  // namespace dare
