// Device helpers of the packed attention's tensor-core kernels.
#pragma once

#include "attn_packed.h"
#include "tc_ptx.cuh"

namespace dare {
namespace packed_tc {

using namespace ptx;

constexpr int BQ = kTcRows, kThreads = 384, kSoftmaxThreads = 256;
constexpr uint32_t kTmemCols = 512;
constexpr float kRescaleStep = 8.f;        // log2 of the growth of a row's maximum that has O rescaled
// Heads of 64: P as two bf16 parts, the rounded weight and what the rounding left (16 bits together), each multiplied with V: together they
// take the columns that the scores had.  As in the layer's attention: see attn_packed_tc.cu.
template <int HD>
constexpr bool kSplitP = HD == 64;
// Two weights as bf16, and of two parts what that leaves of them.
template <bool SPLIT>
__device__ __forceinline__ void pack_weights(float2 e, float& high, float& low) {
  const __nv_bfloat162 h2 = __floats2bfloat162_rn(e.x, e.y);
  high = __uint_as_float(*reinterpret_cast<const uint32_t*>(&h2));
  if constexpr (SPLIT) {
    const float2 rest = __fadd2_rn(e, make_float2(-__low2float(h2), -__high2float(h2)));
    const __nv_bfloat162 l2 = __floats2bfloat162_rn(rest.x, rest.y);
    low = __uint_as_float(*reinterpret_cast<const uint32_t*>(&l2));
  }
}
constexpr int one_cta_per_sm(int bytes) { return bytes > 117 * 1024 ? bytes : 117 * 1024; }   // (a CTA takes all tensor memory)

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* tmap, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
// KEYS rows of a head: HD / 64 chunks of 64 columns, counted on one barrier
template <int HD, int KEYS>
__device__ __forceinline__ void load_block(uint8_t* dst, const CUtensorMap* tm, bool head_inner, int h, int row, uint64_t* bar) {
  mbar_arrive_expect_tx(bar, KEYS * HD * 2);
#pragma unroll
  for (int c = 0; c < HD / 64; ++c)
    tma_load_3d(dst + c * (KEYS * 128), tm, c * 64, head_inner ? h : row, head_inner ? row : h, bar);
}

// 32 finished rows of a warp, thread <-> row, 32 columns at a time: through shared memory (16-byte units swizzled by
// row), from where neighbouring lanes take neighbouring units: stores straight from the threads' rows touch 32 lines each, 2 us a
// tile of 128 rows.
template <int COLS>
__device__ __forceinline__ int stage_at(int row, int unit) {
  constexpr int UPR = COLS / 8;                                       // units a row
  return row * (COLS * 2) + ((unit ^ (row & (UPR < 8 ? UPR - 1 : 7))) << 4);
}
template <int COLS>
__device__ __forceinline__ void stage_row(uint8_t* stage, int lane, int col, const float (&o)[32]) {
#pragma unroll
  for (int q4 = 0; q4 < 4; ++q4) *reinterpret_cast<uint4*>(stage + stage_at<COLS>(lane, col / 8 + q4)) = pack8_bf16(o + 8 * q4);
}
template <int COLS, typename F>
__device__ __forceinline__ void store_rows(const uint8_t* stage, int lane, int rows, F&& row_ptr) {
  constexpr int UPR = COLS / 8, RPI = 32 / UPR;                       // rows an instruction
  __syncwarp();
#pragma unroll 4
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = i * RPI + lane / UPR, unit = lane % UPR;
    if (r < rows) reinterpret_cast<uint4*>(row_ptr(r))[unit] = *reinterpret_cast<const uint4*>(stage + stage_at<COLS>(r, unit));
  }
  __syncwarp();
}

// What a CTA does with one pair, or a part of its keys.
struct Segment {
  Place pl;
  TileRows at;                   // where the CTA's rows begin
  int rows;                      // its rows
  int seen;                      // keys that the last of them sees: none of its rows sees more
  int blk0, n_blk;               // blocks of keys [blk0, blk0 + n_blk)
  int slot;                      // < 0: the rows' keys are all here; else the slot of the partial result
  bool none;                     // the share ends before the pair's keys begin
};
// keys that row `row` of the segment sees
__device__ __forceinline__ int row_sees(const PackedParams& p, const Segment& g, int row) {
  return keys_seen(p, g.pl.s, row_at(p, g.at, 0, row).query);
}
// Values of a block of BLK keys (HD / 64 chunks of 64 columns) from row `keys` on become zeros, by the warp that issues their product: what
// lies there is hidden from all rows or another sequence's, may be anything, and 0 * inf would be NaN.
template <int HD, int BLK>
__device__ __forceinline__ void zero_values(uint8_t* v, int keys, int lane) {
  constexpr int UPR = HD / 8;
  for (int i = lane; i < (BLK - keys) * UPR; i += 32) {
    const int r = keys + i / UPR, unit = i % UPR;
    *reinterpret_cast<uint4*>(v + (unit >> 3) * (BLK * 128) + r * 128 + ((unit & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async_smem();
  __syncwarp();
}

}  // namespace packed_tc

// Tensor map of k or v in boxes of 64 columns x `keys` rows of one head; *head_inner: which dimension comes first.
bool make_head_map(CUtensorMap* m, const void* base, int head_dim, uint64_t heads, uint64_t rows, long long head_stride, long long row_stride,
                   int keys, int* head_inner);
// 256 rows a CTA (attn_packed_tiles.cu)
cudaError_t launch_packed_tiles(const PackedParams& p, int head_dim, cudaStream_t st);

}  // namespace dare
