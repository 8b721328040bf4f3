// Attention over packed sequences (dare_ops.h): what its kernels share: the geometry of a sequence and the shares of work.
//
// Rows: the queries of the G heads that share a key/value head are rows of one matrix, row R = (query R / G, head R % G), so that a
// key is brought in once for all of them and one query a sequence still gives G rows to a tile.
// Work comes in pairs (tile of BQ rows, key/value head).  Two forms:
//   tiles   a CTA takes one pair with all its keys (many rows)
//   shares  the pairs' keys, in units of kUnitKeys, are one long line that the CTAs of the launch cut into equal shares; a CTA
//           walks the segments of its share, writes a pair's rows where it has all of its keys and otherwise leaves the rows'
//           accumulators, maxima and sums in one of its two slots of the workspace (a share can cut at most the pair it
//           begins in and the pair it ends in), which combine_kernel merges in the order of the keys.  The lengths are known
//           to the device only, and sequences of very different lengths still load every SM alike.
#pragma once

#include "ops.h"

namespace dare {

constexpr int kUnitKeys = 128;

struct PackedParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;                    // or nullptr
  const int* q_begin;
  const int* k_begin;
  const int* k_len;              // or nullptr
  int* status;
  float* part_o;                 // shares: [2 * n_ctas slots][BQ][HD]
  float2* part_ml;               // [slots][BQ] (maximum of the scaled scores in log2 units, sum against it)
  long long q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  long long q_rows, k_rows;
  int batch, n_heads, kv_heads, group, causal;
  float scale_log2;              // scale * log2(e)
  int n_ctas;                    // CTAs of the shares launch
  int min_units;                 // a share has at least so many
  int k_head_inner, v_head_inner; // tensor maps: dimension 1 is the head (else the row)
};

#ifdef __CUDACC__
struct SeqGeom {
  int q0, nq, k0, n;             // query rows, key rows
};
// A sequence whose slices are not inside the arrays is flagged and has no rows.
__device__ __forceinline__ SeqGeom seq_geom(const PackedParams& p, int b) {
  SeqGeom s;
  s.q0 = __ldg(p.q_begin + b);
  const long long q1 = __ldg(p.q_begin + b + 1);
  s.k0 = __ldg(p.k_begin + b);
  const long long n = p.k_len ? (long long)__ldg(p.k_len + b) : (long long)__ldg(p.k_begin + b + 1) - s.k0;
  if (s.q0 < 0 || q1 < s.q0 || q1 > p.q_rows || s.k0 < 0 || n < 0 || s.k0 + n > p.k_rows) {
    flag_device_check(p.status);
    s.q0 = s.nq = s.k0 = s.n = 0;
    return s;
  }
  s.nq = (int)(q1 - s.q0);
  s.n = (int)n;
  return s;
}
// keys that query i of the sequence sees
__device__ __forceinline__ int keys_seen(const PackedParams& p, const SeqGeom& s, int i) {
  if (!p.causal) return s.n;
  const long long l = (long long)i + 1 + s.n - s.nq;
  return l < 0 ? 0 : (l > s.n ? s.n : (int)l);
}

struct Place {
  SeqGeom s;
  int tiles, h, tile;            // tiles of the sequence; head and tile of the pair
  int units;                     // of each of its pairs (shares)
  long long first;               // unit of the launch's line where the pair begins
};

__device__ __forceinline__ long long divide(long long a, int b) {       // (64-bit divisions cost ten times as much)
  return a <= 0x7fffffffll ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// The launch's line of pairs, as a warp looks places up in it.  UNITS: a pair counts as its units of keys, else as one.  Lane l holds
// sequence l of the 32 looked at last, so that with at most 32 sequences the lengths are read once.
template <int BQ, bool UNITS>
struct Line {
  const PackedParams& p;
  SeqGeom s;
  int tiles, units, b0;          // of this lane's sequence; first sequence of the 32
  long long base, mine, inc;     // units before the 32; of this lane's sequence; up to and with it

  __device__ __forceinline__ explicit Line(const PackedParams& p_) : p(p_) {
    load(0);
    base = 0;
  }
  __device__ __forceinline__ void load(int first) {
    const int lane = threadIdx.x & 31, b = first + lane;
    b0 = first;
    s = SeqGeom{0, 0, 0, 0};
    if (b < p.batch) s = seq_geom(p, b);
    tiles = (int)(((long long)s.nq * p.group + BQ - 1) / BQ);
    units = UNITS ? max(1, (s.n + kUnitKeys - 1) / kUnitKeys) : 1;
    mine = (long long)tiles * p.kv_heads * units;
    inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
  }
  // next 32 sequences; false: there are none
  __device__ __forceinline__ bool next() {
    if (b0 + 32 >= p.batch) return false;
    base += __shfl_sync(0xffffffffu, inc, 31);
    load(b0 + 32);
    return true;
  }
  __device__ __forceinline__ void rewind() {
    if (b0 != 0) load(0);
    base = 0;
  }
  __device__ __forceinline__ long long total() {
    rewind();
    while (next()) {}
    return base + __shfl_sync(0xffffffffu, inc, 31);
  }
  // Pair that holds unit u; the same for all lanes.  false: u is behind the last one.
  __device__ __forceinline__ bool find(long long u, Place* out) {
    if (u < base) rewind();
    unsigned hit;
    while ((hit = __ballot_sync(0xffffffffu, u < base + inc)) == 0u)
      if (!next()) return false;
    const int src = __ffs((int)hit) - 1;
    const long long begin = base + __shfl_sync(0xffffffffu, inc - mine, src);
    place(src, begin, divide(u - begin, __shfl_sync(0xffffffffu, units, src)), out);
    return true;
  }
  // Pair number `pair` of lane src's sequence, whose units begin at `begin`.
  __device__ __forceinline__ void place(int src, long long begin, long long pair, Place* out) {
    out->s.q0 = __shfl_sync(0xffffffffu, s.q0, src);
    out->s.nq = __shfl_sync(0xffffffffu, s.nq, src);
    out->s.k0 = __shfl_sync(0xffffffffu, s.k0, src);
    out->s.n = __shfl_sync(0xffffffffu, s.n, src);
    out->tiles = __shfl_sync(0xffffffffu, tiles, src);
    out->units = __shfl_sync(0xffffffffu, units, src);
    out->h = (int)divide(pair, out->tiles);                            // head by head
    const int t = (int)(pair - (long long)out->h * out->tiles);
    // shares: first, last, second, last but one ... (causal tiles cost in proportion to their place: any two in a row cost
    // the same); tiles: the longest first
    out->tile = UNITS ? ((t & 1) ? out->tiles - 1 - (t >> 1) : (t >> 1)) : out->tiles - 1 - t;
    out->first = begin + pair * out->units;
  }
};
// units of a share
template <int BQ>
__device__ __forceinline__ long long share_units(const PackedParams& p, long long total) {
  const long long per = divide(total + p.n_ctas - 1, p.n_ctas);
  return per < p.min_units ? p.min_units : per;
}
// Row of a tile -> its place in q, out and lse.
struct RowAt {
  int query, head;               // of the sequence, of all heads
};
__device__ __forceinline__ RowAt row_at(const PackedParams& p, const Place& pl, int row) {
  const int qi = row / p.group;
  return RowAt{qi, pl.h * p.group + row - qi * p.group};
}
#endif

// bf16, heads of 64 or 128, operands TMA can read (attn_packed_tc.cu); tiles: 256 rows a CTA, else shares
cudaError_t launch_packed_tc(const PackedParams& p, int head_dim, bool tiles, cudaStream_t st);
// any type, head width and alignment on the CUDA cores (attn_packed.cu), in shares
cudaError_t launch_packed_simt(const PackedParams& p, int head_dim, bool bf16, cudaStream_t st);
// merges what the shares left (attn_packed.cu); bq: rows of their tiles
cudaError_t launch_packed_combine(const PackedParams& p, int head_dim, int bq, bool bf16, cudaStream_t st);
constexpr int kTcRows = 128, kSimtRows = 32;
constexpr int kSimtCtas = 2 * kSms;             // shares of the CUDA-core kernel: two CTAs an SM

}  // namespace dare
