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

// A unit is 2^kUnitShift keys, more where the line would have 2^31 of them.
constexpr int kUnitShift = 7;

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
  float* part_o;                 // shares: [2 * n_ctas slots][HD / 4][BQ][4]: rows side by side, as the threads that write them are
  float2* part_ml;               // [slots][BQ] (maximum of the scaled scores in log2 units, sum against it)
  long long q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  long long q_rows, k_rows;
  int batch, n_heads, kv_heads, group, causal;
  float scale_log2;              // scale * log2(e)
  int unit_shift;                // log2 of the keys of a unit
  unsigned pair_cost;            // units at the head of a pair that stand for its own cost
  unsigned group_magic;          // ceil(2^24 / group)
  int n_ctas;                    // CTAs of the shares launch
  int k_head_inner, v_head_inner; // tensor maps: dimension 1 is the head (else the row)
};

#ifdef __CUDACC__
struct SeqGeom {
  int q0, nq, k0, n;             // query rows, key rows
};
// A sequence whose slices are not inside the arrays is flagged and has no rows.  PAST_L1: for the merge kernel, which looks lengths up
// before it waits (behind the wait of the kernel in front: what was written before that is in the L2).
template <bool PAST_L1>
__device__ __forceinline__ SeqGeom seq_geom(const PackedParams& p, int b) {
  auto at = [](const int* x) { return PAST_L1 ? __ldcg(x) : *x; };
  SeqGeom s;
  s.q0 = at(p.q_begin + b);
  const long long q1 = at(p.q_begin + b + 1);
  s.k0 = at(p.k_begin + b);
  const long long n = p.k_len ? (long long)at(p.k_len + b) : (long long)at(p.k_begin + b + 1) - s.k0;
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
  unsigned units;                // of its keys (shares)
  unsigned first;                // unit of the launch's line where its keys begin
};

// Units before tile T of a head.  Without a mask every tile has ceil(n / unit).  Causal: the last row of tile t is row (t + 1) BQ - 1 of
// the packed rows, query (that) / G, which sees n - nq more keys than its number plus one; as BQ divides unit * G = band * BQ, its
// units are floor((t + e) / band) + 1 with e = ceil((n - nq) G / BQ) = q0 band + r0, one at least (a tile that sees no key still
// writes its rows; the last tile may count a unit it does not have), and their sum is that of an arithmetic series in steps of
// `band` tiles.
struct UnitCount {
  unsigned per_tile;             // 1 + q0, no mask: units of every tile; and the pair's own cost
  unsigned band;                 // 0: no mask
  int r0;                        // at most band; negative where the first queries see no key
  __device__ __forceinline__ unsigned before(int T) const {
    unsigned units = (unsigned)T * per_tile;
    if (band != 0 && T + r0 > 0) {                                            // + sum of floor(i / band) over i < T + r0
      const unsigned x = (unsigned)(T + r0), q = x / band, r = x - q * band;
      units += band * ((q * (q - 1)) >> 1) + q * r;
    }
    return units;
  }
};

// The launch's line of pairs, as a warp looks places up in it.  UNITS: a pair counts as its units of keys, else as one.  Lane l holds
// sequence l of the 32 looked at last, so that with at most 32 sequences the lengths are read once.  Everything in 32 bits (the host
// sees to it that the line is no longer): this is on the way to a CTA's first key, and fetching the instructions of 64-bit
// divisions through the L2 behind other CTAs' keys took some of them 4 us.
template <int BQ, bool UNITS, bool PAST_L1 = false>
struct Line {
  const PackedParams& p;
  SeqGeom s;
  int tiles, b0;                 // of this lane's sequence; first sequence of the 32
  UnitCount count;
  unsigned base, head, inc;      // units before the 32; of a head of this lane's sequence; up to and with its last head
  // Query slices that do not overlap stay below 2^31 units.  Those that run back and forth may not: sums stop there.
  static constexpr unsigned kFull = 1u << 31;
  static __device__ __forceinline__ unsigned sum(unsigned a, unsigned b) { return a + min(b, kFull - a); }    // (a, b <= kFull)

  __device__ __forceinline__ explicit Line(const PackedParams& p_) : p(p_) {
    load(0);
    base = 0;
  }
  __device__ __forceinline__ void load(int first) {
    const int lane = threadIdx.x & 31, b = first + lane;
    b0 = first;
    s = SeqGeom{0, 0, 0, 0};
    if (b < p.batch) s = seq_geom<PAST_L1>(p, b);
    tiles = (int)(((unsigned)s.nq * (unsigned)p.group + BQ - 1) / BQ);
    head = (unsigned)tiles;
    if (UNITS) {
      const int shift = p.unit_shift, d = s.n - s.nq;
      if (p.causal) {
        count.band = (unsigned)p.group << (shift - kLogBq);
        count.per_tile = p.pair_cost + 1u + (d > 0 ? (unsigned)d >> shift : 0u);
        count.r0 = d > 0 ? (int)(((unsigned)(d & ((1 << shift) - 1)) * (unsigned)p.group + BQ - 1) >> kLogBq)
                         : -(int)(((unsigned)-d * (unsigned)p.group) >> kLogBq);
      } else {
        const unsigned units = ((unsigned)s.n + (1u << shift) - 1) >> shift;
        count.band = 0;
        count.per_tile = p.pair_cost + (units > 1 ? units : 1);
        count.r0 = 0;
      }
      head = count.before(tiles);
    }
    inc = head * (unsigned)p.kv_heads;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc = sum(inc, v);
    }
  }
  // next 32 sequences; false: there are none
  __device__ __forceinline__ bool next() {
    if (b0 + 32 >= p.batch) return false;
    base = sum(base, __shfl_sync(0xffffffffu, inc, 31));
    load(b0 + 32);
    return true;
  }
  __device__ __forceinline__ void rewind() {
    if (b0 != 0) load(0);
    base = 0;
  }
  // 0 too for a line that is longer than its sums can tell, which is flagged: nothing of it is worked on.
  __device__ __forceinline__ unsigned total() {
    rewind();
    while (next()) {}
    const unsigned all = sum(base, __shfl_sync(0xffffffffu, inc, 31));
    if (all < kFull) return all;
    flag_device_check(p.status);
    return 0u;
  }
  // Pair that holds unit u; the same for all lanes.  false: u is behind the last one.
  __device__ __forceinline__ bool find(unsigned u, Place* out) {
    if (u < base) rewind();
    unsigned hit;
    while ((hit = __ballot_sync(0xffffffffu, u < base + inc)) == 0u)
      if (!next()) return false;
    const int src = __ffs((int)hit) - 1;
    out->s.q0 = __shfl_sync(0xffffffffu, s.q0, src);
    out->s.nq = __shfl_sync(0xffffffffu, s.nq, src);
    out->s.k0 = __shfl_sync(0xffffffffu, s.k0, src);
    out->s.n = __shfl_sync(0xffffffffu, s.n, src);
    out->tiles = __shfl_sync(0xffffffffu, tiles, src);
    const unsigned per_head = __shfl_sync(0xffffffffu, head, src);
    const unsigned in_seq = u - base - __shfl_sync(0xffffffffu, inc - head * (unsigned)p.kv_heads, src);
    out->h = (int)(in_seq / per_head);
    const unsigned in_head = in_seq - (unsigned)out->h * per_head;
    if (!UNITS) {
      out->tile = out->tiles - 1 - (int)in_head;                              // the longest first
      out->units = 1;
      out->first = u;
      return true;
    }
    if (out->tiles == 1) {
      out->tile = 0;
      out->units = per_head - p.pair_cost;
      out->first = u - in_head + p.pair_cost;
      return true;
    }
    UnitCount c;
    c.per_tile = __shfl_sync(0xffffffffu, count.per_tile, src);
    c.band = __shfl_sync(0xffffffffu, count.band, src);
    c.r0 = __shfl_sync(0xffffffffu, count.r0, src);
    // last tile with no more than in_head units before it: 32 guesses at a time
    int lo = 0, span = out->tiles;
    const int lane = threadIdx.x & 31;
    while (span > 1) {
      const int step = (span + 31) >> 5, t = lo + lane * step;
      const unsigned ok = __ballot_sync(0xffffffffu, t < lo + span && c.before(t) <= in_head);       // (lane 0 always)
      const int l = 31 - __clz((int)ok);
      span = min(step, span - l * step);
      lo += l * step;
    }
    out->tile = lo;
    const unsigned mine = c.before(lo + (lane & 1));                          // (lanes 0 and 1)
    const unsigned before = __shfl_sync(0xffffffffu, mine, 0);
    out->units = __shfl_sync(0xffffffffu, mine, 1) - before - p.pair_cost;
    out->first = u - (in_head - before) + p.pair_cost;
    return true;
  }
  static constexpr int kLogBq = BQ == 8 ? 3 : (BQ == 32 ? 5 : (BQ == 128 ? 7 : 8));
  static_assert(BQ == 1 << kLogBq, "rows of a tile");
};
// What a share has of a pair, from unit u of the line on: its key units [k0, k1) (none where the share ends before them), and where
// they go: slot < 0: they are all of the pair's, else the slot of the partial result.
struct Part {
  unsigned k0, k1, end;          // end: where the next pair begins, or the share ends
  int slot;
};
__device__ __forceinline__ Part part_of(const Place& pl, unsigned u, unsigned share_begin, unsigned share_end, int cta) {
  Part t;
  const unsigned pair_end = pl.first + pl.units;
  t.end = min(pair_end, share_end);
  t.k0 = u > pl.first ? u - pl.first : 0u;
  t.k1 = t.end > pl.first ? t.end - pl.first : 0u;
  t.slot = t.k0 == 0 && t.k1 == pl.units ? -1 : 2 * cta + (pl.first < share_begin ? 0 : 1);
  return t;
}
// units of a share
__device__ __forceinline__ unsigned share_units(const PackedParams& p, unsigned total) {
  return total <= (unsigned)p.n_ctas ? 1u : (total + (unsigned)p.n_ctas - 1) / (unsigned)p.n_ctas;
}

// Row of a tile -> its place in q, out and lse: row = first query's rows before it + row of the tile.  Tiles begin at query
// row0 / G; the small remainder is divided by a multiplication (x < 2^13, G < 2^11: exact).
struct TileRows {
  int query0, rest;              // row0 / G, row0 % G
};
struct RowAt {
  int query, head;               // of the sequence, of all heads
};
__device__ __forceinline__ TileRows tile_rows(const PackedParams& p, int row0) {
  const int q = (int)((unsigned)row0 / (unsigned)p.group);
  return TileRows{q, row0 - q * p.group};
}
__device__ __forceinline__ RowAt row_at(const PackedParams& p, const TileRows& t, int h, int row) {
  const unsigned x = (unsigned)(t.rest + row);
  const int qi = (int)(((unsigned long long)x * p.group_magic) >> 24);
  return RowAt{t.query0 + qi, h * p.group + (int)x - qi * p.group};
}
#endif

// bf16, heads of 64 or 128, operands TMA can read (attn_packed_tc.cu); tiles: 256 rows a CTA, else shares
cudaError_t launch_packed_tc(const PackedParams& p, int head_dim, bool tiles, cudaStream_t st);
// any type, head width and alignment on the CUDA cores (attn_packed.cu), in shares; bq: kSimtRows or kSimtFewRows rows a tile
cudaError_t launch_packed_simt(const PackedParams& p, int head_dim, int bq, bool bf16, cudaStream_t st);
// merges what the shares left (attn_packed.cu); bq: rows of their tiles
cudaError_t launch_packed_combine(const PackedParams& p, int head_dim, int bq, bool bf16, cudaStream_t st);
constexpr int kTcRows = 128, kSimtRows = 32, kSimtFewRows = 8;
constexpr int kSimtCtas = 2 * kSms;             // shares of the CUDA-core kernel: two CTAs an SM

}  // namespace dare
