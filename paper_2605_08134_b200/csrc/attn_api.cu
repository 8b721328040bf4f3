// C entries of the packed attention: argument checks and the choice of a kernel.
#include <math.h>

#include "attn_packed.h"

using namespace dare;

namespace {

constexpr int kMaxHeads = 1024;
constexpr float kLog2e = 1.4426950408889634f;
// Cost of a pair besides its keys, in units of 128 keys.  Sixteen tokens over 16k keys / a block of 160 over 2500, us: with 2 110.8 / 24.4,
// 3 110.8 / 24.7, 5 111.4 / 25.9, 7 112.5 / 26.6; 4000 causal tokens of 4 and 1 heads: 77 with 0, 44 with 5.  CUDA cores, three causal
// prompts / blocks of 62 over 910: 0 30.5 / 53.3, 1 32.2 / 50.0, 2 32.9 / 54.8.
constexpr unsigned kPairCostTc = 3, kPairCostSimt = 1;

bool valid_config(const dare_attention_config_t* c) {
  if (!c || c->struct_size != sizeof(dare_attention_config_t)) return false;
  if (c->dtype != DARE_F32 && c->dtype != DARE_BF16) return false;
  if (c->causal != 0 && c->causal != 1) return false;
  if (!(c->scale > 0.f) || !isfinite(c->scale * kLog2e)) return false;
  return true;
}
bool shape_ok(const dare_attention_config_t* c) {
  if (c->batch <= 0 || c->batch > 65536 || c->n_kv_heads <= 0 || c->n_heads <= 0 || c->n_heads > kMaxHeads ||
      c->n_heads % c->n_kv_heads != 0)
    return false;
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
  if (c->q_rows < 0 || c->q_rows > (int64_t)1 << 24 || c->k_rows < 0 || c->k_rows > (int64_t)1 << 30) return false;
  if (c->q_rows * c->n_heads >= (int64_t)1 << 31) return false;           // (grids and row numbers stay within 31 bits)
  const int64_t s[8] = {c->q_token, c->q_head, c->k_token, c->k_head, c->v_token, c->v_head, c->o_token, c->o_head};
  for (int64_t v : s)
    if (!stride_ok(v)) return false;
  return places_apart(c->q_rows, c->o_token, c->n_heads, c->o_head, c->head_dim);
}
bool tc_types(const dare_attention_config_t* c) { return c->dtype == DARE_BF16 && (c->head_dim == 64 || c->head_dim == 128); }
size_t part_rows(bool tc) { return (size_t)2 * (tc ? kSms * kTcRows : kSimtCtas * kSimtRows); }      // two slots a CTA

}  // namespace

extern "C" {

size_t dare_attention_workspace_bytes(const dare_attention_config_t* c) {
  if (!valid_config(c) || !shape_ok(c)) return 0;
  return part_rows(tc_types(c)) * (c->head_dim * sizeof(float) + sizeof(float2));
}

dare_status_t dare_attention(const dare_attention_config_t* c, const void* q, const void* k, const void* v, const int32_t* q_begin,
                             const int32_t* k_begin, const int32_t* k_len, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, int32_t* status, void* cuda_stream) {
  if (!valid_config(c)) return DARE_ERR_INVALID_ARG;
  if (!shape_ok(c)) return DARE_ERR_SHAPE;
  if (c->q_rows == 0) return DARE_OK;
  if (!q || !q_begin || !k_begin || !out || !workspace || (c->k_rows > 0 && (!k || !v))) return DARE_ERR_INVALID_ARG;
  auto low = [](const void* p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; };
  const uintptr_t elem = c->dtype == DARE_BF16 ? 1u : 3u;
  if (low(q, elem) || low(k, elem) || low(v, elem) || low(out, elem) || low(q_begin, 3u) || low(k_begin, 3u) || low(k_len, 3u) ||
      low(lse, 3u) || low(workspace, 15u) || low(status, 3u))
    return DARE_ERR_ALIGN;
  if (workspace_bytes < dare_attention_workspace_bytes(c)) return DARE_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)cuda_stream;

  PackedParams p = {};
  p.q = q; p.k = k; p.v = v; p.o = out; p.lse = lse; p.q_begin = q_begin; p.k_begin = k_begin; p.k_len = k_len; p.status = status;
  p.q_token = c->q_token; p.q_head = c->q_head; p.k_token = c->k_token; p.k_head = c->k_head;
  p.v_token = c->v_token; p.v_head = c->v_head; p.o_token = c->o_token; p.o_head = c->o_head;
  p.q_rows = c->q_rows; p.k_rows = c->k_rows;
  p.batch = c->batch; p.n_heads = c->n_heads; p.kv_heads = c->n_kv_heads; p.group = c->n_heads / c->n_kv_heads; p.causal = c->causal;
  p.scale_log2 = c->scale * kLog2e;

  // The tensor-core kernel reads k and v through TMA (16-byte aligned rows and heads that do not overlap), q and out by 16
  // bytes.
  auto eights = [](int64_t a) { return a % 8 == 0; };
  auto tma = [&](int64_t token, int64_t head) {
    return (c->k_rows <= 1 || (token >= c->head_dim && eights(token))) && (c->n_kv_heads <= 1 || (head >= c->head_dim && eights(head)));
  };
  const bool tc = tc_types(c) && c->k_rows > 0 && !low(q, 15u) && !low(k, 15u) && !low(v, 15u) && !low(out, 15u) && eights(c->q_token) &&
                  eights(c->q_head) && eights(c->o_token) && eights(c->o_head) && tma(c->k_token, c->k_head) && tma(c->v_token, c->v_head);
  const int64_t all = c->q_rows * p.group;
  const int rows = tc ? kTcRows : (all <= (int64_t)kSimtFewRows * c->batch ? kSimtFewRows : kSimtRows);
  p.n_ctas = tc ? kSms : kSimtCtas;
  p.group_magic = ((1u << 24) + p.group - 1) / p.group;
  p.unit_shift = kUnitShift;
  p.pair_cost = tc ? kPairCostTc : kPairCostSimt;
  while ((all / rows + c->batch) * c->n_kv_heads >= ((int64_t)1 << 31) / ((c->k_rows >> p.unit_shift) + 2 + p.pair_cost)) ++p.unit_shift;
  p.part_ml = reinterpret_cast<float2*>(workspace);
  p.part_o = reinterpret_cast<float*>(p.part_ml + part_rows(tc));

  cudaError_t e;
  if (tc) {
    // 256 rows a CTA, or shares?  What each takes, in us, from k_rows / batch keys a sequence (a cache may hold fewer): a CTA of the first
    // takes 2 us a 128 keys (1.2 with rows for one stream only), the launch 6; the shares take 1.1 us a 128 keys and tile of 128 rows
    // (0.75 with few rows) over all SMs, five such for a tile itself, and 13 with the merge.  Heads of 64 have two products a weight, which
    // the shares hide better: 1 us (0.7), three for a tile, 11 with the merge, and only the keys that causality leaves count.
    // Tiles / shares in us, heads of 128, 32 query and 8 key heads: a prompt of 300 tokens 12 / 17, 4000 137 / 180, four of up to 1500
    // 66 / 96; 4 and 1 heads: 4000 tokens 56 / 38; two blocks of 256 tokens over 8192 keys 108 / 78, four of 512 225 / 284, one token over
    // 4000 keys 49 / 16, four over 200 8.3 / 11.6.  Heads of 64: a prompt of 300 tokens 12.2 / 13.0, 4000 161 / 149, four of up to 1500
    // 68 / 75; 8 and 8 heads: 4000 tokens 68 / 48, four of up to 700 18 / 16; 4 and 1 heads: four of up to 4000 69 / 52.  Of 108 such
    // shapes the rule takes the slower form, by more than 5 %, in nine, by 34 % at most.  Each CTA of the first looks its
    // pair up among the sequences' lengths, the shares twice a launch: 256 prompts of up to 200 tokens, 8 and 8 heads, 163 / 161 us,
    // 1024 1048 / 607.
    const float keys = (float)(c->k_rows / c->batch) / 128.f + 1.f;
    const int64_t rows_each = all / c->batch;
    const float ctas = (float)((all / 256 > c->batch ? all / 256 : c->batch) * c->n_kv_heads);
    const float pairs = (float)((all / 128 > c->batch ? all / 128 : c->batch) * c->n_kv_heads);
    const float look_up = 0.012f * (float)c->batch;
    const float tiles_us = (6.f + look_up + keys * (rows_each > 128 ? 2.f : 1.2f)) * fmaxf(1.f, ctas / (float)kSms);
    const float seen = c->causal ? 1.f - 0.5f * fminf(1.f, (float)c->q_rows / (float)c->k_rows) : 1.f;
    const float shares_us = c->head_dim == 64 ? 11.f + pairs * (keys * seen + 3.f) * (rows_each > 64 ? 1.f : 0.7f) / (float)kSms
                                              : 13.f + pairs * (keys + 5.f) * (rows_each > 64 ? 1.1f : 0.75f) / (float)kSms;
    const bool tiles = (rows_each > 128 && ctas >= (float)kSms && c->batch <= 256) || tiles_us <= shares_us;
    e = launch_packed_tc(p, c->head_dim, tiles, st);
    if (e == cudaSuccess && !tiles) e = launch_packed_combine(p, c->head_dim, rows, true, st);
  } else {
    // Few keys a sequence: a pair is a unit, a CTA has a pair, and there is nothing to merge.  Shares / pairs, float32, causal, us: 16 heads of
    // 64, four prompts of up to 100 tokens 15.5 / 13.9, 6 of 113 11.9 / 10.0, one of 60 10.7 / 8.5; 14 heads of 256, 18 tokens 18.5 / 14.5;
    // 12 heads of 128, two of 128 26.9 / 18.0.  With more keys it depends on how many pairs there are and how unequal they are, too:
    // pairs ahead with three prompts of up to 333 (14 heads of 64, 38.0 / 32.0), four of up to 200 (8 heads of 32, 13.7 / 11.0), 16 tokens
    // over up to 200 keys (20.0 / 16.2), behind with one prompt of 700 (8 heads of 128, 69 / 106), two blocks of 62 over 910 (29 / 48).  The
    // rule takes pairs only where they are ahead for sure: of 48 such shapes, causal and not, it has the slower form, by more than 5 %, in
    // twelve, by 58 % at most, all of them shares.  (One sequence may hold all the keys: eight units.)
    const int64_t pairs = (all / rows + c->batch) * c->n_kv_heads;                  // at most
    const bool direct = c->k_rows <= (int64_t)(1 << kUnitShift) * (c->batch < 8 ? c->batch : 8) && pairs <= 8 * kSimtCtas;
    if (direct) {
      while (((int64_t)1 << p.unit_shift) < 2 * c->k_rows) ++p.unit_shift;           // (twice: a causal tile's last row is past the end)
      p.pair_cost = 0;
      p.n_ctas = (int)pairs;
    }
    e = launch_packed_simt(p, c->head_dim, rows, c->dtype == DARE_BF16, st);
    if (e == cudaSuccess && !direct) e = launch_packed_combine(p, c->head_dim, rows, c->dtype == DARE_BF16, st);
  }
  if (e != cudaSuccess) { cudaGetLastError(); return DARE_ERR_CUDA; }
  return DARE_OK;
}

}  // extern "C"
