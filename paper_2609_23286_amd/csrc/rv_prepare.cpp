// rv_prepare.cpp -- librv host side of the projection's norms and rotation: argument checks and
// launches.
#include <algorithm>
#include <cmath>

#include "rv_host.h"

namespace {

using rv::fail;

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

// A tensor of rows: its address, the elements between rows, the heads in a row.
rv_status check_rows(const char* name, const void* p, int64_t stride, int heads, int elem_bytes) {
  if (!p) return fail(RV_ERR_INVALID, "%s is required", name);
  if (stride < (int64_t)heads * rv::kHeadDim)
    return fail(RV_ERR_INVALID, "%s: row stride %lld is less than %d heads", name, (long long)stride, heads);
  if (!aligned(p) || stride * elem_bytes % 16 != 0)
    return fail(RV_ERR_INVALID, "%s: address and row stride must be multiples of 16 bytes", name);
  return RV_OK;
}

rv_status check_prep(const rv_qkv_prep* p, rv_dtype dtype, int n_tokens, const int32_t* pos) {
  if (!p) return fail(RV_ERR_INVALID, "the preparation is NULL");
  if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads > 1024 || p->n_kv_heads > 1024)
    return fail(RV_ERR_INVALID, "head counts must be in [1, 1024] (got %d, %d)", p->n_q_heads, p->n_kv_heads);
  if (p->norm < RV_NORM_NONE || p->norm > RV_NORM_LAYER) return fail(RV_ERR_INVALID, "unknown norm %d", p->norm);
  if (p->n_axes < 0 || p->n_axes > 2) return fail(RV_ERR_INVALID, "n_axes must be 0, 1 or 2 (got %d)", p->n_axes);
  if (p->norm != RV_NORM_NONE && !(p->eps >= 0.f && std::isfinite(p->eps)))
    return fail(RV_ERR_INVALID, "eps must be finite and >= 0");
  if (p->n_axes > 0 && !(p->base >= 1.0 && std::isfinite(p->base)))
    return fail(RV_ERR_INVALID, "the frequency base must be finite and >= 1");
  const float* const vecs[4] = {p->q_weight, p->q_bias, p->k_weight, p->k_bias};
  for (const float* v : vecs) {
    if (v && p->norm == RV_NORM_NONE) return fail(RV_ERR_INVALID, "weights and biases belong to a norm");
    if (!aligned(v)) return fail(RV_ERR_INVALID, "weights and biases must be 16-byte aligned");
  }
  if (dtype != RV_BF16 && dtype != RV_F32) return fail(RV_ERR_INVALID, "unknown dtype %d", (int)dtype);
  if (n_tokens < 0) return fail(RV_ERR_INVALID, "n_tokens must be >= 0 (got %d)", n_tokens);
  if (n_tokens > 0 && p->n_axes > 0 && !pos) return fail(RV_ERR_INVALID, "pos is required with n_axes %d", p->n_axes);
  return RV_OK;
}

rv::PrepArgs base_args(const rv_qkv_prep& p, int n_tokens, const int32_t* pos) {
  rv::PrepArgs a{};
  a.pos = pos;
  a.qw = p.q_weight;
  a.qb = p.q_bias;
  a.kw = p.k_weight;
  a.kb = p.k_bias;
  a.n_tokens = n_tokens;
  a.n_q_heads = p.n_q_heads;
  a.n_kv_heads = p.n_kv_heads;
  a.norm = p.norm;
  a.eps = p.eps;
  if (p.n_axes > 0) rv::rotation_turns(p.base, rv::kMaxFreqs / p.n_axes, a.freq);
  return a;
}

// As many tokens a wave as fill its rows of heads: more rows in a wave were slower than more waves
// (8328 tokens of 16 heads: 27 us at three tokens a wave, 20 at one).
void plan_waves(rv::PrepArgs* a, int max_blocks) {
  const int heads = std::max(a->n_q_heads, a->n_kv_heads);
  a->tokens_per_wave = std::min(rv::kPrepMaxTokens, std::max(1, rv::kPrepRows / heads));
  const int64_t blocks = rv::ceil_div64(a->n_tokens, (int64_t)a->tokens_per_wave * (rv::kPrepThreads / 64));
  a->blocks = (int)std::min<int64_t>(blocks, max_blocks);
}

rv_status prepare(const rv_qkv_prep* p, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                  int64_t v_stride, rv_dtype dtype, int n_tokens, const int32_t* pos, void* Q, void* K, void* V,
                  int64_t kv_row, int64_t kv_head, hipStream_t s) {
  rv_status st;
  const int size = dtype == RV_F32 ? 4 : 2;
  if ((st = check_rows("q", q, q_stride, p->n_q_heads, size)) != RV_OK) return st;
  if ((st = check_rows("k", k, k_stride, p->n_kv_heads, size)) != RV_OK) return st;
  if (!v != !V) return fail(RV_ERR_INVALID, "v and V must both be given or both be NULL");
  if (v && (st = check_rows("v", v, v_stride, p->n_kv_heads, size)) != RV_OK) return st;
  if (!Q || !K) return fail(RV_ERR_INVALID, "Q and K are required");
  if (!aligned(Q) || !aligned(K) || !aligned(V)) return fail(RV_ERR_INVALID, "Q, K and V must be 16-byte aligned");
  rv::DeviceContext ctx;
  if ((st = rv::device_context(&ctx)) != RV_OK) return st;
  rv::PrepArgs a = base_args(*p, n_tokens, pos);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.Q = (uint16_t*)Q;
  a.K = (uint16_t*)K;
  a.V = (uint16_t*)V;
  a.kv_row = kv_row;
  a.kv_head = kv_head;
  plan_waves(&a, INT32_MAX);
  if (a.blocks > rv::kMaxGridBlocks) return fail(RV_ERR_INVALID, "too many tokens for one call");
  RV_HIP(rv::launch_prepare(a, dtype == RV_F32, p->n_axes, false, s), "prepare launch");
  return RV_OK;
}

}  // namespace

extern "C" {

rv_status rv_prepare_qkv(const rv_qkv_prep* p, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, rv_dtype dtype, int n_tokens, const int32_t* pos, void* Q,
                         void* K, void* V, void* stream) {
  rv_status st = check_prep(p, dtype, n_tokens, pos);
  if (st != RV_OK || n_tokens == 0) return st;
  return prepare(p, q, q_stride, k, k_stride, v, v_stride, dtype, n_tokens, pos, Q, K, V,
                 (int64_t)p->n_kv_heads * rv::kHeadDim, rv::kHeadDim, (hipStream_t)stream);
}

rv_status rv_mem_stage_qkv(rv_mem m, const rv_qkv_prep* p, const void* q, int64_t q_stride, const void* k,
                           int64_t k_stride, const void* v, int64_t v_stride, rv_dtype dtype, int n_tokens,
                           const int32_t* pos, void* Q, void* stream) {
  if (!m) return fail(RV_ERR_INVALID, "memory is NULL");
  rv_status st = check_prep(p, dtype, n_tokens, pos);
  if (st != RV_OK) return st;
  if (p->n_kv_heads != m->n_heads)
    return fail(RV_ERR_INVALID, "%d kv heads for a memory of %d", p->n_kv_heads, m->n_heads);
  if (!q || !k || !v || !Q) return fail(RV_ERR_INVALID, "q, k, v and Q are required");
  const int size = dtype == RV_F32 ? 4 : 2;
  if ((st = check_rows("q", q, q_stride, p->n_q_heads, size)) != RV_OK) return st;
  if ((st = check_rows("k", k, k_stride, p->n_kv_heads, size)) != RV_OK) return st;
  if ((st = check_rows("v", v, v_stride, p->n_kv_heads, size)) != RV_OK) return st;
  if (!aligned(Q)) return fail(RV_ERR_INVALID, "Q must be 16-byte aligned");
  void *K, *V;
  int64_t stride;
  if ((st = rv_mem_stage(m, n_tokens, &K, &V, &stride, stream)) != RV_OK) return st;
  return prepare(p, q, q_stride, k, k_stride, v, v_stride, dtype, n_tokens, pos, Q, K, V, rv::kHeadDim,
                 stride * rv::kHeadDim, (hipStream_t)stream);
}

rv_status rv_prepare_qkv_bwd(const rv_qkv_prep* p, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                             rv_dtype dtype, int n_tokens, const int32_t* pos, const void* dQ, const void* dK,
                             const void* dV, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, void* dv,
                             int64_t dv_stride, float* dq_weight, float* dq_bias, float* dk_weight, float* dk_bias,
                             void* stream) {
  rv_status st = check_prep(p, dtype, n_tokens, pos);
  if (st != RV_OK) return st;
  const bool sums = dq_weight || dq_bias || dk_weight || dk_bias;
  if (sums && p->norm == RV_NORM_NONE) return fail(RV_ERR_INVALID, "weights and biases belong to a norm");
  if (n_tokens > 0) {
    const int size = dtype == RV_F32 ? 4 : 2;
    if ((st = check_rows("q", q, q_stride, p->n_q_heads, size)) != RV_OK) return st;
    if ((st = check_rows("k", k, k_stride, p->n_kv_heads, size)) != RV_OK) return st;
    if ((st = check_rows("dq", dq, dq_stride, p->n_q_heads, size)) != RV_OK) return st;
    if ((st = check_rows("dk", dk, dk_stride, p->n_kv_heads, size)) != RV_OK) return st;
    if (!dV != !dv) return fail(RV_ERR_INVALID, "dV and dv must both be given or both be NULL");
    if (dv && (st = check_rows("dv", dv, dv_stride, p->n_kv_heads, size)) != RV_OK) return st;
    if (!dQ || !dK) return fail(RV_ERR_INVALID, "dQ and dK are required");
    if (!aligned(dQ) || !aligned(dK) || !aligned(dV))
      return fail(RV_ERR_INVALID, "dQ, dK and dV must be 16-byte aligned");
  } else if (!sums) {
    return RV_OK;
  }
  rv::DeviceContext ctx;
  if ((st = rv::device_context(&ctx)) != RV_OK) return st;
  rv::PrepArgs a = base_args(*p, n_tokens, pos);
  a.q = q;
  a.k = k;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.dQ = (const uint16_t*)dQ;
  a.dK = (const uint16_t*)dK;
  a.dV = (const uint16_t*)dV;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dq_stride = dq_stride;
  a.dk_stride = dk_stride;
  a.dv_stride = dv_stride;
  a.dqw = dq_weight;
  a.dqb = dq_bias;
  a.dkw = dk_weight;
  a.dkb = dk_bias;
  // a workgroup's sums are 256 floats; the workspace holds far more than two workgroups a CU need
  const int64_t room = (int64_t)(ctx.part_floats / (4 * rv::kHeadDim));
  plan_waves(&a, (int)std::min<int64_t>(2 * ctx.n_cus, room));
  a.part = sums ? ctx.part : nullptr;
  RV_HIP(rv::launch_prepare(a, dtype == RV_F32, p->n_axes, true, (hipStream_t)stream), "prepare launch");
  return RV_OK;
}

}  // extern "C"
