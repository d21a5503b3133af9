// C ABI of cross attention and of attention with a learned relative position
// bias: argument validation on the host, then asynchronous launches on the
// caller's stream.  No device memory is allocated here.
#include <math.h>
#include <string.h>

#pragma GCC visibility push(default)
#include "adaspa.h"
#pragma GCC visibility pop
#include "cross.hpp"

using namespace adaspa;

namespace {

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Strides of a [B, H, L, D] view: rows 16-byte aligned, offsets of a tile of
// rows within 31 bits (whole sequences may be longer: kernels address tiles
// from 64-bit bases).
adaspa_status check_strides(const int64_t* s) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0) return ADASPA_ERR_INVALID_ARG;
  return s[2] < ((int64_t)1 << 23) ? ADASPA_OK : ADASPA_ERR_UNSUPPORTED;
}

// An output's rows must not overlap (an expanded tensor's would).
bool overlaps(const int64_t* s, int B, int H, int L, int D) {
  if (B == 0 || L == 0) return false;
  return (B > 1 && s[0] < D) || (H > 1 && s[1] < D) || (L > 1 && s[2] < D);
}

adaspa_status check_cross(const adaspa_cross_problem* p) {
  if (!p) return ADASPA_ERR_INVALID_ARG;
  if (p->batch < 0 || p->heads < 1 || p->kv_heads < 1 || p->q_len < 0 || p->k_len < 0) return ADASPA_ERR_INVALID_ARG;
  if (p->heads % p->kv_heads != 0) return ADASPA_ERR_INVALID_ARG;
  if (!isfinite(p->softmax_scale)) return ADASPA_ERR_INVALID_ARG;
  if (p->dtype != ADASPA_BF16 && p->dtype != ADASPA_FP16) return ADASPA_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return ADASPA_ERR_UNSUPPORTED;
  if ((int64_t)p->batch * p->heads >= 65536) return ADASPA_ERR_UNSUPPORTED;
  if (p->q_len >= (1 << 28) || p->k_len >= (1 << 28)) return ADASPA_ERR_UNSUPPORTED;
  // Row and workgroup numbers are 32-bit.
  if ((int64_t)p->batch * p->heads * p->q_len >= ((int64_t)1 << 31)) return ADASPA_ERR_UNSUPPORTED;
  if ((int64_t)p->batch * p->kv_heads * p->k_len >= ((int64_t)1 << 31)) return ADASPA_ERR_UNSUPPORTED;
  const int64_t* in[] = {p->q_stride, p->k_stride, p->v_stride, p->out_stride};
  for (const int64_t* s : in) {
    const adaspa_status st = check_strides(s);
    if (st != ADASPA_OK) return st;
  }
  if (overlaps(p->out_stride, p->batch, p->heads, p->q_len, p->head_dim)) return ADASPA_ERR_INVALID_ARG;
  if (p->key_mask_stride < 0) return ADASPA_ERR_INVALID_ARG;
  return ADASPA_OK;
}

adaspa_status check_grads(const adaspa_cross_problem* p) {
  const int64_t* s[] = {p->dout_stride, p->dq_stride, p->dk_stride, p->dv_stride};
  for (const int64_t* x : s) {
    const adaspa_status st = check_strides(x);
    if (st != ADASPA_OK) return st;
  }
  if (overlaps(p->dq_stride, p->batch, p->heads, p->q_len, p->head_dim) ||
      overlaps(p->dk_stride, p->batch, p->kv_heads, p->k_len, p->head_dim) ||
      overlaps(p->dv_stride, p->batch, p->kv_heads, p->k_len, p->head_dim))
    return ADASPA_ERR_INVALID_ARG;
  return ADASPA_OK;
}

adaspa_status check_bias(const adaspa_rel_bias* r) {
  if (!r) return ADASPA_ERR_INVALID_ARG;
  if (r->num_buckets < 1 || (r->bidirectional && r->num_buckets % 2 != 0) || !r->bucket_start)
    return ADASPA_ERR_INVALID_ARG;
  const int side = r->bidirectional ? r->num_buckets / 2 : r->num_buckets;
  if (side > kMaxBucketSide) return ADASPA_ERR_UNSUPPORTED;
  if (r->bucket_start[0] != 0) return ADASPA_ERR_INVALID_ARG;
  for (int i = 1; i < side; ++i)
    if (r->bucket_start[i] < r->bucket_start[i - 1]) return ADASPA_ERR_INVALID_ARG;
  if (r->bucket_start[side - 1] > kMaxFar) return ADASPA_ERR_UNSUPPORTED;
  if (r->q_offset <= -(1 << 28) || r->q_offset >= (1 << 28)) return ADASPA_ERR_INVALID_ARG;
  if (r->table_fp32 != 0 && r->table_fp32 != 1) return ADASPA_ERR_UNSUPPORTED;
  return ADASPA_OK;
}

Strides strides(const int64_t* s) { return Strides{s[0], s[1], s[2]}; }

CrossParams params(const adaspa_cross_problem* p, const adaspa_rel_bias* r) {
  CrossParams c;
  memset(&c, 0, sizeof c);
  c.sq = strides(p->q_stride);
  c.sk = strides(p->k_stride);
  c.sv = strides(p->v_stride);
  c.so = strides(p->out_stride);
  c.sdo = strides(p->dout_stride);
  c.sdq = strides(p->dq_stride);
  c.sdk = strides(p->dk_stride);
  c.sdv = strides(p->dv_stride);
  c.B = p->batch;
  c.H = p->heads;
  c.Hk = p->kv_heads;
  c.G = p->heads / p->kv_heads;
  c.Lq = p->q_len;
  c.Lk = p->k_len;
  c.scale = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  c.sl2 = c.scale * 1.4426950408889634f;
  c.mask_stride = p->key_mask_stride;
  if (r) {
    c.rb.table_f32 = r->table_fp32;
    c.rb.both = r->bidirectional != 0;
    c.rb.side = c.rb.both ? r->num_buckets / 2 : r->num_buckets;
    // At least 1: the kernels take every distance from far on as one bucket on either
    // side, and distance 0, the key at the query's own place, belongs to neither side
    // alone (with one bucket a direction its value is the first direction's, and an
    // order mask leaves it visible).
    c.rb.far = r->bucket_start[c.rb.side - 1] > 1 ? r->bucket_start[c.rb.side - 1] : 1;
    c.rb.causal = r->causal != 0;
    c.rb.at_end = r->queries_at_end != 0;
    c.rb.q_offset = r->q_offset;
    for (int i = 0; i < c.rb.side; ++i) c.rb.start[i] = (uint16_t)r->bucket_start[i];
  }
  return c;
}

// Pointers that a call dereferences only where the tensor has elements.
bool bad(const void* p, bool used, unsigned align) { return (used && !p) || !aligned(p, align); }

adaspa_status forward(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias, bool with_bias,
                      const void* q, const void* k, const void* v, const void* table, const int32_t* key_lens,
                      const uint8_t* key_mask, void* out, float* lse, void* workspace, size_t workspace_bytes,
                      void* stream) {
  adaspa_status st = check_cross(prob);
  if (st == ADASPA_OK && with_bias) st = check_bias(bias);
  if (st != ADASPA_OK) return st;
  const bool rows = prob->batch > 0 && prob->q_len > 0, keys = prob->batch > 0 && prob->k_len > 0;
  if (bad(q, rows, 16) || bad(out, rows, 16) || bad(k, keys, 16) || bad(v, keys, 16) || bad(lse, false, 4) ||
      bad(key_lens, false, 4))
    return ADASPA_ERR_INVALID_ARG;
  if (with_bias && bad(table, true, bias->table_fp32 ? 4 : 2)) return ADASPA_ERR_INVALID_ARG;
  CrossParams c = params(prob, bias);
  c.q = (const u16*)q;
  c.k = (const u16*)k;
  c.v = (const u16*)v;
  c.out = (u16*)out;
  c.lse = lse;
  c.rb.table = table;
  c.key_lens = key_lens;
  c.key_mask = key_mask;
  const CrossPlan plan = plan_fwd(c, prob->head_dim, with_bias);
  if (plan.bytes > 0 && (!workspace || workspace_bytes < (size_t)plan.bytes || !aligned(workspace, 256)))
    return ADASPA_ERR_WORKSPACE;
  if (!rows) return ADASPA_OK;
  c.part_o = (float*)((char*)workspace + plan.part_o);
  c.part_ml = (float*)((char*)workspace + plan.part_ml);
  return launch_cross_fwd(c, prob->head_dim, prob->dtype == ADASPA_FP16, with_bias, plan, (hipStream_t)stream) ==
                 hipSuccess
             ? ADASPA_OK
             : ADASPA_ERR_HIP;
}

adaspa_status backward(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias, bool with_bias,
                       const void* dout, const void* q, const void* k, const void* v, const void* table,
                       const int32_t* key_lens, const uint8_t* key_mask, const void* out, const float* lse, void* dq,
                       void* dk, void* dv, void* dtable, void* workspace, size_t workspace_bytes, void* stream) {
  adaspa_status st = check_cross(prob);
  if (st == ADASPA_OK) st = check_grads(prob);
  if (st == ADASPA_OK && with_bias) st = check_bias(bias);
  if (st != ADASPA_OK) return st;
  const bool rows = prob->batch > 0 && prob->q_len > 0, keys = prob->batch > 0 && prob->k_len > 0;
  if (bad(q, rows, 16) || bad(out, rows, 16) || bad(dout, rows, 16) || bad(dq, rows, 16) || bad(lse, rows, 4) ||
      bad(k, keys, 16) || bad(v, keys, 16) || bad(dk, keys, 16) || bad(dv, keys, 16) || bad(key_lens, false, 4))
    return ADASPA_ERR_INVALID_ARG;
  const unsigned ta = with_bias && bias->table_fp32 ? 4 : 2;
  if (with_bias && (bad(table, true, ta) || bad(dtable, true, ta))) return ADASPA_ERR_INVALID_ARG;
  CrossParams c = params(prob, bias);
  c.q = (const u16*)q;
  c.k = (const u16*)k;
  c.v = (const u16*)v;
  c.dout = (const u16*)dout;
  c.out = (u16*)out;
  c.lse = (float*)lse;
  c.dq = (u16*)dq;
  c.dk = (u16*)dk;
  c.dv = (u16*)dv;
  c.rb.table = table;
  c.rb.dtable = dtable;
  c.key_lens = key_lens;
  c.key_mask = key_mask;
  const CrossPlan plan = plan_bwd(c, prob->head_dim, with_bias);
  if (plan.bytes > 0 && (!workspace || workspace_bytes < (size_t)plan.bytes || !aligned(workspace, 256)))
    return ADASPA_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  c.row_ld = (float2*)(ws + plan.row_ld);
  c.part_o = (float*)(ws + plan.part_o);
  c.part_d = (float*)(ws + plan.part_d);
  c.part_kv = (float*)(ws + plan.part_kv);
  c.part_t = (float*)(ws + plan.part_t);
  return launch_cross_bwd(c, prob->head_dim, prob->dtype == ADASPA_FP16, with_bias, plan, (hipStream_t)stream) ==
                 hipSuccess
             ? ADASPA_OK
             : ADASPA_ERR_HIP;
}

// Sizes are multiples of 256; kNoWorkspace for a valid call that needs none,
// since 0 means invalid.
constexpr size_t kNoWorkspace = 16;
size_t bytes_of(int64_t n) { return n == 0 ? kNoWorkspace : (size_t)n; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t adaspa_cross_attn_workspace(const adaspa_cross_problem* prob) {
  if (check_cross(prob) != ADASPA_OK) return 0;
  return bytes_of(plan_fwd(params(prob, nullptr), prob->head_dim, false).bytes);
}

adaspa_status adaspa_cross_attn(const adaspa_cross_problem* prob, const void* q, const void* k, const void* v,
                                const int32_t* key_lens, const uint8_t* key_mask, void* out, float* lse,
                                void* workspace, size_t workspace_bytes, void* stream) {
  return forward(prob, nullptr, false, q, k, v, nullptr, key_lens, key_mask, out, lse, workspace, workspace_bytes,
                 stream);
}

size_t adaspa_cross_attn_bwd_workspace(const adaspa_cross_problem* prob) {
  if (check_cross(prob) != ADASPA_OK || check_grads(prob) != ADASPA_OK) return 0;
  return bytes_of(plan_bwd(params(prob, nullptr), prob->head_dim, false).bytes);
}

adaspa_status adaspa_cross_attn_bwd(const adaspa_cross_problem* prob, const void* dout, const void* q, const void* k,
                                    const void* v, const int32_t* key_lens, const uint8_t* key_mask, const void* out,
                                    const float* lse, void* dq, void* dk, void* dv, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  return backward(prob, nullptr, false, dout, q, k, v, nullptr, key_lens, key_mask, out, lse, dq, dk, dv, nullptr,
                  workspace, workspace_bytes, stream);
}

size_t adaspa_rel_bias_attn_workspace(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias) {
  if (check_cross(prob) != ADASPA_OK || check_bias(bias) != ADASPA_OK) return 0;
  return bytes_of(plan_fwd(params(prob, bias), prob->head_dim, true).bytes);
}

adaspa_status adaspa_rel_bias_attn(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias, const void* q,
                                   const void* k, const void* v, const void* table, const int32_t* key_lens,
                                   const uint8_t* key_mask, void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  return forward(prob, bias, true, q, k, v, table, key_lens, key_mask, out, lse, workspace, workspace_bytes, stream);
}

size_t adaspa_rel_bias_attn_bwd_workspace(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias) {
  if (check_cross(prob) != ADASPA_OK || check_grads(prob) != ADASPA_OK || check_bias(bias) != ADASPA_OK) return 0;
  return bytes_of(plan_bwd(params(prob, bias), prob->head_dim, true).bytes);
}

adaspa_status adaspa_rel_bias_attn_bwd(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias,
                                       const void* dout, const void* q, const void* k, const void* v,
                                       const void* table, const int32_t* key_lens, const uint8_t* key_mask,
                                       const void* out, const float* lse, void* dq, void* dk, void* dv, void* dtable,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  return backward(prob, bias, true, dout, q, k, v, table, key_lens, key_mask, out, lse, dq, dk, dv, dtable, workspace,
                  workspace_bytes, stream);
}

}  // extern "C"
#pragma GCC visibility pop
