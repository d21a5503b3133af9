// C ABI of the key/value cache in 8 bits: argument validation on the host, then
// asynchronous launches on the caller's stream.  No device memory is allocated here.
#include <math.h>
#include <string.h>

#pragma GCC visibility push(default)
#include "adaspa.h"
#pragma GCC visibility pop
#include "cache.hpp"

using namespace adaspa;

namespace {

bool bad(const void* p, bool used, unsigned align) { return (used && !p) || ((uintptr_t)p & (align - 1)) != 0; }

// (batch, head, token) strides of a view of n of each; an output's rows must not overlap.
adaspa_status check_strides(const int64_t* s, const int* n, int D, bool output) {
  output = output && n[0] > 0 && n[1] > 0 && n[2] > 0;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0 || (output && n[i] > 1 && s[i] < D)) return ADASPA_ERR_INVALID_ARG;
  return ADASPA_OK;
}

// What the three calls share; attn: attention (strides of q and out; else those of k and
// v), output: k and v are written.
adaspa_status check_cache(const adaspa_cache_problem* p, const adaspa_cache* c, bool attn, bool output) {
  if (!p) return ADASPA_ERR_INVALID_ARG;
  if (p->batch < 0 || p->heads < 1 || p->kv_heads < 1 || p->len < 0 || p->heads % p->kv_heads != 0)
    return ADASPA_ERR_INVALID_ARG;
  if (!attn && p->heads != p->kv_heads) return ADASPA_ERR_INVALID_ARG;
  if (p->pages < 0 || p->max_pages < 0 || p->table_stride < 0) return ADASPA_ERR_INVALID_ARG;
  if (!isfinite(p->softmax_scale)) return ADASPA_ERR_INVALID_ARG;
  if (p->dtype != ADASPA_BF16 && p->dtype != ADASPA_FP16) return ADASPA_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return ADASPA_ERR_UNSUPPORTED;
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128) return ADASPA_ERR_UNSUPPORTED;
  // Batch and heads are grid dimensions; rows and positions 32-bit numbers.
  if ((int64_t)p->batch * p->heads >= 65536 || p->kv_heads >= 32768) return ADASPA_ERR_UNSUPPORTED;
  if (p->len >= (1 << 28) || (int64_t)p->max_pages * p->page >= (1 << 28)) return ADASPA_ERR_UNSUPPORTED;
  if ((int64_t)p->batch * p->heads * p->len >= ((int64_t)1 << 31)) return ADASPA_ERR_UNSUPPORTED;
  const int nq[] = {p->batch, p->heads, p->len}, nk[] = {p->batch, p->kv_heads, p->len};
  adaspa_status st;
  if (attn) {
    st = check_strides(p->q_stride, nq, p->head_dim, false);
    if (st == ADASPA_OK) st = check_strides(p->out_stride, nq, p->head_dim, true);
  } else {
    st = check_strides(p->k_stride, nk, p->head_dim, output);
    if (st == ADASPA_OK) st = check_strides(p->v_stride, nk, p->head_dim, output);
  }
  if (st != ADASPA_OK) return st;
  if (!c) return ADASPA_OK;
  const bool used = p->pages > 0;
  if (bad(c->k, used, 16) || bad(c->v, used, 16) || bad(c->k_scale, used, 4) || bad(c->v_scale, used, 4) ||
      bad(c->page_table, p->batch > 0 && p->max_pages > 0, 4))
    return ADASPA_ERR_INVALID_ARG;
  return ADASPA_OK;
}

Strides strides(const int64_t* s) { return Strides{s[0], s[1], s[2]}; }

CacheParams params(const adaspa_cache_problem* p, const adaspa_cache* c) {
  CacheParams r;
  memset(&r, 0, sizeof r);
  if (c) {
    r.c.k = (uint8_t*)c->k;
    r.c.v = (uint8_t*)c->v;
    r.c.k_scale = c->k_scale;
    r.c.v_scale = c->v_scale;
    r.c.table = c->page_table;
  }
  r.c.table_stride = p->table_stride;
  r.c.pages = p->pages;
  r.c.page = p->page;
  r.c.max_pages = p->max_pages;
  r.B = p->batch;
  r.H = p->heads;
  r.Hk = p->kv_heads;
  r.G = p->heads / p->kv_heads;
  r.D = p->head_dim;
  r.L = p->len;
  r.sq = strides(p->q_stride);
  r.sk = strides(p->k_stride);
  r.sv = strides(p->v_stride);
  r.so = strides(p->out_stride);
  r.causal = p->causal != 0;
  r.sl2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->head_dim)) * 1.4426950408889634f;
  return r;
}

adaspa_status done(hipError_t e) { return e == hipSuccess ? ADASPA_OK : ADASPA_ERR_HIP; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

adaspa_status adaspa_cache_write(const adaspa_cache_problem* prob, const adaspa_cache* cache, const void* k,
                                 const void* v, const int32_t* lens, const int32_t* new_lens, void* stream) {
  if (!cache) return ADASPA_ERR_INVALID_ARG;
  const adaspa_status st = check_cache(prob, cache, false, false);
  if (st != ADASPA_OK) return st;
  const bool rows = prob->batch > 0 && prob->len > 0;
  if (bad(k, rows, 16) || bad(v, rows, 16) || bad(lens, rows, 4) || bad(new_lens, false, 4)) return ADASPA_ERR_INVALID_ARG;
  CacheParams p = params(prob, cache);
  p.k = (const u16*)k;
  p.v = (const u16*)v;
  p.lens = lens;
  p.new_lens = new_lens;
  return done(launch_cache_write(p, prob->dtype == ADASPA_FP16, (hipStream_t)stream));
}

adaspa_status adaspa_cache_read(const adaspa_cache_problem* prob, const adaspa_cache* cache, const int32_t* lens,
                                const int32_t* starts, void* k, void* v, void* stream) {
  if (!cache) return ADASPA_ERR_INVALID_ARG;
  const adaspa_status st = check_cache(prob, cache, false, true);
  if (st != ADASPA_OK) return st;
  const bool rows = prob->batch > 0 && prob->len > 0;
  if (bad(k, rows, 16) || bad(v, rows, 16) || bad(lens, rows, 4) || bad(starts, false, 4)) return ADASPA_ERR_INVALID_ARG;
  if (rows && k == v) return ADASPA_ERR_INVALID_ARG;
  CacheParams p = params(prob, cache);
  p.k_out = (u16*)k;
  p.v_out = (u16*)v;
  p.lens = lens;
  p.starts = starts;
  return done(launch_cache_read(p, prob->dtype == ADASPA_FP16, (hipStream_t)stream));
}

size_t adaspa_cache_attn_workspace(const adaspa_cache_problem* prob) {
  if (check_cache(prob, nullptr, true, true) != ADASPA_OK) return 0;
  const int64_t n = plan_cache_attn(params(prob, nullptr), prob->dtype == ADASPA_FP16).bytes;
  return n == 0 ? 16 : (size_t)n;
}

adaspa_status adaspa_cache_attn(const adaspa_cache_problem* prob, const adaspa_cache* cache, const void* q,
                                const int32_t* lens, const int32_t* q_lens, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (!cache) return ADASPA_ERR_INVALID_ARG;
  const adaspa_status st = check_cache(prob, cache, true, true);
  if (st != ADASPA_OK) return st;
  const bool rows = prob->batch > 0 && prob->len > 0;
  if (bad(q, rows, 16) || bad(out, rows, 16) || bad(lens, rows, 4) || bad(q_lens, false, 4) || bad(lse, false, 4))
    return ADASPA_ERR_INVALID_ARG;
  CacheParams p = params(prob, cache);
  const CachePlan plan = plan_cache_attn(p, prob->dtype == ADASPA_FP16);
  if (plan.bytes > 0 && (!workspace || workspace_bytes < (size_t)plan.bytes || ((uintptr_t)workspace & 255) != 0))
    return ADASPA_ERR_WORKSPACE;
  if (!rows) return ADASPA_OK;
  p.q = (const u16*)q;
  p.out = (u16*)out;
  p.lse = lse;
  p.lens = lens;
  p.new_lens = q_lens;
  p.part_o = (float*)workspace;
  p.part_ml = (float*)((char*)workspace + plan.part_ml);
  p.before = (int64_t*)((char*)workspace + plan.before);
  return done(launch_cache_attn(p, prob->dtype == ADASPA_FP16, plan, (hipStream_t)stream));
}

}  // extern "C"
#pragma GCC visibility pop
