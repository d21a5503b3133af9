// C ABI of rotary positions: argument validation on the host, then an
// asynchronous launch on the caller's stream.
#include <math.h>
#include <string.h>

#pragma GCC visibility push(default)
#include "adaspa.h"
#pragma GCC visibility pop
#include "rotary.hpp"

using namespace adaspa;

namespace {

// (batch, head, token) strides of a view of n of each; an output's rows must not overlap.
adaspa_status check_strides(const int64_t* s, const int* n, int D, bool output) {
  output = output && n[0] > 0 && n[1] > 0 && n[2] > 0;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0 || (output && n[i] > 1 && s[i] < D)) return ADASPA_ERR_INVALID_ARG;
  return ADASPA_OK;
}

adaspa_status check_rotary(const adaspa_rotary_problem* p) {
  if (!p) return ADASPA_ERR_INVALID_ARG;
  if (p->batch < 0 || p->heads < 1 || p->kv_heads < 0 || p->len < 0) return ADASPA_ERR_INVALID_ARG;
  if (p->dtype != ADASPA_BF16 && p->dtype != ADASPA_FP16) return ADASPA_ERR_UNSUPPORTED;
  if (p->layout != ADASPA_ROTARY_HALF && p->layout != ADASPA_ROTARY_INTERLEAVED) return ADASPA_ERR_INVALID_ARG;
  if (p->head_dim < 8 || p->head_dim > 2 * kMaxRotaryPairs || p->head_dim % 8 != 0) return ADASPA_ERR_UNSUPPORTED;
  if (p->pairs < 1 || p->pairs > p->head_dim / 2 || !p->freq || !isfinite(p->magnitude)) return ADASPA_ERR_INVALID_ARG;
  if (p->axes < 1 || p->axes > kMaxRotaryAxes) return ADASPA_ERR_INVALID_ARG;
  int64_t sum = 0;
  for (int a = 0; a < p->axes; ++a) {
    if (p->axis_pairs[a] < 0) return ADASPA_ERR_INVALID_ARG;
    sum += p->axis_pairs[a];
  }
  if (sum != p->pairs) return ADASPA_ERR_INVALID_ARG;
  for (int i = 0; i < p->pairs; ++i)
    if (!isfinite(p->freq[i])) return ADASPA_ERR_INVALID_ARG;
  // Work items and workgroups are 32-bit numbers.
  const int64_t tokens = (int64_t)p->batch * p->len, heads = (int64_t)p->heads + p->kv_heads;
  if (heads >= 65536 || tokens >= ((int64_t)1 << 31) / (p->head_dim / 2)) return ADASPA_ERR_UNSUPPORTED;
  if (p->position_stride[0] < 0 || p->position_stride[1] < 0) return ADASPA_ERR_INVALID_ARG;
  const int nq[] = {p->batch, p->heads, p->len}, nk[] = {p->batch, p->kv_heads, p->len};
  adaspa_status st = check_strides(p->q_stride, nq, p->head_dim, false);
  if (st == ADASPA_OK) st = check_strides(p->q_out_stride, nq, p->head_dim, true);
  if (st == ADASPA_OK && p->kv_heads) st = check_strides(p->k_stride, nk, p->head_dim, false);
  if (st == ADASPA_OK && p->kv_heads) st = check_strides(p->k_out_stride, nk, p->head_dim, true);
  return st;
}

Strides strides(const int64_t* s) { return Strides{s[0], s[1], s[2]}; }
bool bad(const void* p, bool used, unsigned align) { return (used && !p) || ((uintptr_t)p & (align - 1)) != 0; }

adaspa_status turn(const adaspa_rotary_problem* p, const void* q, const void* k, const int32_t* positions,
                   int64_t offset, const int32_t* offsets, void* q_out, void* k_out, float way, void* stream) {
  const adaspa_status st = check_rotary(p);
  if (st != ADASPA_OK) return st;
  const bool rows = p->batch > 0 && p->len > 0, keys = rows && p->kv_heads > 0;
  if (bad(q, rows, 16) || bad(q_out, rows, 16) || bad(k, keys, 16) || bad(k_out, keys, 16) || bad(positions, false, 4) ||
      bad(offsets, false, 4))
    return ADASPA_ERR_INVALID_ARG;
  if (p->axes > 1 && rows && !positions) return ADASPA_ERR_INVALID_ARG;
  if (offset <= -((int64_t)1 << 40) || offset >= ((int64_t)1 << 40)) return ADASPA_ERR_INVALID_ARG;
  RotaryParams r;
  memset(&r, 0, sizeof r);
  r.x[0] = (const u16*)q;
  r.x[1] = (const u16*)k;
  r.y[0] = (u16*)q_out;
  r.y[1] = (u16*)k_out;
  r.sx[0] = strides(p->q_stride);
  r.sx[1] = strides(p->k_stride);
  r.sy[0] = strides(p->q_out_stride);
  r.sy[1] = strides(p->k_out_stride);
  r.heads[0] = p->heads;
  r.heads[1] = p->kv_heads;
  r.B = p->batch;
  r.L = p->len;
  r.D = p->head_dim;
  r.P = p->pairs;
  r.axes = p->axes;
  for (int a = 0, end = 0; a < p->axes; ++a) r.axis_end[a] = end += p->axis_pairs[a];
  r.positions = positions;
  r.pos_b = p->position_stride[0];
  r.pos_t = p->position_stride[1];
  r.offsets = offsets;
  r.offset = offset;
  r.cos_by = p->magnitude;
  r.sin_by = way * p->magnitude;
  for (int i = 0; i < p->pairs; ++i) r.turns[i] = p->freq[i] / 6.283185307179586476925;
  return launch_rotary(r, p->dtype == ADASPA_FP16, p->layout == ADASPA_ROTARY_INTERLEAVED, (hipStream_t)stream) ==
                 hipSuccess
             ? ADASPA_OK
             : ADASPA_ERR_HIP;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

adaspa_status adaspa_rotary(const adaspa_rotary_problem* prob, const void* q, const void* k,
                            const int32_t* positions, int64_t offset, const int32_t* offsets, void* q_out,
                            void* k_out, void* stream) {
  return turn(prob, q, k, positions, offset, offsets, q_out, k_out, 1.f, stream);
}

adaspa_status adaspa_rotary_bwd(const adaspa_rotary_problem* prob, const void* dq_out, const void* dk_out,
                                const int32_t* positions, int64_t offset, const int32_t* offsets, void* dq, void* dk,
                                void* stream) {
  return turn(prob, dq_out, dk_out, positions, offset, offsets, dq, dk, -1.f, stream);
}

}  // extern "C"
#pragma GCC visibility pop
