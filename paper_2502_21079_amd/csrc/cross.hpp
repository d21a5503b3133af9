// Attention of queries over keys of another length (cross attention) and
// attention with a learned relative position bias: parameters shared by the
// C ABI (cross_api.hip) and the kernels (cross_fwd.hip, cross_bwd.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace adaspa {

typedef uint16_t u16;

// A [batch, head, token, D] view, strides in elements, D contiguous.
struct Strides {
  int64_t b, h, t;
};

constexpr int kMaxBucketSide = 256;    // buckets of one direction
constexpr int kMaxFar = 1024;          // distance from which on the bucket is the last one

struct RelBias {
  const void* table;                   // [buckets, H], fp32 or the type of q
  void* dtable;                        // its gradient, the same type (backward)
  int table_f32;
  int side;                            // buckets of one direction
  int both;                            // keys after the query have buckets of their own
  int far;                             // start[side - 1]
  int causal;
  int q_offset;                        // position of query 0 among the keys
  int at_end;                          // instead of q_offset: the queries end with their sample's keys
  uint16_t start[kMaxBucketSide];      // distance at which each bucket begins, ascending
};

struct CrossParams {
  const u16 *q, *k, *v, *dout;
  u16 *out, *dq, *dk, *dv;
  float* lse;                          // [B, H, Lq], may be null in the forward call
  Strides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  int B, H, Hk, G;                     // G = H / Hk query heads per key head
  int Lq, Lk;
  float scale, sl2;                    // sl2 = scale * log2(e)
  const int32_t* key_lens;             // [B], may be null
  const uint8_t* key_mask;             // [B, Lk], may be null; 0 = masked
  int64_t mask_stride;
  int splits;                          // ranges that an axis is divided into
  float* part_o;                       // forward: [splits, B*H*Lq, D]; backward dq: the same
  float* part_ml;                      // forward: [splits, B*H*Lq, 2] reference and sum
  float2* row_ld;                      // backward: [B*H*Lq] -LSE / scale (-inf for an empty row) and -delta
  float* part_kv;                      // backward: [splits, 2, B*Hk*Lk, D]
  int kv_splits;
  float* part_t;                       // backward: [B*H, key tiles * kv_splits, buckets] sums of dS
  int n_wg;                            // workgroups (set by the launcher)
  RelBias rb;
};

// Row tiles, splits and scratch of a call: by its shape alone, so that a
// workspace size, the launches and the results follow the shape.
struct CrossPlan {
  bool resident;                       // forward: the keys of a head stay in LDS, splits workgroups share its rows
  int splits, kv_splits;
  int64_t part_o, part_ml, row_ld, part_kv, part_t;   // byte offsets into the workspace
  int64_t bytes;
};
CrossPlan plan_fwd(const CrossParams& p, int D, bool bias);
CrossPlan plan_bwd(const CrossParams& p, int D, bool bias);

hipError_t launch_cross_fwd(CrossParams p, int D, bool f16, bool bias, const CrossPlan& plan, hipStream_t st);
hipError_t launch_cross_bwd(CrossParams p, int D, bool f16, bool bias, const CrossPlan& plan, hipStream_t st);

}  // namespace adaspa
