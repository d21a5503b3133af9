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
  int far;                             // start[side - 1], at least 1
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
  float* part_d;                       // backward: [splits, B*H*Lq] shares of delta
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
  bool resident;                       // the keys of a head stay in LDS, splits workgroups share its rows
  bool small;                          // backward: queries and keys of a head fit in LDS, one kernel does all
  bool delta_first;                    // backward: a pass for delta, which dq then takes
  int splits, kv_splits;
  int64_t part_o, part_ml, part_d, row_ld, part_kv, part_t;   // byte offsets into the workspace
  int64_t bytes;
};

// Keys of a head kept in LDS: few enough for it, and rows enough for a tile of
// each wave of 256 workgroups.
constexpr int kKeepBytes = 131072;     // K, then V
constexpr int kKeepWaves = 8;
// Row blocks of 32 that a wave of the forward kernel works on at a time: at d 64
// registers are there for two, which share every operand read from LDS and
// have twice the bytes in flight.
constexpr int keep_rows(int D) { return D == 64 ? 2 : 1; }
inline int64_t keep_tiles(const CrossParams& p, int row_blocks) {
  return ((int64_t)p.G * p.Lq + 32 * row_blocks - 1) / (32 * row_blocks);
}
inline bool keep_keys(const CrossParams& p, int D, bool bias, int row_blocks) {
  return !bias && (int64_t)(p.Lk + 63) / 64 * 64 * D * 4 <= kKeepBytes &&
         (int64_t)p.B * p.Hk * keep_tiles(p, row_blocks) >= 256 * kKeepWaves;
}
// Workgroups that share a unit's rows: as many as fill the rounds of 256 best
// (a workgroup's start counts as three tiles), and at least two rounds where
// samples have lengths of their own, so that those with few keys make room.
inline int keep_chunks(const CrossParams& p, int row_blocks) {
  const int64_t units = (int64_t)p.B * p.Hk, tiles = keep_tiles(p, row_blocks);
  int64_t best = -1, chunks = 1;
  for (int64_t n = 1; n <= 256 && n * kKeepWaves < tiles + kKeepWaves; ++n) {
    if (p.key_lens && units * n < 512 && (n + 1) * kKeepWaves < tiles + kKeepWaves) continue;
    const int64_t cost = (units * n + 255) / 256 * ((tiles + n * kKeepWaves - 1) / (n * kKeepWaves) + 3);
    if (best < 0 || cost < best) {
      best = cost;
      chunks = n;
    }
  }
  return (int)chunks;
}
inline uint32_t keep_lds_bytes(int Lk) { return kKeepBytes + (uint32_t)(Lk + 63) / 64 * 256; }

CrossPlan plan_fwd(const CrossParams& p, int D, bool bias);
CrossPlan plan_bwd(const CrossParams& p, int D, bool bias);

hipError_t launch_cross_fwd(CrossParams p, int D, bool f16, bool bias, const CrossPlan& plan, hipStream_t st);
hipError_t launch_cross_bwd(CrossParams p, int D, bool f16, bool bias, const CrossPlan& plan, hipStream_t st);

}  // namespace adaspa
