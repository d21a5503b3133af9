// Rotary positions: parameters shared by the C ABI (rotary_api.hip) and the
// kernel (rotary.hip).
#pragma once

#include "cross.hpp"

namespace adaspa {

constexpr int kMaxRotaryPairs = 128;   // head dimensions up to 256
constexpr int kMaxRotaryAxes = 4;

struct RotaryParams {
  const u16* x[2];                     // queries, keys
  u16* y[2];
  Strides sx[2], sy[2];
  int heads[2];                        // 0: no such tensor
  int B, L, D, P;                      // the first 2 P elements of a head are turned
  int axes;
  int axis_end[kMaxRotaryAxes];        // pairs below axis_end[a] and not below axis_end[a - 1] go by axis a
  const int32_t* positions;            // [B, L, axes], may be null: the token's place
  int64_t pos_b, pos_t;                // its strides
  const int32_t* offsets;              // [B], may be null; added to every position of a sample
  int64_t offset;                      // added to every position
  float cos_by, sin_by;                // the factors on cosine and sine (sine: negative for the backward pass)
  int chunks;                          // work items of a token (set by the launcher)
  int groups, per_group;               // heads are divided into groups (set by the launcher)
  uint32_t items;                      // B * L * chunks (set by the launcher)
  double turns[kMaxRotaryPairs];       // revolutions per position of each pair
};

// Elements of a vector access: both the turned part and the rest are whole
// numbers of pairs of vectors.
inline int rotary_vector(int D, int P) {
  for (int v = 8; v > 1; v /= 2)
    if (P % v == 0 && (D / 2 - P) % v == 0) return v;
  return 1;
}

hipError_t launch_rotary(RotaryParams p, bool f16, bool interleaved, hipStream_t st);

}  // namespace adaspa
