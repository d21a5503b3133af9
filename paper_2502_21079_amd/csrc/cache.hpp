// A key/value cache in 8 bits: its layout and the parameters shared by the C
// ABI (cache_api.hip) and the kernels (cache_rw.hip, cache_attn.hip).
#pragma once

#include "cross.hpp"

namespace adaspa {

// A pool of pages.  A page holds `page` tokens (16, 32, 64 or 128) of one
// sequence, for every key head
//   keys    e4m3 [page, D], rows of a token;
//   values  e4m3 [page / 16, D, 16]: sixteen tokens of a channel side by side,
//           the order in which the second product of attention takes them, so
//           that nothing has to be transposed where it is read;
//   two scales, powers of two in fp32: a value is its code times the scale.
struct CachePool {
  uint8_t *k, *v;                      // [pages, Hk, page * D]
  float *k_scale, *v_scale;            // [pages, Hk]
  const int32_t* table;                // [B, max_pages]: pages of a sequence in order
  int64_t table_stride;
  int pages, page, max_pages;
};

struct CacheParams {
  CachePool c;
  int B, H, Hk, G, D;
  int L;                               // tokens to write or read, or queries
  const int32_t* lens;                 // [B]: tokens of a sequence (write: before the call)
  const int32_t* new_lens;             // [B], may be null: how many of the L are there
  const int32_t* starts;               // read: [B], may be null: position of row 0
  const u16 *q, *k, *v;                // attention: queries; write: new keys and values
  u16 *out, *k_out, *v_out;            // attention: output; read: keys and values
  Strides sq, sk, sv, so;              // sk, sv: also those of k_out and v_out
  float* lse;                          // [B, H, L], may be null
  float sl2;                           // softmax scale * log2(e)
  int causal;
  int shares;                          // few rows: workgroups of a key head that share all samples' keys, 0: one a
                                       // sample
  int64_t* before;                     // few rows: [B + 1] turns before each sample
  int chunk, chunks;                   // many rows: keys of a range, ranges of a sequence at most
  float* part_o;                       // [2 * shares, Hk, G * L, D], or [chunks, B * H * L, D]
  float* part_ml;                      // the same with 2 in place of D: reference and sum
  int n_wg;
};

// Ranges and scratch of an attention call, by its shape alone.
struct CachePlan {
  bool few;                            // the rows of a key head fit in a wave's tiles
  bool bypass;                         // few rows: keys and values are read past the last-level cache
  int shares, chunk, chunks;
  int64_t part_ml, before, bytes;      // byte offsets into the workspace
};
// Few rows of a key head: up to kFewRows, and up to kSharedRows where the table is kSharedSteps turns
// (256 keys each) wide or wider.  Up to kWholeSteps turns a workgroup takes a sequence.
constexpr int kFewRows = 32, kSharedRows = 48, kWholeSteps = 8, kSharedSteps = 12;

CachePlan plan_cache_attn(const CacheParams& p, bool f16);
hipError_t launch_cache_write(CacheParams p, bool f16, hipStream_t st);
hipError_t launch_cache_read(CacheParams p, bool f16, hipStream_t st);
hipError_t launch_cache_attn(CacheParams p, bool f16, const CachePlan& plan, hipStream_t st);

}  // namespace adaspa
