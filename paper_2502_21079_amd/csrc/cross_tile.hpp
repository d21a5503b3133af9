// Building blocks of the cross-attention kernels (gfx950): element types,
// strided tiles in LDS that are read by rows and transposed alike, key
// visibility, the table of a relative position bias.
#pragma once

#include "attn_tile.hpp"
#include "cross.hpp"

namespace adaspa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Element types: eight values of an MFMA operand, the product, rounding.
struct BF16 {
  typedef bf16x8 x8;
  static constexpr bool kHalf = false;
  __device__ __forceinline__ static f32x16 mfma(x8 a, x8 b, f32x16 c) { return mfma32(a, b, c); }
  __device__ __forceinline__ static uint32_t pack(float a, float b) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
  }
  __device__ __forceinline__ static void unpack(uint32_t v, float& a, float& b) {
    a = __uint_as_float(v << 16);
    b = __uint_as_float(v & 0xFFFF0000u);
  }
  __device__ __forceinline__ static float load(const void* p, int64_t i) {
    return __uint_as_float((uint32_t)((const u16*)p)[i] << 16);
  }
  __device__ __forceinline__ static void store(void* p, int64_t i, float v) {
    ((__bf16*)p)[i] = (__bf16)v;
  }
};
struct FP16 {
  typedef f16x8 x8;
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static constexpr bool kHalf = true;
  __device__ __forceinline__ static f32x16 mfma(x8 a, x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  __device__ __forceinline__ static uint32_t pack(float a, float b) {
    const x2 r = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, r);
  }
  __device__ __forceinline__ static void unpack(uint32_t v, float& a, float& b) {
    const x2 r = __builtin_bit_cast(x2, v);
    a = (float)r[0];
    b = (float)r[1];
  }
  __device__ __forceinline__ static float load(const void* p, int64_t i) { return (float)((const _Float16*)p)[i]; }
  __device__ __forceinline__ static void store(void* p, int64_t i, float v) { ((_Float16*)p)[i] = (_Float16)v; }
};

// A [rows, D] tile of 16-bit elements in LDS, rows back to back, the 16-byte
// chunks of a row in an order of the row's own: chunk c of row r is at place
// c ^ order(r).  One order serves both ways a tile is read here: 16 rows at
// one column (operands along the row) fall in distinct banks, and so do the
// four rows of 64 bytes that 32 lanes of a transposed read take.
template <int D>
__device__ __forceinline__ int row_order(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
// MFMA step ks of a sum over D takes chunk row_chunk(ks) + 2 hw of each row:
// steps come in pairs over four chunks, the way load_tile finds them.  (Any
// order will do that both operands share.)
__host__ __device__ constexpr int row_chunk(int ks) { return 4 * (ks >> 1) + (ks & 1); }
// Lane address (elements) of a read along rows: row c32; the chunk of step ks
// of row 32 g + c32 is at (row_lane ^ 8 row_chunk(ks)) + 32 g D.
template <int D>
__device__ __forceinline__ int row_lane(int c32, int hw) {
  return c32 * D + ((2 * hw) ^ row_order<D>(c32)) * 8;
}
// Lane address of a transposed read; output block d of rows 16 s further down
// begins at (col_lane ^ 32 d) + 16 s D, and its second half at
// (col_lane ^ 16 ^ 32 d) + (16 s + 8) D.
template <int D>
__device__ __forceinline__ int col_lane(int lane) {
  const int gi = lane & 15, grp = lane >> 4, row = 4 * (lane >> 5) + (gi >> 2);
  return row * D + ((2 * (grp & 1) + ((gi & 3) >> 1)) ^ row_order<D>(row)) * 8 + 4 * (gi & 1);
}
template <class T>
__device__ __forceinline__ typename T::x8 read_row(const u16* p) {
  return *reinterpret_cast<const typename T::x8*>(p);
}
// Transposed operand from this lane's places in its two halves of 8 rows.
template <class T>
__device__ __forceinline__ typename T::x8 read_cols(const u16* lower, const u16* upper) {
  const s16x4 lo = lds_read_tr16(lower), hi = lds_read_tr16(upper);
  typename T::x8 v;
  __builtin_memcpy(&v, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
  return v;
}
// Transposed operand: 16 rows from `r16` on of output block d.
template <class T, int D>
__device__ __forceinline__ typename T::x8 read_col(const u16* tile, int ca, int d, int r16) {
  return read_cols<T>(tile + (ca ^ (32 * d)) + r16 * D, tile + (ca ^ 16 ^ (32 * d)) + (r16 + 8) * D);
}

// Loads of ROWS-row tiles straight into LDS by NW waves.  The source is the
// tile's first row (a 64-bit address: a long cache passes 32 bits) and offsets
// inside the tile; rows from `valid` on are left out by the buffer's bounds.
template <int D, int NW, int ROWS = 64>
struct TileLoad {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NINST = ROWS / RPI, PER = NINST / NW;
  static_assert(NINST % NW == 0 && (NW * RPI) % 16 == 0, "every wave loads alike, whole periods of the row order apart");
  uint32_t rel, step, wbase;
  __device__ __forceinline__ void init(int wave, int lane, int64_t row_stride) {
    const int p = wave * 64 + lane, row = p / CPR;
    rel = (uint32_t)(row * row_stride + ((p % CPR) ^ row_order<D>(row)) * 8) * 2u;
    step = (uint32_t)(NW * RPI * row_stride) * 2u;
    wbase = (uint32_t)wave * 1024u;
  }
  template <int J = 0>
  __device__ __forceinline__ void go(u32x4 r, uint32_t dst, uint32_t off) const {
    if constexpr (J < PER) {
      dma16<J * NW * 1024>(r, dst + wbase, off, 0u);
      go<J + 1>(r, dst, off + step);
    }
  }
  __device__ __forceinline__ static u32x4 buffer(const u16* first, int64_t row_stride, int valid) {
    const int n = valid < ROWS ? valid : ROWS;
    return rsrc_words(first, n <= 0 ? 0u : ((uint32_t)(n - 1) * (uint32_t)row_stride + D) * 2u);
  }
  __device__ __forceinline__ void issue(uint32_t dst, const u16* first, int64_t row_stride, int valid) const {
    go(buffer(first, row_stride, valid), dst, rel);
  }
  // Load n of this wave alone (a constant once the caller's loop is unrolled).
  template <int J = 0>
  __device__ __forceinline__ void issue_n(int n, uint32_t dst, u32x4 r) const {
    if constexpr (J < PER) {
      if (n == J) dma16<J * NW * 1024>(r, dst + wbase, rel + J * step, 0u);
      else issue_n<J + 1>(n, dst, r);
    }
  }
};

// A value that the compiler takes as new at this point: what is derived from it
// inside a loop is formed there (a few VALU operations) instead of being kept
// in registers, or spilled, over the whole loop.
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// f(0) ... f(N - 1) with compile-time indices.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}

// Clears rows of a tile whose bit in `keep` is 0 (rows below n), so that
// whatever a masked row holds, infinities and NaN too, meets a weight of zero
// as zero.
template <int D, int NT>
__device__ __forceinline__ void clear_rows(u16* tile, uint64_t keep, int tid) {
  for (int c = tid; c < 64 * (D / 8); c += NT)
    if (!((keep >> (c / (D / 8))) & 1)) *reinterpret_cast<u32x4*>(tile + c * 8) = u32x4{0, 0, 0, 0};
}

// Keys of sample b: the count of its own, within [0, Lk].
__device__ __forceinline__ int key_count(const CrossParams& p, int b) {
  if (!p.key_lens) return p.Lk;
  const int n = __builtin_amdgcn_readfirstlane(p.key_lens[b]);
  return n < 0 ? 0 : (n < p.Lk ? n : p.Lk);
}
// Bits of the 64 keys from j0 on that lie below n.
__device__ __forceinline__ uint64_t below(int j0, int n) {
  const int left = n - j0;
  return left >= 64 ? ~0ull : (left <= 0 ? 0ull : (1ull << left) - 1);
}
// One mask byte per lane of the 64 keys from j0 on (1 past n).
__device__ __forceinline__ int mask_byte(const CrossParams& p, int b, int j0, int n, int lane) {
  return j0 + lane < n ? p.key_mask[b * p.mask_stride + j0 + lane] : 1;
}

// --- relative position bias --------------------------------------------------
// The value added to a score depends on the head and on key position minus
// query position alone, and is constant beyond +-far.  Each workgroup keeps
// one head's values, times log2(e), in LDS: rel = -far - kPad .. far + kPad.
// A wave's tile of 32 x 64 scores spans 95 diagonals, so one that is not
// wholly beyond far never leaves the table.
// With `causal` the values of keys after the query are -inf.  Behind the table
// stand 32 entries of -inf, where a masked key's lane reads.
constexpr int kPad = 96;
__host__ __device__ __forceinline__ int bias_entries(int far) { return 2 * (far + kPad) + 1 + 32; }

// Table row of a relative position.
__device__ __forceinline__ int bucket_of(const uint16_t* start, const RelBias& rb, int rel) {
  int n = rb.both ? (rel < 0 ? -rel : rel) : (rel < 0 ? -rel : 0);
  n = n < rb.far ? n : rb.far;
  int lo = 0, hi = rb.side;                  // start[lo] <= n < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= n) lo = mid;
    else hi = mid;
  }
  return lo + (rb.both && rel > 0 ? rb.side : 0);
}
template <class T>
__device__ __forceinline__ float table_value(const RelBias& rb, int64_t i) {
  return rb.table_f32 ? ((const float*)rb.table)[i] : T::load(rb.table, i);
}
// Fills bt (bias_entries floats) for head h; start: LDS room of side entries.
// The caller has a barrier between this and the first read.  (shift: added to every
// value.)
template <class T, int NT>
__device__ __forceinline__ void fill_bias(float* bt, uint16_t* start, const CrossParams& p, int h, int tid,
                                          float shift = 0.f) {
  for (int i = tid; i < p.rb.side; i += NT) start[i] = p.rb.start[i];
  __syncthreads();
  const int n = bias_entries(p.rb.far);
  for (int i = tid; i < n; i += NT) {
    const int rel = i - p.rb.far - kPad;
    float v = -INFINITY;
    if (i < n - 32 && !(p.rb.causal && rel > 0))
      v = table_value<T>(p.rb, (int64_t)bucket_of(start, p.rb, rel) * p.H + h) * kLog2e + shift;
    bt[i] = v;
  }
}
// A 32 x 32 block whose smallest key minus query position is lo reads the
// table from here on: blocks beyond far take its constant ends.
__device__ __forceinline__ int bias_from(int lo, int far) {
  return lo >= far ? far : (lo <= -far - 62 ? -far - 62 : lo);
}
__device__ __forceinline__ int query_offset(const CrossParams& p, int n) { return p.rb.at_end ? n - p.Lq : p.rb.q_offset; }

// --- tiles of 32 rows between memory and registers ----------------------------
// An MFMA operand has row c32 in lanes c32 and c32 + 32, so an access that
// follows it takes 32 bytes of each of 32 rows.  Here each access takes 64 bytes
// of 16 rows (groups of 16 lanes take one chunk each), and two accesses, the
// lower and the upper 16 rows, exchange groups (one v_permlane16_swap per
// register).
template <class T, int D>
struct TileRegs {
  u32x4 w[D / 16];                                       // chunk 4 j + lane / 16 of rows (2 j: lower, 2 j + 1: upper)
  // a, b: this lane's rows lane % 16 and 16 + lane % 16.
  __device__ __forceinline__ void load(const u16* a, bool a_ok, const u16* b, bool b_ok, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      w[2 * j] = w[2 * j + 1] = u32x4{0, 0, 0, 0};
      if (a_ok) w[2 * j] = *reinterpret_cast<const u32x4*>(a + 32 * j + 8 * g);
      if (b_ok) w[2 * j + 1] = *reinterpret_cast<const u32x4*>(b + 32 * j + 8 * g);
    }
  }
  // The operands of MFMA steps 2 j and 2 j + 1.
  __device__ __forceinline__ void operands(typename T::x8 (&f)[D / 16]) const {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      u32x4 even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(w[2 * j][i], w[2 * j + 1][i], false, false);
        even[i] = r[0];
        odd[i] = r[1];
      }
      f[2 * j] = __builtin_bit_cast(typename T::x8, even);
      f[2 * j + 1] = __builtin_bit_cast(typename T::x8, odd);
    }
  }
};
template <class T, int D>
__device__ __forceinline__ void load_tile(const u16* a, bool a_ok, const u16* b, bool b_ok, int lane,
                                          typename T::x8 (&f)[D / 16]) {
  TileRegs<T, D> t;
  t.load(a, a_ok, b, b_ok, lane);
  t.operands(f);
}

// Writes a 32 x D tile held transposed (lane = row c32, columns 32 d + 8 i +
// 4 hw + j), scaled by inv: the halves, then groups of 16 lanes exchange until
// each store takes 64 bytes of 16 rows (a, b: rows lane % 16 and 16 + lane % 16).
template <class T, int D>
__device__ __forceinline__ void store_tile(const f32x16 (&o)[D / 32], float inv, u16* a, bool a_ok, u16* b, bool b_ok,
                                           int lane) {
  const int g = lane >> 4, chunk = ((g & 1) << 1) | (g >> 1);
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    u32x4 w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t x = T::pack(o[d][8 * i + 2 * j] * inv, o[d][8 * i + 2 * j + 1] * inv);
        const uint32_t y = T::pack(o[d][8 * i + 4 + 2 * j] * inv, o[d][8 * i + 5 + 2 * j] * inv);
        const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
        w[i][j] = r[0];
        w[i][2 + j] = r[1];
      }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto r = __builtin_amdgcn_permlane16_swap(w[0][j], w[1][j], false, false);
      w[0][j] = r[0];
      w[1][j] = r[1];
    }
    if (a_ok) *reinterpret_cast<u32x4*>(a + 32 * d + 8 * chunk) = w[0];
    if (b_ok) *reinterpret_cast<u32x4*>(b + 32 * d + 8 * chunk) = w[1];
  }
}
// The same in fp32, 16 bytes per lane as they lie.
template <int D>
__device__ __forceinline__ void store_tile_f32(const f32x16 (&o)[D / 32], float* row, bool ok, int hw) {
  if (!ok) return;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(row + 32 * d + 8 * i + 4 * hw) =
          f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
}
__device__ __forceinline__ float both_halves_max(float v) {
  float a, b;
  half_pair(v, a, b);
  return vmax(a, b);
}
__device__ __forceinline__ float both_halves_sum(float v) {
  float a, b;
  half_pair(v, a, b);
  return a + b;
}

// --- keys of a head kept in LDS ------------------------------------------------
// All keys and values of one (sample, key head), for kKeepWaves waves: K in the
// first half of kKeepBytes of LDS, V in the second, then 0 or -inf per key.
// Tiles lie at constant distances, so a lane needs its places in tile 0 and the
// rest of an address is the instruction's own.
template <class T, int D>
struct KeptKeys {
  static constexpr int TILES = kKeepBytes / 256 / D;
  int nt;                                                // tiles of 64 keys
  uint32_t whole;                                        // those of which every key is visible
  const float* mask;
  const u16* kp[D / 16];                                 // K along rows, per MFMA step
  const u16* vrow[D / 16];                               // V along rows
  const u16* vp[D / 32][2];                              // V transposed, per output block and half of 8 rows
  const u16* kcol[D / 32][2];                            // K transposed
  // meanwhile(): done while the tiles are on their way.
  template <typename F>
  __device__ __forceinline__ KeptKeys(const CrossParams& p, int b, int hk, int n, u16* lds, int wave, int lane, int tid,
                                      F&& meanwhile) {
    u16* sK = lds;
    u16* sV = lds + kKeepBytes / 4;
    float* sB = reinterpret_cast<float*>(lds + kKeepBytes / 2);
    const u16* kh = p.k + b * p.sk.b + hk * p.sk.h;
    const u16* vh = p.v + b * p.sv.b + hk * p.sv.h;
    nt = (n + 63) / 64;
    // All tiles are on their way before the first is waited for.
    TileLoad<D, kKeepWaves> lk, lv;
    lk.init(wave, lane, p.sk.t);
    lv.init(wave, lane, p.sv.t);
    int mb[TILES];
    static_for<TILES>([&](auto t) {
      mb[t] = 1;
      if (t >= nt) return;
      lk.issue(lds_addr(sK) + t * 128 * D, kh + t * 64 * p.sk.t, p.sk.t, n - t * 64);
      lv.issue(lds_addr(sV) + t * 128 * D, vh + t * 64 * p.sv.t, p.sv.t, n - t * 64);
      if (p.key_mask) mb[t] = mask_byte(p, b, t * 64, n, lane);
    });
    meanwhile();
    wait_vmem();
    __syncthreads();
    // Masked rows and those past n become zeros.
    whole = 0;
    static_for<TILES>([&](auto t) {
      if (t >= nt) return;
      const uint64_t keep = below(t * 64, n) & __ballot(mb[t] != 0);
      if (keep == ~0ull) {
        whole |= 1u << t;
        return;
      }
      if (wave == 0) sB[t * 64 + lane] = (keep >> lane) & 1 ? 0.f : -INFINITY;
      clear_rows<D, 64 * kKeepWaves>(sK + t * 64 * D, keep, tid);
      clear_rows<D, 64 * kKeepWaves>(sV + t * 64 * D, keep, tid);
    });
    __syncthreads();
    mask = sB;
    const int ra = row_lane<D>(lane & 31, lane >> 5), ca = col_lane<D>(lane);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      kp[ks] = sK + (ra ^ (8 * row_chunk(ks)));
      vrow[ks] = sV + (ra ^ (8 * row_chunk(ks)));
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        vp[d][h] = sV + (ca ^ (16 * h) ^ (32 * d));
        kcol[d][h] = sK + (ca ^ (16 * h) ^ (32 * d));
      }
  }
};

// Which query row a lane works on.  Without a bias the query heads that share
// a key head are rows of one problem (unit = (sample, key head), G * Lq rows);
// with one a unit is a (sample, query head).
struct RowOf {
  int b, h, i;
};
// The unit (sample b, head h; b * heads + h) at place u of the launch order:
// samples change first, so that every XCD, which gets a run of that order, has
// a share of the long samples and of the short ones.
__device__ __forceinline__ int unit_at(const CrossParams& p, int u, int heads) { return u % p.B * heads + u / p.B; }
// What a workgroup of a launch over units, ranges and tiles of rows or keys works
// on.  Tiles of a unit run side by side on one XCD, whose L2 then holds what they
// share; but under an order mask, where they differ in length, all units' longest
// tiles come first and the short ones fill the gaps (last: the last tiles are the
// longest, as with rows).
struct Place {
  int unit, split, tile;
};
template <bool BIAS>
__device__ __forceinline__ Place place_of(const CrossParams& p, int heads, int tiles, int splits, bool last) {
  Place w;
  if (BIAS && p.rb.causal && tiles > 1) {
    const int n = p.n_wg / tiles, u = xcd_remap(blockIdx.x % n, n), t = blockIdx.x / n;
    w.unit = unit_at(p, u / splits, heads);
    w.split = u % splits;
    w.tile = last ? tiles - 1 - t : t;
  } else {
    const int lid = xcd_remap(blockIdx.x, p.n_wg);
    w.unit = unit_at(p, lid / (tiles * splits), heads);
    w.split = lid / tiles % splits;
    w.tile = lid % tiles;
  }
  return w;
}
// Where the view with these strides has it.
template <typename P>
__device__ __forceinline__ P* at(P* base, const Strides& s, const RowOf& r) {
  return base + r.b * s.b + r.h * s.h + r.i * s.t;
}
template <bool BIAS>
__device__ __forceinline__ RowOf row_of(const CrossParams& p, int unit, int r) {
  RowOf o;
  if (BIAS) {
    o.b = unit / p.H;
    o.h = unit % p.H;
    o.i = r;
  } else {
    o.b = unit / p.Hk;
    const int g = p.G == 1 ? 0 : r / p.Lq;
    o.h = (unit % p.Hk) * p.G + g;
    o.i = r - g * p.Lq;
  }
  return o;
}

// The two rows that a lane loads and stores of the 32 from r on.
struct TwoRows {
  RowOf a, b;
  bool a_ok, b_ok;
};
template <bool BIAS>
__device__ __forceinline__ TwoRows two_rows(const CrossParams& p, int unit, int r, int n_rows, int lane) {
  TwoRows t;
  const int a = r + (lane & 15);
  t.a_ok = a < n_rows;
  t.b_ok = a + 16 < n_rows;
  t.a = row_of<BIAS>(p, unit, t.a_ok ? a : 0);
  t.b = row_of<BIAS>(p, unit, t.b_ok ? a + 16 : 0);
  return t;
}

}  // namespace adaspa
