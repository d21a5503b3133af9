// Backward pass of the attention in cross_fwd.hip (gfx950).
//
//   P = exp(S - lse), dP = dO V^T, delta_i = dO_i . O_i, dS = P (dP - delta)
//   dq = scale dS K, dk = scale dS^T Q, dv = P^T dO   (dk, dv summed over the
//   query heads that share a key head)
//   dtable[u, h] = sum of dS over the pairs of bucket u
//
// Two kernels, each with its own axis in registers: cross_dq_kernel walks the
// keys for 128 query rows, cross_dkv_kernel the queries for its keys.  Both
// form S and dP again.  The table's gradient is added up in cross_dkv_kernel:
// its delta is the exact one.  No sum is added
// to memory by more than one workgroup: partial sums go to the workspace and
// are added in a fixed order, so results are the same from call to call.
//
// P and dS enter the second products in the inputs' type, which is what the matrix
// pipe takes; all sums are fp32.  Either is off by half a step of its own, so dv, dk and
// dq are within 1.4 to 1.5 times their final rounding.  A value is split in two
// (split_pair), at one product more, only where something else would come on top: delta
// from the rounded output (dq at d 128), or chance among a few values (problems of up to
// 64 queries and keys).  The table's gradient takes dS in fp32.
#include "cross_tile.hpp"

namespace adaspa {

namespace {
constexpr int kDqRows = 128;           // query rows of a workgroup of cross_dq_kernel
constexpr int kDkvWaves = 4;           // waves of 32 keys of a workgroup of cross_dkv_kernel
// delta from the rounded output is off by its rounding, which dq carries
// times sum_j P_ij k_j.  Where registers allow that sum next to dq (d 64), dq is
// put right by it once the row's exact delta is known: dq's error against 64 bits
// falls from about 1.5 to 1.4 times that of the final rounding alone (the rest
// is dS, rounded for the product).
template <int D>
constexpr bool kExactDq = D == 64;
// At d 128 they do not, and delta's error can be as large as dS's rounding (162
// rows over 2,245 keys: 1.6 times the final rounding together).  There dS goes
// into the product as a sum of two values, its upper bits and what they leave, so
// that delta's error and the final rounding are all that is left: 1.3 times the latter
// for scores of unit variance, 1.7 for scores that spread three times as far.
template <class T>
__device__ __forceinline__ uint2 split_pair(float a, float b) {
  const uint32_t hi = T::pack(a, b);
  float c, d;
  T::unpack(hi, c, d);
  return make_uint2(hi, T::pack(a - c, b - d));
}

// fp16 weights for dv carry 2^14 (no weight is above 1): of 100,000 keys most have
// weights below fp16's smallest normal number, and so have keys that no query looks at
// (weights of 1e-6 without it: the dv of those keys off by 0.3 to 0.8%).
template <class T>
constexpr float kShift = T::kHalf ? 14.f : 0.f;
template <class T>
constexpr float kUnshift = T::kHalf ? 1.f / 16384.f : 1.f;

// fp16 ends at 65504 and has its 11 bits down to 2^-14 only, while dS goes with the
// sizes of dO (a loss's mean over many elements, or its scale) and of v and with one
// over the number of keys.  So in fp16 dS enters its products times a power of two, and
// the sums are divided by it where they are stored: one per row for dq, one per key for
// dk, which are lanes of the accumulators, so that a lane changes its own alone.  The
// first values other than 0 bring their largest to [2^6, 2^7); a later one that would
// pass 2^15 brings the factor, and what has been added up, down again.  All of it is
// exact, and what still falls below fp16's smallest step is 2^-31 of the largest.
// (Without it output gradients of 1e-4 over 200 to 9,000 keys left dq off by 2e-3 to
// 9e-2 of its size, those of 1e-5 by up to 0.6, and some of 12,000 gave infinities.)
// A maximum per pair of values and a product per value: training passes in fp16 take 3
// to 5% longer (24 x 50,000 rows over 256 keys, d 128: 975 and 1,013 us; 12 x 4,095
// tokens under an order mask 404 and 423).  bf16 has fp32's range and needs none.
template <class T>
struct Spread {
  float up = T::kHalf ? 0x1p64f : 1.f, down = T::kHalf ? 0x1p-64f : 1.f;
  __device__ __forceinline__ static bool over(float most) { return !(most <= 0x1p15f); }   // also NaN
  // A new factor where `most`, the largest magnitude of this lane's values with the
  // present one, or its other half's is over; returns what it changed by.
  template <int N>
  __device__ __forceinline__ float lower(float most, f32x16 (&acc)[N]) {
    const float was = down;
    most = both_halves_max(most);
    if (over(most)) {
      // 2^e <= most < 2^(e + 1), without the factor; the new one is 2^(6 - e), at most 2^64.
      const uint32_t e = __float_as_uint(most * down) >> 23, b = 254 + 6 - e;
      up = __uint_as_float((b < 191 ? b : 191) << 23);
      down = 1.f / up;
    }
    const float by = up * was;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] *= by;
    return by;
  }
  // dS as it enters the product that is summed up in acc.
  template <int N>
  __device__ __forceinline__ void apply(f32x16& y, f32x16 (&acc)[N]) {
    if constexpr (T::kHalf) {
      float m[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 16; e += 2)
        m[(e >> 1) & 1] = vmax(m[(e >> 1) & 1], vmax(__builtin_fabsf(y[e]), __builtin_fabsf(y[e + 1])));
      const float most = vmax(m[0], m[1]) * up;
      if (__any(over(most))) lower(most, acc);
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] *= up;
    }
  }
  template <int N>
  __device__ __forceinline__ void undo(f32x16 (&acc)[N]) const {
    if constexpr (T::kHalf) {
#pragma unroll
      for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= down;
    }
  }
};

// What a launch of cross_dq_kernel does.  Where few rows share many keys the
// keys are split, and delta, which needs them all, comes first, as it does at d 128
// wherever a row can see more than 2,048 keys: DELTA leaves each
// range's sum of P dP, DQ adds these up and forms its range's dq.  (With delta
// from the rounded output there, 25 queries over 18,266 keys had dq off by 5.4e-3
// of its size where rounding dS and dq alone gives 2.4e-3.)
enum { WHOLE = 0, DELTA = 1, DQ = 2 };
}  // namespace

// dq of 128 query rows over one range of their keys: four waves of 32 rows, whose q
// and dO stay in registers, tiles of 64 keys through two slots.  What bounds it: under
// an order mask the last rows' walk (12 x 4,095 tokens at d 128, fp16: 64 tiles one after
// the other, 101 us for delta and 127 for dq, the matrix pipe 19 and 23% busy); otherwise products and exponentials
// that two waves per SIMD overlap only in part.
template <class T, int D, bool BIAS, int PASS>
__global__ __launch_bounds__(256, 2) void cross_dq_kernel(const CrossParams p) {
  constexpr int NW = 4, KE = 64 * D;
  constexpr bool EXACT = PASS == WHOLE && kExactDq<D>, SPLIT = PASS == WHOLE && !kExactDq<D>;
  __shared__ __attribute__((aligned(1024))) u16 ring[2][2 * KE];
  __shared__ uint16_t start[BIAS ? kMaxBucketSide : 1];
  extern __shared__ __attribute__((aligned(16))) float bt[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;

  const int n_rows = BIAS ? p.Lq : p.G * p.Lq, n_rt = (n_rows + kDqRows - 1) / kDqRows;
  const Place place = place_of<BIAS>(p, BIAS ? p.H : p.Hk, n_rt, p.splits, true);
  const int unit = place.unit, split = place.split, r0 = place.tile * kDqRows;
  const int rw = r0 + wave * 32, r = rw + c32;             // first row of the wave, row of the lane
  const bool row_ok = r < n_rows;
  const RowOf ro = row_of<BIAS>(p, unit, row_ok ? r : 0);
  const int b = BIAS ? unit / p.H : unit / p.Hk, hk = BIAS ? (unit % p.H) / p.G : unit % p.Hk;
  const int n = key_count(p, b), off = query_offset(p, n);

  int kend = n;
  if (BIAS && p.rb.causal) {
    const int64_t last = (int64_t)(r0 + kDqRows < n_rows ? r0 + kDqRows : n_rows) + off;
    kend = last < kend ? (last < 0 ? 0 : (int)last) : kend;
  }
  const int nt = (kend + 63) / 64;
  const int t0 = (int)((int64_t)nt * split / p.splits), t1 = (int)((int64_t)nt * (split + 1) / p.splits);

  TileLoad<D, NW> lk, lv;
  lk.init(wave, lane, p.sk.t);
  lv.init(wave, lane, p.sv.t);
  const u16* kh = p.k + b * p.sk.b + hk * p.sk.h;
  const u16* vh = p.v + b * p.sv.b + hk * p.sv.h;
  int mb[2] = {1, 1};
  auto issue = [&](auto slot, int t) {
    const uint32_t dst = lds_addr(ring[0]) + slot * 4 * KE;
    lk.issue(dst, kh + (int64_t)t * 64 * p.sk.t, p.sk.t, n - t * 64);
    lv.issue(dst + KE * 2, vh + (int64_t)t * 64 * p.sv.t, p.sv.t, n - t * 64);
    if (p.key_mask) mb[slot] = mask_byte(p, b, t * 64, n, fresh(lane));
  };
  // Both tiles of a short walk fit in the ring: there delta comes exactly from a walk
  // of its own.  Rows with few keys have the largest outputs, whose rounding would
  // be more than dS's (36 causal rows: dq 1.5 times the final rounding without).
  const bool few = SPLIT && nt <= 2;
  if (t0 < t1) issue(integral_constant<int, 0>{}, t0);
  if (few && nt == 2) issue(integral_constant<int, 1>{}, 1);

  const int64_t row = ((int64_t)ro.b * p.H + ro.h) * p.Lq + ro.i;
  const TwoRows two = two_rows<BIAS>(p, unit, rw, n_rows, lane);
  typename T::x8 qf[D / 16], gf[D / 16];
  load_tile<T, D>(at(p.q, p.sq, two.a), two.a_ok, at(p.q, p.sq, two.b), two.b_ok, lane, qf);
  load_tile<T, D>(at(p.dout, p.sdo, two.a), two.a_ok, at(p.dout, p.sdo, two.b), two.b_ok, lane, gf);
  float nlse2 = -INFINITY, delta = 0.f;                    // -log2-LSE; a row without a key: every weight 0
  const int64_t all_rows = (int64_t)p.B * p.H * p.Lq;
  if (PASS == WHOLE) {
    typename T::x8 of[D / 16];
    load_tile<T, D>(at((const u16*)p.out, p.so, two.a), two.a_ok, at((const u16*)p.out, p.so, two.b), two.b_ok, lane, of);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[ks][e], (float)of[ks][e], delta);
    delta = both_halves_sum(delta);
  }
  if (PASS == DQ && row_ok) {
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) delta += p.part_d[s * all_rows + row];
  }
  {
    const float z = row_ok ? p.lse[row] : -INFINITY;
    if (z != -INFINITY) nlse2 = -z * kLog2e;
  }
  if (BIAS) fill_bias<T, 256>(bt, start, p, unit % p.H, tid);
  float more = 0.f;                                        // sum of dS: what delta lacks (DELTA: of P dP)
  Spread<T> spread;

  f32x16 acc[D / 32], pk[EXACT ? D / 32 : 1];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc[d] = f32x16{};
  if (EXACT) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) pk[EXACT ? d : 0] = f32x16{};
  }
  // This lane's places in slot 0; the slots lie at constant distances.
  const u16* kp[D / 16];
  const u16* kcol[D / 32][2];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) kp[ks] = ring[0] + (row_lane<D>(c32, hw) ^ (8 * row_chunk(ks)));
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int h = 0; h < 2; ++h) kcol[d][h] = ring[0] + (col_lane<D>(lane) ^ (16 * h) ^ (32 * d));
  const int rel0 = 4 * hw - (ro.i + off);

  const int far = BIAS ? p.rb.far : 0;
  // Waits for tile t and has the next one loaded; its visible keys, the others
  // cleared (none: left as it is).
  auto enter = [&](auto u, int t) {
    wait_vmem();
    const uint64_t keep = below(t * 64, n) & (p.key_mask ? __ballot(mb[u] != 0) : ~0ull);
    __syncthreads();
    if (!few && t + 1 < t1) issue(integral_constant<int, 1 - u>{}, t + 1);
    if (keep != ~0ull && keep != 0) {
      clear_rows<D, 256>(ring[u], keep, fresh(tid));
      clear_rows<D, 256>(ring[u] + KE, keep, fresh(tid));
      __syncthreads();
    }
    return keep;
  };
  // Not for a wave without rows, or whose rows come before all of these keys.
  auto idle = [&](int t) { return rw >= n_rows || (BIAS && p.rb.causal && t * 64 > rw + 31 + off); };
  // P and dP - delta of tile t's keys 32 g and on.
  auto block = [&](auto u, int t, int g, uint64_t keep, f32x16& x, f32x16& y) {
    const int row0 = u * 128 + 32 * g;                     // a slot is two tiles of 64 rows
    x = f32x16{};
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = -delta;            // dP's sums begin at -delta
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      x = T::mfma(read_row<T>(kp[ks] + row0 * D), qf[ks], x);
      y = T::mfma(read_row<T>(kp[ks] + KE + row0 * D), gf[ks], y);
    }
    if (BIAS) {
      const int lo = t * 64 + 32 * g - (rw + 31 + off);    // the block's smallest key minus query position
      if (lo >= far || lo <= -far - 62) {
        const float c = bt[lo >= far ? 2 * (far + kPad) : 0] + nlse2;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = fmaf(x[e], p.sl2, c);
      } else {
        const float* at = bt + (row_ok ? rel0 + t * 64 + 32 * g : lo) + far + kPad;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = fmaf(x[e], p.sl2, at[8 * (e >> 2) + (e & 3)] + nlse2);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = fmaf(x[e], p.sl2, nlse2);
    }
    if (keep != ~0ull) {
      const uint32_t mine = (uint32_t)(keep >> (32 * g)) >> (4 * hw);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((mine >> (8 * (e >> 2) + (e & 3))) & 1)) x[e] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = fast_exp2(x[e]);
  };
  uint64_t keeps[2] = {0, 0};                              // of a short walk's tiles
  if (few) {
    static_for<2>([&](auto u) {
      if (u < nt) keeps[u] = enter(u, u);
    });
    float s = 0.f;
    delta = 0.f;
    static_for<2>([&](auto u) {
      if (keeps[u] == 0 || idle(u)) return;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        f32x16 x, y;
        block(u, u, g, keeps[u], x, y);
#pragma unroll
        for (int e = 0; e < 16; ++e) s = fmaf(x[e], y[e], s);
      }
    });
    delta = both_halves_sum(s);
  }
  auto tile = [&](auto u, int t) {
    const uint64_t keep = few ? keeps[u] : enter(u, t);
    if (keep == 0 || idle(t)) return;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int row0 = u * 128 + 32 * g;
      f32x16 x, y;
      block(u, t, g, keep, x, y);
      float s0 = 0.f, s1 = 0.f;
      if (PASS == DELTA) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          s0 = fmaf(x[e], y[e], s0);
          s1 = fmaf(x[e + 1], y[e + 1], s1);
        }
        more += s0 + s1;
        continue;
      }
      u32x4 w[2], wp[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] *= x[e];
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        s0 += y[e];
        s1 += y[e + 1];
      }
      spread.apply(y, acc);
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        if (SPLIT) {
          const uint2 v = split_pair<T>(y[e], y[e + 1]);
          w[e >> 3][(e & 7) >> 1] = v.x;
          wp[e >> 3][(e & 7) >> 1] = v.y;
        } else {
          w[e >> 3][(e & 7) >> 1] = T::pack(y[e], y[e + 1]);
          wp[e >> 3][(e & 7) >> 1] = T::pack(x[e], x[e + 1]);
        }
      }
      more += s0 + s1;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const typename T::x8 ds = __builtin_bit_cast(typename T::x8, w[s]);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const typename T::x8 kf = read_cols<T>(kcol[d][0] + (row0 + 16 * s) * D, kcol[d][1] + (row0 + 16 * s + 8) * D);
          acc[d] = T::mfma(kf, ds, acc[d]);
          if (SPLIT) acc[d] = T::mfma(kf, __builtin_bit_cast(typename T::x8, wp[s]), acc[d]);
          if (EXACT) pk[EXACT ? d : 0] = T::mfma(kf, __builtin_bit_cast(typename T::x8, wp[s]), pk[EXACT ? d : 0]);
        }
      }
    }
  };
  for (int t = t0; t < t1; t += 2) {
    tile(integral_constant<int, 0>{}, t);
    if (t + 1 < t1) tile(integral_constant<int, 1>{}, t + 1);
  }

  more = both_halves_sum(more);
  if (PASS == DELTA) {
    if (row_ok && hw == 0) p.part_d[split * all_rows + row] = more;
    return;
  }
  spread.undo(acc);
  if (EXACT) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] = fmaf(-more, pk[EXACT ? d : 0][e], acc[d][e]);
  }
  if (PASS == DQ && p.splits > 1) store_tile_f32<D>(acc, p.part_o + (split * all_rows + row) * D, row_ok, hw);
  else store_tile<T, D>(acc, p.scale, at(p.dq, p.sdq, two.a), two.a_ok, at(p.dq, p.sdq, two.b), two.b_ok, lane);
  // What cross_dkv_kernel takes as delta is free of the output's rounding: the
  // weights add up to 1, so the sum of P dP is delta and the sum of dS.
  const float exact = PASS == DQ ? delta : delta + more;
  if (row_ok && hw == 0 && split == 0) p.row_ld[row] = make_float2(nlse2 / p.sl2, -exact);
}

// dq with few keys: they stay in LDS, as in the forward pass, and each wave
// walks row tiles of 32 on its own, without barriers.  TWICE is for the fewest:
// S and dP are formed twice, delta exactly from the first time, and the output is
// not read, since there the rows' way through memory takes longer than the products
// (us, one walk and the output against two walks: 24 x 110,080 rows over 64 keys,
// d 64 311 and 259, d 128 593 and 452; whole training passes at d 128, 24 x 50,000
// rows over 128 keys 602 and 580, 48 x 20,000 over 100 479 and 474).  What bounds it
// otherwise: the products beside the rows' way through memory (24 x 110,080 rows
// over 256 keys, d 128: 2.7 GB, 565 us at a large copy's rate; four products, 692
// GFLOP, 600 us at a large product's; 772 us, the matrix pipe 45% busy).
template <int D>
constexpr int kTwiceBlocks = D == 64 ? 2 : 4;              // blocks of 32 keys that are walked twice
template <class T, int D, bool TWICE>
__global__ __launch_bounds__(64 * kKeepWaves, kKeepWaves / 4) void cross_keep_dq_kernel(const CrossParams p) {
  constexpr int NW = kKeepWaves;
  constexpr bool EXACT = !TWICE && kExactDq<D>, SPLIT = !TWICE && !kExactDq<D>;
  extern __shared__ __attribute__((aligned(1024))) u16 keep_lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;
  const int lid = xcd_remap(blockIdx.x, p.n_wg);
  const int unit = unit_at(p, lid / p.splits, p.Hk), chunk = lid % p.splits;
  const int b = unit / p.Hk, hk = unit % p.Hk, n = key_count(p, b);
  const int n_rows = p.G * p.Lq, n_rt = (n_rows + 31) / 32;
  const int rt1 = (int)((int64_t)n_rt * (chunk + 1) / p.splits);
  int rt = (int)((int64_t)n_rt * chunk / p.splits) + wave;

  const KeptKeys<T, D> keys(p, b, hk, n, keep_lds, wave, lane, tid, []() {});
  for (; rt < rt1; rt += NW) {
    const int r = rt * 32 + c32;
    const int64_t row = (int64_t)unit * n_rows + r;        // a unit's rows are consecutive
    typename T::x8 qf[D / 16], gf[D / 16];
    float delta = 0.f, nlse2 = -INFINITY;                  // -log2-LSE; a row without a key: every weight 0
    {
      const TwoRows two = two_rows<false>(p, unit, rt * 32, n_rows, fresh(lane));
      TileRegs<T, D> q, g, o;
      g.load(at(p.dout, p.sdo, two.a), two.a_ok, at(p.dout, p.sdo, two.b), two.b_ok, lane);
      if (!TWICE) o.load(at((const u16*)p.out, p.so, two.a), two.a_ok, at((const u16*)p.out, p.so, two.b), two.b_ok, lane);
      q.load(at(p.q, p.sq, two.a), two.a_ok, at(p.q, p.sq, two.b), two.b_ok, lane);
      const float z = r < n_rows ? p.lse[row] : -INFINITY;
      if (z != -INFINITY) nlse2 = -z * kLog2e;
      g.operands(gf);
      if (!TWICE) {
        typename T::x8 of[D / 16];
        o.operands(of);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[ks][e], (float)of[ks][e], delta);
      }
      q.operands(qf);
    }
    // P and dP - delta of block j of 32 keys.
    f32x16 from;                                           // dP's sums begin at -delta
    auto block = [&](auto j, f32x16& x, f32x16& y) {
      constexpr int row0 = 32 * j;
      x = f32x16{};
      y = from;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        x = T::mfma(read_row<T>(keys.kp[ks] + row0 * D), qf[ks], x);
        y = T::mfma(read_row<T>(keys.vrow[ks] + row0 * D), gf[ks], y);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = fmaf(x[e], p.sl2, nlse2);
      if (!((keys.whole >> (j / 2)) & 1)) {
        const float* at = keys.mask + row0 + 4 * hw;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] += at[8 * (e >> 2) + (e & 3)];
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = fast_exp2(x[e]);
    };
    if (TWICE) {
      from = f32x16{};
      static_for<kTwiceBlocks<D>>([&](auto j) {
        if (j / 2 >= keys.nt) return;
        f32x16 x, y;
        block(j, x, y);
#pragma unroll
        for (int e = 0; e < 16; ++e) delta = fmaf(x[e], y[e], delta);
      });
    }
    delta = both_halves_sum(delta);
    f32x16 acc[D / 32], pk[EXACT ? D / 32 : 1];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) acc[d] = pk[EXACT ? d : 0] = f32x16{};
#pragma unroll
    for (int e = 0; e < 16; ++e) from[e] = -delta;
    float more = 0.f;                                      // sum of dS: what delta lacks
    Spread<T> spread;
    static_for<TWICE ? kTwiceBlocks<D> : 2 * KeptKeys<T, D>::TILES>([&](auto j) {
      constexpr int row0 = 32 * j;
      if (j / 2 >= keys.nt) return;
      f32x16 x, y;
      block(j, x, y);
      u32x4 w[2], wp[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] *= x[e];
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        s0 += y[e];
        s1 += y[e + 1];
      }
      spread.apply(y, acc);
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        if (SPLIT) {
          const uint2 v = split_pair<T>(y[e], y[e + 1]);
          w[e >> 3][(e & 7) >> 1] = v.x;
          wp[e >> 3][(e & 7) >> 1] = v.y;
        } else {
          w[e >> 3][(e & 7) >> 1] = T::pack(y[e], y[e + 1]);
          wp[e >> 3][(e & 7) >> 1] = T::pack(x[e], x[e + 1]);
        }
      }
      more += s0 + s1;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const typename T::x8 ds = __builtin_bit_cast(typename T::x8, w[s]);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const u16* lo = keys.kcol[d][0] + (row0 + 16 * s) * D;
          const u16* hi = keys.kcol[d][1] + (row0 + 16 * s + 8) * D;
          const typename T::x8 kf = read_cols<T>(lo, hi);
          acc[d] = T::mfma(kf, ds, acc[d]);
          if (SPLIT) acc[d] = T::mfma(kf, __builtin_bit_cast(typename T::x8, wp[s]), acc[d]);
          if (EXACT) pk[EXACT ? d : 0] = T::mfma(kf, __builtin_bit_cast(typename T::x8, wp[s]), pk[EXACT ? d : 0]);
        }
      }
    });
    // What cross_dkv_kernel takes as delta is free of the output's rounding: the
    // weights add up to 1, so the sum of P dP is delta and the sum of dS.
    more = both_halves_sum(more);
    const float exact = delta + more;
    spread.undo(acc);
    if (EXACT) {
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = fmaf(-more, pk[EXACT ? d : 0][e], acc[d][e]);
    }
    if (r < n_rows && hw == 0) p.row_ld[row] = make_float2(nlse2 / p.sl2, -exact);
    const TwoRows two = two_rows<false>(p, unit, rt * 32, n_rows, fresh(lane));
    store_tile<T, D>(acc, p.scale, at(p.dq, p.sdq, two.a), two.a_ok, at(p.dq, p.sdq, two.b), two.b_ok, lane);
  }
}

// Diagonal sums of a 32 x 32 block held as lane (hw, c32) = column c32, element
// e = row 8 (e / 4) + 4 hw + e % 4, added to at[31 + column - row].  Row by row,
// the sum so far moves up one lane and the next row is added, so a diagonal's
// sum gathers in one lane: two chains of 16 rows side by side, the first one's
// then moved up by 16 lanes.
__device__ __forceinline__ void add_diagonals(const f32x16& x, float* at, int lane) {
  uint32_t row[32];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int r = 8 * (e >> 2) + (e & 3);
    const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[e]), 0u, false, false);
    row[r] = v[0];                                        // the lower half's row, nothing above it
    row[r + 4] = v[1];
  }
  float s[2] = {__uint_as_float(row[0]), __uint_as_float(row[16])};
#pragma unroll
  for (int r = 1; r < 16; ++r)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int moved = __builtin_amdgcn_update_dpp(0, __float_as_int(s[c]), 0x138, 0xF, 0xF, true);   // wave_shr:1
      s[c] = __int_as_float(moved) + __uint_as_float(row[16 * c + r]);
    }
  // Rows of 16 lanes [a0 a1 a2 0] to [0 a0 a1 a2].
  const auto odd = __builtin_amdgcn_permlane16_swap(0u, __float_as_uint(s[0]), false, false);   // [0 a0 0 a2], [0 a1 0 0]
  const auto even = __builtin_amdgcn_permlane16_swap(odd[1], 0u, false, false);                 // ..., [a1 0 0 0]
  const auto third = __builtin_amdgcn_permlane32_swap(0u, even[1], false, false);               // [0 0 a1 0], ...
  s[1] += __uint_as_float(odd[0]) + __uint_as_float(third[0]);
  // No two lanes share a place, so the order of a place's additions is the program's.
  if (lane < 63) __hip_atomic_fetch_add(at + lane, s[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
constexpr int kDiagPad = 62;           // diagonals of a block near the diagonal that lie beyond far
__host__ __device__ __forceinline__ int diag_entries(int far) { return 2 * (far + kDiagPad) + 1; }

// A workgroup's sums of dS for the head it is at: by diagonal in LDS (each wave
// its own, so that their order is the program's), and beyond far on either side
// in registers.  They lie behind the bias table bt.
template <int NW>
struct TableSums {
  float *bt, *all, *mine;
  float (*far_sum)[NW];
  const uint16_t* start;
  int far, nd, buckets, wave, lane, tid;
  float below, above;
  __device__ __forceinline__ TableSums(const CrossParams& p, float* bt, float (*far_sum)[NW], const uint16_t* start, int far,
                                       int wave, int lane, int tid)
      : bt(bt), all(bt + bias_entries(far)), far_sum(far_sum), start(start), far(far), nd(diag_entries(far)),
        buckets(p.rb.both ? 2 * p.rb.side : p.rb.side), wave(wave), lane(lane), tid(tid), below(0.f), above(0.f) {
    mine = all + wave * nd;
  }
  __device__ __forceinline__ void clear() {
    for (int i = tid; i < NW * nd; i += 64 * NW) all[i] = 0.f;
  }
  // dS of a block whose smallest key minus query position is lo.
  __device__ __forceinline__ void add(const f32x16& ds, int lo) {
    if (lo >= far || lo <= -far - 62) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) s += ds[e];
      if (lo >= far) above += s;
      else below += s;
    } else {
      add_diagonals(ds, mine + lo + far + kDiagPad, lane);
    }
  }
  // Writes the share and starts over (the bias table is overwritten).
  __device__ __forceinline__ void flush(const CrossParams& p, float* share) {
    const float lo = wave_sum(below), hi = wave_sum(above);
    below = above = 0.f;
    if (lane == 0) {
      far_sum[0][wave] = lo;
      far_sum[1][wave] = hi;
    }
    __syncthreads();
    for (int i = tid; i < nd; i += 64 * NW) {
      float s = 0.f;
      for (int w = 0; w < NW; ++w) {
        s += all[w * nd + i];
        all[w * nd + i] = 0.f;
      }
      bt[i] = s;
    }
    __syncthreads();
    const int mid = far + kDiagPad;
    for (int u = wave; u < buckets; u += NW) {
      const bool ahead = u >= p.rb.side;
      const int m = ahead ? u - p.rb.side : u;
      const bool last = m == p.rb.side - 1;
      int d = start[m];
      const int d1 = last ? mid + 1 : start[m + 1];
      if (ahead && d == 0) d = 1;
      // One direction: every key after the query is in the bucket of distance 0, the last
      // that begins there.
      const bool after = !p.rb.both && d == 0 && d1 > 0;
      float s = 0.f;
      for (d += lane; d < d1; d += 64) s += bt[ahead ? mid + d : mid - d];
      if (after)
        for (int i = mid + 1 + lane; i < nd; i += 64) s += bt[i];
      s = wave_sum(s);
      if (last)
        for (int w = 0; w < NW; ++w) s += far_sum[ahead][w];
      if (after)
        for (int w = 0; w < NW; ++w) s += far_sum[1][w];
      if (lane == 0) share[u] = s;
    }
    __syncthreads();
  }
};

// The whole backward pass of one (sample, key head) whose queries and keys both
// fit in LDS (256 of each at d 64, 128 at d 128), in one launch: a wave takes 32
// rows for dq and delta, then, with the rows' statistics in LDS, 32 keys for dk
// and dv.  A text encoder's prompts are of this size, and three launches one after
// the other cost more than their work (8 x 24 heads x 226 tokens with a position
// bias, d 64, forward and backward: 89 us with them, 51 so, 36 of them here).  What
// bounds it: one workgroup's walk, 16 blocks of 32 keys or rows one after the other
// (waves wait 57% of their time; the vector units issue in 19% of it, the matrix pipe
// works in 8%); 192 such workgroups have a CU each.
template <int D>
constexpr int kSmallWaves = D == 64 ? 8 : 4;
constexpr int kSmallFar = 256;         // the most far with which the sums by diagonal fit as well

// TINY is for up to 64 queries and keys: fewer waves, and P and dS go into their
// products as two values each, since the gradients of a few rows and keys are a few
// hundred values, whose rounding errors may by chance lie well above their mean
// (6 x 8, d 128: dk's 1.7 times the final rounding alone).
constexpr int kTiny = 64;
template <int D>
constexpr int kTinyWaves = D == 64 ? 2 : 4;               // waves load a tile in periods of its row order

template <class T, int D, bool BIAS, bool TINY>
__global__ __launch_bounds__(64 * (TINY ? kTinyWaves<D> : kSmallWaves<D>), D == 64 && !TINY ? 2 : 1) void cross_small_bwd_kernel(
    const CrossParams p) {
  constexpr int NW = TINY ? kTinyWaves<D> : kSmallWaves<D>, NT = 64 * NW, L = 32 * NW, TILES = L / 64;
  __shared__ __attribute__((aligned(1024))) u16 sQ[L * D], sG[L * D], sK[L * D], sV[L * D];
  __shared__ __attribute__((aligned(16))) float st[2][L]; // -LSE / scale and -delta of the rows
  __shared__ float mask[L];                               // 0 or -inf per key
  __shared__ uint16_t start[BIAS ? kMaxBucketSide : 1];
  __shared__ float far_sum[2][NW];
  extern __shared__ __attribute__((aligned(16))) float bt[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;
  const int unit = unit_at(p, xcd_remap(blockIdx.x, p.n_wg), p.Hk), b = unit / p.Hk, hk = unit % p.Hk;
  const int n = key_count(p, b), off = query_offset(p, n), far = BIAS ? p.rb.far : 0;
  const int rw = wave * 32;                               // the wave's first row, and first key
  const int nkb = (n + 31) / 32, nqb = (p.Lq + 31) / 32;

  TileLoad<D, NW> ld;
  auto load = [&](u16* dst, const u16* first, int64_t stride, int count) {
    ld.init(wave, lane, stride);
    for (int t = 0; t < TILES; ++t)
      if (t * 64 < count) ld.issue(__builtin_amdgcn_readfirstlane(lds_addr(dst + t * 64 * D)), first + t * 64 * stride, stride, count - t * 64);
  };
  const u16* kh = p.k + b * p.sk.b + hk * p.sk.h;
  const u16* vh = p.v + b * p.sv.b + hk * p.sv.h;
  load(sK, kh, p.sk.t, n);
  load(sV, vh, p.sv.t, n);
  load(sQ, p.q + b * p.sq.b + hk * p.G * p.sq.h, p.sq.t, p.Lq);
  load(sG, p.dout + b * p.sdo.b + hk * p.G * p.sdo.h, p.sdo.t, p.Lq);
  auto visible = [&](int key) { return key < n && !(p.key_mask && p.key_mask[b * p.mask_stride + key] == 0); };
  if (tid < L) mask[tid] = visible(tid) ? 0.f : -INFINITY;
  TableSums<NW> table(p, bt, far_sum, start, far, wave, lane, tid);
  if (BIAS) table.clear();
  wait_vmem();
  __syncthreads();
  // Whatever the loads have left out or a mask hides is zero.
  for (int i = tid; i < L * (D / 8); i += NT) {
    const int row = i / (D / 8);
    if (mask[row] != 0.f) {
      *reinterpret_cast<u32x4*>(sK + i * 8) = u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4*>(sV + i * 8) = u32x4{0, 0, 0, 0};
    }
    if (row >= p.Lq) {
      *reinterpret_cast<u32x4*>(sQ + i * 8) = u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4*>(sG + i * 8) = u32x4{0, 0, 0, 0};
    }
  }
  __syncthreads();

  const int ra0 = row_lane<D>(c32, hw), ca0 = col_lane<D>(lane);
  const bool key_ok = mask[rw + c32] == 0.f;
  uint32_t whole = 0;                                     // blocks of 32 keys that are all visible
  for (int j = 0; j < nkb; ++j)
    if (__all(mask[32 * j + c32] == 0.f)) whole |= 1u << j;
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f32x16{};
  Spread<T> spread_k;

  for (int g = 0; g < p.G; ++g) {
    const int h = hk * p.G + g;
    if (g > 0) {                                          // the next query head that shares these keys
      load(sQ, p.q + b * p.sq.b + h * p.sq.h, p.sq.t, p.Lq);
      load(sG, p.dout + b * p.sdo.b + h * p.sdo.h, p.sdo.t, p.Lq);
    }
    const RowOf lower = {b, h, rw + (lane & 15)}, upper = {b, h, rw + (lane & 15) + 16};
    const bool a_ok = lower.i < p.Lq, b_ok = upper.i < p.Lq;
    typename T::x8 of[D / 16];
    load_tile<T, D>(at((const u16*)p.out, p.so, lower), a_ok, at((const u16*)p.out, p.so, upper), b_ok, lane, of);
    if (BIAS) fill_bias<T, NT>(bt, start, p, h, tid);
    wait_vmem();
    __syncthreads();

    // dq of rows rw .. rw + 31, put right by sum_j P_ij k_j once the rows' exact
    // delta is known, as in cross_dq_kernel.
    {
      const int i = rw + c32;
      const int64_t row = ((int64_t)b * p.H + h) * p.Lq + i;
      const int ra = fresh(ra0);
      typename T::x8 qf[D / 16], gf[D / 16];
      const float z = i < p.Lq ? p.lse[row] : -INFINITY;
      const float nlse2 = z == -INFINITY ? -INFINITY : -z * kLog2e;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        qf[ks] = read_row<T>(sQ + (ra ^ (8 * row_chunk(ks))) + rw * D);
        gf[ks] = read_row<T>(sG + (ra ^ (8 * row_chunk(ks))) + rw * D);
      }
      float delta = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[ks][e], (float)of[ks][e], delta);
      delta = both_halves_sum(delta);
      int last = rw < p.Lq ? nkb : 0;                     // blocks of keys that some row sees
      if (BIAS && p.rb.causal && rw + 31 + off < 32 * last) last = rw + 31 + off < 0 ? 0 : (rw + 31 + off) / 32 + 1;
      // P and dP - delta of block j.
      auto block = [&](int j, f32x16& x, f32x16& y) {
        const int ra = fresh(ra0);
        const u16* tK = sK + 32 * j * D;
        const u16* tV = sV + 32 * j * D;
        x = f32x16{};
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = -delta;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          x = T::mfma(read_row<T>(tK + (ra ^ (8 * row_chunk(ks)))), qf[ks], x);
          y = T::mfma(read_row<T>(tV + (ra ^ (8 * row_chunk(ks)))), gf[ks], y);
        }
        const int lo = 32 * j - (rw + 31 + off);          // the block's smallest key minus query position
        const float* at = bt + bias_from(lo, far) + far + kPad + 31 + 4 * hw - c32;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = fmaf(x[e], p.sl2, BIAS ? at[8 * (e >> 2) + (e & 3)] + nlse2 : nlse2);
        if (!((whole >> j) & 1)) {
          const float* hide = mask + 32 * j + 4 * hw;
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] += hide[8 * (e >> 2) + (e & 3)];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = fast_exp2(x[e]);
      };
      f32x16 acc[D / 32], pk[D / 32];
#pragma unroll
      for (int d = 0; d < D / 32; ++d) acc[d] = pk[d] = f32x16{};
      float more = 0.f;
      Spread<T> spread;
      for (int j = 0; j < last; ++j) {
        f32x16 x, y;
        block(j, x, y);
        const int ca = fresh(ca0);
        float s0 = 0.f, s1 = 0.f;
        u32x4 w[2], wp[2], wr[2];
        auto put = [&](int e) {
          const uint2 v = split_pair<T>(y[e], y[e + 1]);
          w[e >> 3][(e & 7) >> 1] = v.x;
          if (TINY) wr[e >> 3][(e & 7) >> 1] = v.y;
          wp[e >> 3][(e & 7) >> 1] = T::pack(x[e], x[e + 1]);
        };
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          y[e] *= x[e];
          y[e + 1] *= x[e + 1];
          s0 += y[e];
          s1 += y[e + 1];
          if (!T::kHalf) put(e);
        }
        if (T::kHalf) {
          spread.apply(y, acc);
#pragma unroll
          for (int e = 0; e < 16; e += 2) put(e);
        }
        more += s0 + s1;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            const typename T::x8 kf = read_col<T, D>(sK + 32 * j * D, ca, d, 16 * s);
            acc[d] = T::mfma(kf, __builtin_bit_cast(typename T::x8, w[s]), acc[d]);
            if (TINY) acc[d] = T::mfma(kf, __builtin_bit_cast(typename T::x8, wr[s]), acc[d]);
            pk[d] = T::mfma(kf, __builtin_bit_cast(typename T::x8, wp[s]), pk[d]);
          }
      }
      more = both_halves_sum(more);
      delta += more;
      spread.undo(acc);
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = fmaf(-more, pk[d][e], acc[d][e]);
      if (hw == 0) {
        st[0][i] = nlse2 / p.sl2;                         // past the last row -inf: weight 0
        st[1][i] = -delta;
      }
      store_tile<T, D>(acc, p.scale, at(p.dq, p.sdq, lower), a_ok, at(p.dq, p.sdq, upper), b_ok, lane);
    }
    __syncthreads();

    // dk and dv of keys rw .. rw + 31.
    if (rw < n) {
      const int ra = fresh(ra0);
      typename T::x8 kf[D / 16], vf[D / 16];
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        kf[ks] = read_row<T>(sK + (ra ^ (8 * row_chunk(ks))) + rw * D);
        vf[ks] = read_row<T>(sV + (ra ^ (8 * row_chunk(ks))) + rw * D);
      }
      const int first = BIAS && p.rb.causal && rw - off > 0 ? (rw - off) / 32 : 0;
      for (int i = first; i < nqb; ++i) {
        const int ra = fresh(ra0), ca = fresh(ca0);
        const u16* tQ = sQ + 32 * i * D;
        const u16* tG = sG + 32 * i * D;
        const int lo = rw - (32 * i + 31 + off);
        f32x16 x, y;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] = st[0][32 * i + 8 * (e >> 2) + 4 * hw + (e & 3)];
          y[e] = st[1][32 * i + 8 * (e >> 2) + 4 * hw + (e & 3)];
        }
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          x = T::mfma(read_row<T>(tQ + (ra ^ (8 * row_chunk(ks)))), kf[ks], x);
          y = T::mfma(read_row<T>(tG + (ra ^ (8 * row_chunk(ks)))), vf[ks], y);
        }
        const float* at = bt + bias_entries(far) - 1;     // a masked key's: -inf
        if (BIAS && key_ok) at = bt + bias_from(lo, far) + far + kPad + 31 + c32 - 4 * hw;
        u32x4 wp[2], ws[2], pr[2], sr[2];
        auto put = [&](int e) {
          if (T::kHalf) {
            x[e] *= 1.f / kUnshift<T>;
            x[e + 1] *= 1.f / kUnshift<T>;
          }
          if (TINY) {
            const uint2 v = split_pair<T>(x[e], x[e + 1]), t = split_pair<T>(y[e], y[e + 1]);
            wp[e >> 3][(e & 7) >> 1] = v.x;
            pr[e >> 3][(e & 7) >> 1] = v.y;
            ws[e >> 3][(e & 7) >> 1] = t.x;
            sr[e >> 3][(e & 7) >> 1] = t.y;
          } else {
            wp[e >> 3][(e & 7) >> 1] = T::pack(x[e], x[e + 1]);
            ws[e >> 3][(e & 7) >> 1] = T::pack(y[e], y[e + 1]);
          }
        };
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const int r = 8 * (e >> 2) + (e & 3);
          x[e] = fast_exp2(BIAS ? fmaf(x[e], p.sl2, at[-r]) : x[e] * p.sl2);
          x[e + 1] = fast_exp2(BIAS ? fmaf(x[e + 1], p.sl2, at[-r - 1]) : x[e + 1] * p.sl2);
          y[e] *= x[e];
          y[e + 1] *= x[e + 1];
          if (!T::kHalf) put(e);
        }
        if (BIAS) table.add(y, lo);
        if (T::kHalf) {
          spread_k.apply(y, dk);
#pragma unroll
          for (int e = 0; e < 16; e += 2) put(e);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            const typename T::x8 gc = read_col<T, D>(tG, ca, d, 16 * s), qc = read_col<T, D>(tQ, ca, d, 16 * s);
            dv[d] = T::mfma(gc, __builtin_bit_cast(typename T::x8, wp[s]), dv[d]);
            dk[d] = T::mfma(qc, __builtin_bit_cast(typename T::x8, ws[s]), dk[d]);
            if (TINY) {
              dv[d] = T::mfma(gc, __builtin_bit_cast(typename T::x8, pr[s]), dv[d]);
              dk[d] = T::mfma(qc, __builtin_bit_cast(typename T::x8, sr[s]), dk[d]);
            }
          }
      }
    }
    __syncthreads();
    if (BIAS) table.flush(p, p.part_t + ((int64_t)b * p.H + h) * table.buckets);
  }
  if (!key_ok) {                                          // a masked key took part with a row of zeros
#pragma unroll
    for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f32x16{};
  }
  const RowOf lower = {b, hk, rw + (lane & 15)}, upper = {b, hk, rw + (lane & 15) + 16};
  const bool a_ok = lower.i < p.Lk, b_ok = upper.i < p.Lk;
  store_tile<T, D>(dk, p.scale * spread_k.down, at(p.dk, p.sdk, lower), a_ok, at(p.dk, p.sdk, upper), b_ok, lane);
  store_tile<T, D>(dv, kUnshift<T>, at(p.dv, p.sdv, lower), a_ok, at(p.dv, p.sdv, upper), b_ok, lane);
}

// dk and dv of 32 keys per wave, over one range of the (query head, 64-row
// query tile) items that see them.
//
// Blocks of 32 rows run through three stages: S and dP (MFMA), P and dS (VALU),
// dv and dk (MFMA).  A step works on the first stage of one block, the second
// of the one before and the third of the one before that, so that the matrix
// pipe has work while the VALU does: at d 128 the accumulators leave one wave
// per SIMD, and no other wave would fill the gaps.  Tiles stay in a ring of
// three for it.  What bounds it: the matrix pipe at one wave's pace (24 heads x 110,080
// rows over 256 keys, d 128: 692 GFLOP in 713 us, 971 TFLOP/s, the pipe 50% busy; a
// large product reaches 1,154); under an order mask the first keys' walk, with the
// table's sums by diagonal (12 x 4,095 tokens, d 128, fp16: 170 us).
template <class T, int D, bool BIAS>
__global__ __launch_bounds__(64 * kDkvWaves, D == 64 ? 2 : 1) void cross_dkv_kernel(const CrossParams p) {
  constexpr int NW = kDkvWaves, NT = 64 * NW, KE = 64 * D;
  __shared__ __attribute__((aligned(1024))) u16 ring[3][2 * KE];      // slots [Q | dO]
  __shared__ __attribute__((aligned(16))) float ld[3][2][64];         // -LSE / scale and -delta of their rows
  __shared__ uint16_t start[kMaxBucketSide];
  __shared__ float far_sum[2][NW];
  extern __shared__ __attribute__((aligned(16))) float bt[];          // the bias, then the sums per diagonal
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;

  const int n_kt = (p.Lk + 32 * NW - 1) / (32 * NW);
  const Place place = place_of<BIAS>(p, p.Hk, n_kt, p.kv_splits, false);
  const int unit = place.unit, split = place.split, j0 = place.tile * 32 * NW;
  const int b = unit / p.Hk, hk = unit % p.Hk;
  const int n = key_count(p, b), off = query_offset(p, n);
  const int key = j0 + wave * 32 + c32;
  const bool key_ok = key < n && !(p.key_mask && p.key_mask[b * p.mask_stride + key] == 0);

  const int nqt = (p.Lq + 63) / 64;
  int q_first = 0;                                        // first query tile that sees a key of this tile
  if (BIAS && p.rb.causal) q_first = j0 - off <= 0 ? 0 : (j0 - off) / 64;
  const int per_head = j0 >= n || q_first >= nqt ? 0 : nqt - q_first;
  const int64_t items = (int64_t)per_head * p.G;
  const int i0 = (int)(items * split / p.kv_splits), i1 = (int)(items * (split + 1) / p.kv_splits);

  typename T::x8 kf[D / 16], vf[D / 16];
  // The two keys this lane loads and stores (key is the one it computes).
  const int key_a = j0 + wave * 32 + (lane & 15), key_b = key_a + 16;
  {
    auto visible = [&](int k) { return k < n && !(p.key_mask && p.key_mask[b * p.mask_stride + k] == 0); };
    const bool a_ok = visible(key_a), b_ok = visible(key_b);
    const u16* kh = p.k + b * p.sk.b + hk * p.sk.h;
    const u16* vh = p.v + b * p.sv.b + hk * p.sv.h;
    load_tile<T, D>(kh + (int64_t)key_a * p.sk.t, a_ok, kh + (int64_t)key_b * p.sk.t, b_ok, lane, kf);
    load_tile<T, D>(vh + (int64_t)key_a * p.sv.t, a_ok, vh + (int64_t)key_b * p.sv.t, b_ok, lane, vf);
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f32x16{};

  TileLoad<D, NW> lq, lg;
  lq.init(wave, lane, p.sq.t);
  lg.init(wave, lane, p.sdo.t);
  const int ra0 = row_lane<D>(c32, hw), ca0 = col_lane<D>(lane);
  // The item to be loaded next: its head and first row, and where they are.
  const int q_begin = q_first * 64;
  int in_h = hk * p.G + (per_head > 0 ? i0 / per_head : 0), in_q = (q_first + (per_head > 0 ? i0 % per_head : 0)) * 64;
  const u16* qp = p.q + b * p.sq.b + in_h * p.sq.h + in_q * p.sq.t;
  const u16* gp = p.dout + b * p.sdo.b + in_h * p.sdo.h + in_q * p.sdo.t;
  const int64_t q_step = 64 * p.sq.t, g_step = 64 * p.sdo.t;
  float2 mine = make_float2(0.f, 0.f);
  u32x4 q_buf, g_buf;
  auto prepare = [&]() {
    q_buf = lq.buffer(qp, p.sq.t, p.Lq - in_q);
    g_buf = lg.buffer(gp, p.sdo.t, p.Lq - in_q);
    if (tid < 64) {
      mine = make_float2(-INFINITY, 0.f);                 // past the last row: weight 0
      if (in_q + tid < p.Lq) mine = p.row_ld[((int64_t)b * p.H + in_h) * p.Lq + in_q + tid];
    }
    in_q += 64;
    qp += q_step;
    gp += g_step;
    if (in_q >= p.Lq) {
      in_q = q_begin;
      ++in_h;
      qp = p.q + b * p.sq.b + in_h * p.sq.h + in_q * p.sq.t;
      gp = p.dout + b * p.sdo.b + in_h * p.sdo.h + in_q * p.sdo.t;
    }
  };
  auto slot_addr = [&](int slot) { return (uint32_t)__builtin_amdgcn_readfirstlane(lds_addr(ring[slot])); };
  auto issue = [&](int slot) {
    prepare();
    const uint32_t dst = slot_addr(slot);
    lq.go(q_buf, dst, lq.rel);
    lg.go(g_buf, dst + KE * 2, lg.rel);
  };
  // A tile that ends past the last row leaves those rows of its slot as they
  // were: they have to be numbers, since they meet weights of zero.  So do the
  // blocks before the first and after the last, and their statistics.
  if (tid < 64)
    for (int i = 0; i < 6; ++i) (&ld[0][0][0])[64 * i + tid] = 0.f;
  for (int c = tid; c < 3 * 2 * KE / 8; c += NT) *reinterpret_cast<u32x4*>(&ring[0][0] + c * 8) = u32x4{0, 0, 0, 0};
  __syncthreads();
  const int far = BIAS ? p.rb.far : 0;
  TableSums<NW> table(p, bt, far_sum, start, far, wave, lane, tid);
  int head = 0;
  // The head that the workgroup leaves: its share of dtable.
  auto flush = [&]() {
    table.flush(p, p.part_t + ((((int64_t)b * p.H + hk * p.G + head) * n_kt + j0 / (32 * NW)) * p.kv_splits + split) *
                                  table.buckets);
    ++head;
  };
  f32x16 x, y;                                            // S and dP of the block in the second stage
  Spread<T> spread;
  typename T::x8 pf[2], sf[2];                            // P and dS of the one in the third
#pragma unroll
  for (int s = 0; s < 2; ++s) pf[s] = sf[s] = typename T::x8{};
  // The first stage's sums begin at the rows' -LSE / scale and -delta, so that
  // the second finds S - LSE / scale and dP - delta.
  auto begin = [&](const float* st, f32x16& xn, f32x16& yn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(st + 8 * i + 4 * hw);
      const f32x4 c = *reinterpret_cast<const f32x4*>(st + 64 + 8 * i + 4 * hw);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        xn[4 * i + j] = a[j];
        yn[4 * i + j] = c[j];
      }
    }
  };
  auto first = [&](const u16* tile, const float* st, int ra, f32x16& xn, f32x16& yn) {
    begin(st, xn, yn);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      xn = T::mfma(read_row<T>(tile + (ra ^ (8 * row_chunk(ks)))), kf[ks], xn);
      yn = T::mfma(read_row<T>(tile + KE + (ra ^ (8 * row_chunk(ks)))), vf[ks], yn);
    }
  };
  auto third = [&](const u16* tile, int g, int ca) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        dv[d] = T::mfma(read_col<T, D>(tile + KE, ca, d, 32 * g + 16 * s), pf[s], dv[d]);
        dk[d] = T::mfma(read_col<T, D>(tile, ca, d, 32 * g + 16 * s), sf[s], dk[d]);
      }
  };
  // One step: block (next, gn) in the first stage, with its rows' statistics st,
  // the one whose smallest key minus query position is lo in the second, block
  // (prev, gp) in the third.
  auto step = [&](auto&& hook, const u16* next, int gn, const float* st, const u16* prev, int gp, int lo) {
    constexpr int NM = D / 4;                             // slots, one MFMA each: first and third stage in turn
    constexpr int LA = D == 64 ? 2 : 4;                                 // slots between an operand's read and its use
    constexpr int PER = NM / 8;                           // slots per pair of rows of the second stage
    // At d 128 registers are there for the lanes' addresses.
    const int ra = (D == 64 ? fresh(ra0) : ra0) , ca = D == 64 ? fresh(ca0) : ca0;
    f32x16 xn, yn;
    begin(st, xn, yn);
    typename T::x8 op[NM];
    auto fetch = [&](int i) {
      const int j = i >> 1;
      if ((i & 1) == 0) {
        op[i] = read_row<T>(next + (j & 1) * KE + 32 * gn * D + (ra ^ (8 * row_chunk(j >> 1))));
      } else {
        const int s = j / (D / 16), d = j % (D / 16) >> 1;
        op[i] = read_col<T, D>(prev + ((j & 1) ? 0 : KE), ca, d, 32 * gp + 16 * s);
      }
    };
    auto mfma = [&](int i) {
      const int j = i >> 1;
      if ((i & 1) == 0) {
        if (j & 1) yn = T::mfma(op[i], vf[j >> 1], yn);
        else xn = T::mfma(op[i], kf[j >> 1], xn);
      } else {
        const int s = j / (D / 16), d = j % (D / 16) >> 1;
        if (j & 1) dk[d] = T::mfma(op[i], sf[s], dk[d]);
        else dv[d] = T::mfma(op[i], pf[s], dv[d]);
      }
    };
    const float* at = bt + bias_entries(far) - 1;         // a masked key's: -inf
    if (BIAS && key_ok) at = bt + bias_from(lo, far) + far + kPad + 31 + c32 - 4 * hw;
    // Second stage, pair u: rows r and r + 1 of 8 (e / 4) + 4 hw + e % 4.
    float bias[16], arg[16];
    u32x4 wp[2], ws[2];
    auto biases = [&](int u) {
      const int e = 2 * u, r = 8 * (e >> 2) + (e & 3);
      if (BIAS) {
        bias[e] = at[-r];
        bias[e + 1] = at[-r - 1];
      }
    };
    auto stage_arg = [&](int u) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        arg[2 * u + k] = fmaf(x[2 * u + k], p.sl2, BIAS ? bias[2 * u + k] : kShift<T>);
        pin(arg[2 * u + k]);
      }
    };
    auto stage_exp = [&](int u) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        arg[2 * u + k] = fast_exp2(arg[2 * u + k]);
        pin(arg[2 * u + k]);
      }
    };
    // fp16: y becomes dS with the factor that it enters its product with, or, where the
    // table's gradient takes it too, without.
    const float factor = kUnshift<T> * (BIAS ? 1.f : spread.up), later = BIAS ? spread.up : 1.f;
    float most = 0.f;
    auto stage_ds = [&](int u) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float v = arg[2 * u + k] * y[2 * u + k];
        if (T::kHalf) v *= factor;
        pin(v);
        y[2 * u + k] = v;
      }
    };
    auto stage_pack = [&](int u) {
      uint32_t a = T::pack(arg[2 * u], arg[2 * u + 1]), c;
      if constexpr (T::kHalf && BIAS) c = T::pack(y[2 * u] * later, y[2 * u + 1] * later);
      else c = T::pack(y[2 * u], y[2 * u + 1]);
      asm volatile("" : "+v"(a), "+v"(c));
      wp[u >> 2][u & 3] = a;
      ws[u >> 2][u & 3] = c;
      if (T::kHalf) most = vmax(most, vmax(__builtin_fabsf(y[2 * u]), __builtin_fabsf(y[2 * u + 1])));
    };
    biases(0);
#pragma unroll
    for (int i = 0; i < LA; ++i) fetch(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      const int u = i / PER, ph = i % PER;
      if (i + LA < NM) fetch(i + LA);
      if (ph == 0 && u + 1 < 8) biases(u + 1);
      mfma(i);
      hook(i);
      if (ph == 0) stage_arg(u);
      if (ph == 0 && u > 0 && PER == 2) stage_ds(u - 1);
      if (ph == 1) stage_exp(u);
      if (ph == 1 && u > 0 && PER == 2) stage_pack(u - 1);
      if (ph == 2) stage_ds(u);
      if (ph == 3) stage_pack(u);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (PER == 2) {
      stage_ds(7);
      stage_pack(7);
    }
    if (BIAS) table.add(y, lo);
    if constexpr (T::kHalf) {
      // The third stage has by now added up all that was packed with the factor so far.
      most *= later;
      if (__any(spread.over(most))) {
        const float by = spread.lower(most, dk) * later;
#pragma unroll
        for (int u = 0; u < 8; ++u) ws[u >> 2][u & 3] = T::pack(y[2 * u] * by, y[2 * u + 1] * by);
      }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      pf[s] = __builtin_bit_cast(typename T::x8, wp[s]);
      sf[s] = __builtin_bit_cast(typename T::x8, ws[s]);
    }
    x = xn;
    y = yn;
  };
  auto put = [&](int slot) {
    if (tid < 64) {
      ld[slot][0][tid] = mine.x;
      ld[slot][1][tid] = mine.y;
    }
  };
  if (i0 < i1) issue(0);
  if (BIAS) {
    table.clear();
    fill_bias<T, NT>(bt, start, p, hk * p.G, tid, kShift<T>);
  }
  int q0 = in_q, g_head = in_h - hk * p.G;                // of the current item
  if (i0 < i1) {
    q0 = (q_first + i0 % per_head) * 64;
    g_head = i0 / per_head;
    put(0);
    if (i0 + 1 < i1) issue(1);
    wait_vmem();
    if (i0 + 1 < i1) put(1);
    __syncthreads();
    first(ring[0], ld[0][0], ra0, x, y);
  }
  int slot = 0;                                           // of this item's tile
  for (int it = i0; it < i1; ++it) {
    if (BIAS && g_head != head) {                         // another query head: its own bias
      __syncthreads();
      while (head < g_head) flush();
      fill_bias<T, NT>(bt, start, p, hk * p.G + g_head, tid, kShift<T>);
      __syncthreads();
    }
    const int after = slot == 2 ? 0 : slot + 1, before = slot == 0 ? 2 : slot - 1;
    const int lo = j0 + wave * 32 - (q0 + 31 + off);
    step([](int) {}, ring[slot], 1, ld[slot][0] + 32, ring[before], 1, lo);
    wait_vmem();
    if (it > i0 && it + 1 < i1) put(after);
    __syncthreads();
    // The tile after the next goes to the slot that the first step was the last
    // to read, one load per slot of the second step.
    const bool more = it + 2 < i1;
    if (more) prepare();
    const uint32_t dst = slot_addr(before);
    step(
        [&](int i) {
          constexpr int PL = TileLoad<D, NW>::PER;
          if (i < 2 * PL && more) {
            if (i < PL) lq.issue_n(i, dst, q_buf);
            else lg.issue_n(i - PL, dst + KE * 2, g_buf);
          }
        },
        ring[after], 0, ld[after][0], ring[slot], 0, lo - 32);
    slot = after;
    q0 += 64;
    if (q0 >= p.Lq) {
      q0 = q_begin;
      ++g_head;
    }
  }
  if (i0 < i1) third(ring[slot == 0 ? 2 : slot - 1], 1, ca0);
  if (BIAS) {
    __syncthreads();
    while (head < p.G) flush();
  }
  // A masked key took part with a row of zeros: its sums are dropped.
  if (!key_ok) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f32x16{};
  }
  spread.undo(dk);
  const bool ok = key < p.Lk;
  if (p.kv_splits > 1) {
    const int64_t all = (int64_t)p.B * p.Hk * p.Lk, at = (int64_t)unit * p.Lk + key;
    store_tile_f32<D>(dk, p.part_kv + ((2 * split) * all + at) * D, ok, hw);
    store_tile_f32<D>(dv, p.part_kv + ((2 * split + 1) * all + at) * D, ok, hw);
    return;
  }
  u16* dkh = p.dk + b * p.sdk.b + hk * p.sdk.h;
  u16* dvh = p.dv + b * p.sdv.b + hk * p.sdv.h;
  const bool a_in = key_a < p.Lk, b_in = key_b < p.Lk;
  store_tile<T, D>(dk, p.scale, dkh + (int64_t)key_a * p.sdk.t, a_in, dkh + (int64_t)key_b * p.sdk.t, b_in, lane);
  store_tile<T, D>(dv, kUnshift<T>, dvh + (int64_t)key_a * p.sdv.t, a_in, dvh + (int64_t)key_b * p.sdv.t, b_in, lane);
}

// Rows of a result from the splits' partial rows, added in order.  Two results
// (dk and dv) side by side in one launch: blockIdx.y chooses.  Bound by its bytes, of
// which L2 holds a part (101 MB of dk's and dv's partial rows of the long video: 18 us).
struct SumOf {
  const float* part;
  u16* out;
  Strides so;
  float scale;
};
template <class T, int D>
__global__ __launch_bounds__(256) void cross_sum_kernel(SumOf first, SumOf second, int64_t stride, int splits,
                                                        int64_t rows, int heads, int len) {
  constexpr int TPR = D / 4;
  const SumOf& s = blockIdx.y == 0 ? first : second;
  const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (row >= rows) return;
  const int c = threadIdx.x % TPR * 4;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < splits; ++i) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(s.part + i * stride + row * D + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += v[j];
  }
  const RowOf r = {(int)(row / len / heads), (int)(row / len % heads), (int)(row % len)};
  uint2 w;
  w.x = T::pack(o[0] * s.scale, o[1] * s.scale);
  w.y = T::pack(o[2] * s.scale, o[3] * s.scale);
  *reinterpret_cast<uint2*>(at(s.out, s.so, r) + c) = w;
}

// dtable[u, h]: the shares of head h over samples and workgroups, 64 runs of them
// for four buckets at a time, each in order, then the runs' sums in order.  A chain of
// loads: 4.6 us for 32 shares of 64 buckets as for 8 of 32.
template <class T>
__global__ __launch_bounds__(256) void cross_dtable_kernel(const CrossParams p, int per) {
  __shared__ float sum[64][4];
  const int h = blockIdx.x, buckets = p.rb.both ? 2 * p.rb.side : p.rb.side;
  const int t = threadIdx.x & 3, u = blockIdx.y * 4 + t, part = threadIdx.x >> 2;
  float s = 0.f;
  if (u < buckets) {
    const int64_t n = (int64_t)p.B * per;
#pragma unroll 4
    for (int64_t a = n * part / 64; a < n * (part + 1) / 64; ++a)
      s += p.part_t[((a / per * p.H + h) * per + a % per) * buckets + u];
  }
  sum[part][t] = s;
  __syncthreads();
  if (part != 0 || u >= buckets) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 64; ++i) s += sum[i][t];
  const int64_t at = (int64_t)u * p.H + h;
  if (p.rb.table_f32) ((float*)p.rb.dtable)[at] = s;
  else T::store(p.rb.dtable, at, s);
}

namespace {
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
int64_t row_tiles(const CrossParams& p, bool bias) {
  return ((bias ? p.Lq : (int64_t)p.G * p.Lq) + kDqRows - 1) / kDqRows;
}
int clamp_splits(int64_t s, int64_t most) {
  s = s < most ? s : most;
  return s < 1 ? 1 : (s > 128 ? 128 : (int)s);
}
}  // namespace

CrossPlan plan_bwd(const CrossParams& p, int D, bool bias) {
  CrossPlan c{};
  const int64_t units = (int64_t)p.B * (bias ? p.H : p.Hk), tiles = units * row_tiles(p, bias);
  const int64_t nt = (p.Lk + 63) / 64;
  const int fit = 32 * (D == 64 ? kSmallWaves<64> : kSmallWaves<128>);
  c.small = p.Lq > 0 && p.Lq <= fit && p.Lk <= fit && (!bias || p.rb.far <= kSmallFar);
  if (c.small) {
    c.splits = c.kv_splits = 1;
    c.bytes = bias ? up256((int64_t)p.B * p.H * (p.rb.both ? 2 : 1) * p.rb.side * 4) : 0;
    return c;
  }
  // Split keys cost a pass for delta and a sum, so only for few rows: whole calls
  // whole against split, us: 200 tiles of d 64 x 49 key tiles 233 and 254 (in two),
  // 192 of d 128 x 15 116 and 141, 64 of d 64 x 63 163 and 126, 16 x 286 567 and
  // 128, 24 of d 128 x 24 83 and 69, 24 of d 64 x 11 75 and 83.
  c.splits = tiles > 0 && tiles <= 96 && nt > 12 ? clamp_splits(512 / tiles, nt / 4) : 1;
  c.resident = keep_keys(p, D, bias, 1);
  if (c.resident) c.splits = keep_chunks(p, 1);
  // dq shrinks with the square root of the number of keys, what an error of delta
  // puts into it does not (sum_j P_ij k_j leans towards q_i): where no correction sum
  // follows (d 128), long walks have their delta formed first as well.  dq's error, in
  // units of its final rounding, with delta from the output: 1.3 at 2,245 keys, 3.6 at
  // 49,836; 1.4 so, at one product in five more.  What counts is how many keys a row can
  // see, the last row's where there is an order: 110 heads of 5 rows that end with 4,095
  // keys, values with a mean of half their spread, 1.9 and 1.4.
  int64_t seen = p.Lk;
  if (bias && p.rb.causal && !p.rb.at_end) seen = (int64_t)p.Lq + p.rb.q_offset < seen ? (int64_t)p.Lq + p.rb.q_offset : seen;
  constexpr int64_t kLong = 32 * 64;
  c.delta_first = !c.resident && (c.splits > 1 || (D == 128 && seen > kLong));
  const int64_t ktiles = (int64_t)p.B * p.Hk * ((p.Lk + 32 * kDkvWaves - 1) / (32 * kDkvWaves));
  const int64_t items = (int64_t)p.G * ((p.Lq + 63) / 64);
  // Ranges of the queries: rounds of as many workgroups as run at a time (two
  // per CU at d 64, one at d 128), each item about 1.2 or 2.3 us and three more
  // for a workgroup's start and end, and the partial sums' way through memory.
  const double item = D == 64 ? 1.2 : 2.3, at_once = D == 64 ? 512 : 256;
  double best = 0;
  c.kv_splits = 1;
  // (With an order mask the workgroups' lengths differ, and rounds do not end
  // together: 384 of 12 heads x 4,095 tokens are faster whole, 216 us for 256.)
  const int64_t most = bias && p.rb.causal && ktiles >= 256 ? 1 : 128;
  for (int64_t n = 1; n <= most && (n == 1 || n * 2 <= items); ++n) {
    const double rounds = (double)((int64_t)((ktiles * n + at_once - 1) / at_once)), per = (double)((items + n - 1) / n);
    const double cost = rounds * (per + 3) * item + (n > 1 ? 8 + n * ((double)p.B * p.Hk * p.Lk * D * 16 / 4.8e6) : 0);
    if (n == 1 || cost < best) {
      best = cost;
      c.kv_splits = (int)n;
    }
  }
  const int64_t rows = (int64_t)p.B * p.H * p.Lq;
  int64_t off = up256(rows * 8);                     // row_ld at 0
  c.part_o = off;
  if (c.splits > 1 && !c.resident) off += up256(c.splits * rows * D * 4);
  c.part_d = off;
  // (Room by the keys alone: sizes are asked for without an offset.)
  if (!c.resident && (c.splits > 1 || (D == 128 && p.Lk > kLong))) off += up256(c.splits * rows * 4);
  c.part_kv = off;
  if (c.kv_splits > 1) off += up256((int64_t)c.kv_splits * 2 * p.B * p.Hk * p.Lk * D * 4);
  c.part_t = off;
  if (bias) off += up256(ktiles * p.G * c.kv_splits * (p.rb.both ? 2 : 1) * p.rb.side * 4);
  c.bytes = off;
  return c;
}

template <class T, int D, int PASS>
static void launch_dq(const CrossParams& p, bool bias, uint32_t lds, hipStream_t st) {
  if (bias) hipLaunchKernelGGL((cross_dq_kernel<T, D, true, PASS>), dim3(p.n_wg), dim3(256), lds, st, p);
  else hipLaunchKernelGGL((cross_dq_kernel<T, D, false, PASS>), dim3(p.n_wg), dim3(256), 0, st, p);
}

template <class T, int D, bool TINY>
static void launch_small(const CrossParams& p, bool bias, uint32_t lds, hipStream_t st) {
  constexpr int NW = TINY ? kTinyWaves<D> : kSmallWaves<D>;
  if (bias) hipLaunchKernelGGL((cross_small_bwd_kernel<T, D, true, TINY>), dim3(p.n_wg), dim3(64 * NW),
                               lds + NW * diag_entries(p.rb.far) * 4, st, p);
  else hipLaunchKernelGGL((cross_small_bwd_kernel<T, D, false, TINY>), dim3(p.n_wg), dim3(64 * NW), 0, st, p);
}

template <class T, int D>
static hipError_t run_bwd(CrossParams p, bool bias, const CrossPlan& c, hipStream_t st) {
  p.splits = c.splits;
  p.kv_splits = c.kv_splits;
  const int64_t units = (int64_t)p.B * (bias ? p.H : p.Hk), rt = row_tiles(p, bias);
  const int64_t rows = (int64_t)p.B * p.H * p.Lq, keys = (int64_t)p.B * p.Hk * p.Lk;
  const uint32_t lds = bias ? bias_entries(p.rb.far) * 4 : 0, per = 256 / (D / 4);
  const int buckets = p.rb.both ? 2 * p.rb.side : p.rb.side;
  const dim3 table(p.H, (buckets + 3) / 4);
  if (c.small) {
    p.n_wg = p.B * p.Hk;
    if (p.n_wg > 0 && p.Lq <= kTiny && p.Lk <= kTiny) launch_small<T, D, true>(p, bias, lds, st);
    else if (p.n_wg > 0) launch_small<T, D, false>(p, bias, lds, st);
    if (bias) hipLaunchKernelGGL((cross_dtable_kernel<T>), table, dim3(256), 0, st, p, 1);
    return hipGetLastError();
  }
  p.n_wg = (int)(units * (c.resident ? 1 : rt) * p.splits);
  if (c.resident) {
    const dim3 grid(p.n_wg), block(64 * kKeepWaves);
    if (p.Lk <= 32 * kTwiceBlocks<D>) hipLaunchKernelGGL((cross_keep_dq_kernel<T, D, true>), grid, block, keep_lds_bytes(p.Lk), st, p);
    else hipLaunchKernelGGL((cross_keep_dq_kernel<T, D, false>), grid, block, keep_lds_bytes(p.Lk), st, p);
  } else if (p.n_wg > 0) {
    if (c.delta_first) {
      launch_dq<T, D, DELTA>(p, bias, lds, st);
      launch_dq<T, D, DQ>(p, bias, lds, st);
    } else {
      launch_dq<T, D, WHOLE>(p, bias, lds, st);
    }
    if (p.splits > 1) {
      const SumOf dq = {p.part_o, p.dq, p.sdq, p.scale};
      hipLaunchKernelGGL((cross_sum_kernel<T, D>), dim3((uint32_t)((rows + per - 1) / per)), dim3(256), 0, st, dq, dq,
                         rows * D, p.splits, rows, p.H, p.Lq);
    }
  }
  p.n_wg = (int)((int64_t)p.B * p.Hk * ((p.Lk + 32 * kDkvWaves - 1) / (32 * kDkvWaves)) * p.kv_splits);
  if (p.n_wg > 0) {
    if (bias) hipLaunchKernelGGL((cross_dkv_kernel<T, D, true>), dim3(p.n_wg), dim3(64 * kDkvWaves),
                                 lds + kDkvWaves * diag_entries(p.rb.far) * 4, st, p);
    else hipLaunchKernelGGL((cross_dkv_kernel<T, D, false>), dim3(p.n_wg), dim3(64 * kDkvWaves), 0, st, p);
    const SumOf dk = {p.part_kv, p.dk, p.sdk, p.scale}, dv = {p.part_kv + keys * D, p.dv, p.sdv, kUnshift<T>};
    if (p.kv_splits > 1)
      hipLaunchKernelGGL((cross_sum_kernel<T, D>), dim3((uint32_t)((keys + per - 1) / per), 2), dim3(256), 0, st, dk, dv,
                         2 * keys * D, p.kv_splits, keys, p.Hk, p.Lk);
  }
  if (bias)
    hipLaunchKernelGGL((cross_dtable_kernel<T>), table, dim3(256), 0, st, p,
                       (int)((p.Lk + 32 * kDkvWaves - 1) / (32 * kDkvWaves) * p.kv_splits));
  return hipGetLastError();
}

hipError_t launch_cross_bwd(CrossParams p, int D, bool f16, bool bias, const CrossPlan& c, hipStream_t st) {
  if (D == 64) return f16 ? run_bwd<FP16, 64>(p, bias, c, st) : run_bwd<BF16, 64>(p, bias, c, st);
  return f16 ? run_bwd<FP16, 128>(p, bias, c, st) : run_bwd<BF16, 128>(p, bias, c, st);
}

}  // namespace adaspa
