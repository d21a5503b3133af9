// Forward attention of queries over keys of another length, with an optional
// learned relative position bias (gfx950).
//
//   out_i = sum_j exp(S_ij - lse_i) v_j,  lse_i = log sum_j exp(S_ij),
//   S_ij = scale q_i . k_j (+ bias[bucket(j - i - offset), h])
//
// over the visible keys of the sample; a row without any gives 0 and -inf.
#include "cross_tile.hpp"

namespace adaspa {

namespace {

constexpr int kRows = 128;             // query rows of a workgroup: four waves of 32
// Weights against a row's maximum go down to e^-18 and less where one key stands out,
// and fp16's smallest step is 2^-24.  So in fp16 they carry 2^kLift (the reference is
// that far below the maximum), which leaves a factor of 32 up to kSumLimit: 100,000 keys
// of unit-variance scores beside one at 16 whose value is 0 had an output off by 2.5e-3
// of its size, and with one at 18 by 0.23; now by the roundings alone.  It is divided out
// with the sum of the weights.  References move more often, which costs 2.5% under a bias
// (12 x 8,191 tokens, d 64: 266 and 272 us) and nothing measurable without.
template <class T>
constexpr float kLift = T::kHalf ? 10.f : 0.f;
// A lane's weights of one tile add up to no more, or the reference moves.
template <class T>
constexpr float kSumLimit = T::kHalf ? 32768.f : 256.f;

// Running softmax of the rows of a wave (lane = row c32, the two half-waves
// hold its keys between them).  Weights are taken against a reference m (log2
// units): the maximum of a row's first tile (less kLift), then whatever it is until the
// weights of a tile, summed over one lane's 32 keys, pass kSumLimit; only then
// is the maximum looked for, the reference moved there and the tile's weights
// taken again.  So no weight exceeds kSumLimit, which fp16 holds too, and most tiles
// need neither a maximum nor a rescaled accumulator.
// They enter the product with V in the inputs' type, which is what the matrix pipe
// takes, and their fp32 sum before that.  Each is off by half a step of its own, so the
// output's error is between its final rounding alone (values with a mean) and 1.4 times
// that (values without one, weights that hardly differ); two values per weight would
// take the product twice.
template <class T, int D, int G = 2>
struct Rows {
  f32x16 o[D / 32];
  float m, l;
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};
    m = -INFINITY;
    l = 0.f;
  }
  // Weights of G times 32 scores (sl2 x in log2 units), returns this lane's sum.
  __device__ __forceinline__ float weights(const f32x16 (&x)[G], float sl2, typename T::x8 (&pb)[G][2]) const {
    const float ref = m == -INFINITY ? 0.f : -m;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      u32x4 w[2];
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float a = fast_exp2(fmaf(x[g][e], sl2, ref)), b = fast_exp2(fmaf(x[g][e + 1], sl2, ref));
        s0 += a;
        s1 += b;
        w[e >> 3][(e & 7) >> 1] = T::pack(a, b);
      }
      pb[g][0] = __builtin_bit_cast(typename T::x8, w[0]);
      pb[g][1] = __builtin_bit_cast(typename T::x8, w[1]);
    }
    return s0 + s1;
  }
  // Moves the reference of the rows that need it to the maximum where that is
  // above it.  (In the first tile there is nothing yet to rescale.)
  __device__ __forceinline__ void raise(const f32x16 (&x)[G], float sl2, bool first, bool need) {
    float mt = -INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 16; e += 2) mt = vmax(mt, vmax(x[g][e], x[g][e + 1]));
    mt = both_halves_max(mt) * sl2;
    if (T::kHalf) mt -= kLift<T>;
    const bool move = need && !(mt <= m);                  // also where it is NaN: the row becomes NaN
    const float a = move ? fast_exp2(m - mt) : 1.f;
    if (move) m = mt;
    if (first) return;
    l *= a;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] *= a;
  }
  // Scores of the keys: weights into pb, their fp32 sum into l.  first: of the
  // first tile, whose rows have no reference yet.
  __device__ __forceinline__ void weigh(const f32x16 (&x)[G], float sl2, typename T::x8 (&pb)[G][2], bool first) {
    if (first) raise(x, sl2, true, true);
    float s = weights(x, sl2, pb);
    // A row that has seen no key yet has no reference either.  Whether a row
    // moves is its own matter, so that its bits do not follow its neighbours.
    if (!first) {
      const float most = both_halves_max(s);
      const bool need = !(most <= kSumLimit<T>) || m == -INFINITY;
      if (__any(need)) {
        raise(x, sl2, false, need);
        s = weights(x, sl2, pb);
      }
    }
    l += s;
  }
};

}  // namespace

// Workgroup: 128 query rows of one unit over one range of its keys, 64-key
// tiles through two slots in LDS, one on its way while the other is used.  What
// bounds it: one row over long keys at d 128, HBM (4 samples of 4 key heads, 17,664
// keys: 145 MB in 24 us, and the join 4); many rows, products and weights that two
// or three waves per SIMD overlap only in part (24 x 256 rows over 110,080 keys,
// d 128: 346 GFLOP in 399 us, matrix pipe 46% busy and vector units 34%; 12 x 8,191
// at d 64 with a bias: 206 GFLOP in 237 us, 38% and 63%).
template <class T, int D, bool BIAS>
__global__ __launch_bounds__(256, 2) void cross_fwd_kernel(const CrossParams p) {
  constexpr int NW = 4, KE = 64 * D;
  __shared__ __attribute__((aligned(1024))) u16 ring[2][2 * KE];
  __shared__ uint16_t start[BIAS ? kMaxBucketSide : 1];
  extern __shared__ __attribute__((aligned(16))) float bt[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;

  const int n_rows = BIAS ? p.Lq : p.G * p.Lq, n_rt = (n_rows + kRows - 1) / kRows;
  const Place place = place_of<BIAS>(p, BIAS ? p.H : p.Hk, n_rt, p.splits, true);
  const int unit = place.unit, split = place.split, r0 = place.tile * kRows;
  const int rw = r0 + wave * 32, r = rw + c32;           // first row of the wave, row of the lane
  const bool row_ok = r < n_rows;
  const RowOf ro = row_of<BIAS>(p, unit, row_ok ? r : 0);
  const int b = BIAS ? unit / p.H : unit / p.Hk, hk = BIAS ? (unit % p.H) / p.G : unit % p.Hk;
  const int n = key_count(p, b), off = query_offset(p, n);

  int kend = n;
  if (BIAS && p.rb.causal) {
    const int64_t last = (int64_t)(r0 + kRows < n_rows ? r0 + kRows : n_rows) + off;   // past the last visible key
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
  if (t0 < t1) issue(integral_constant<int, 0>{}, t0);
  typename T::x8 qf[D / 16];
  const TwoRows two = two_rows<BIAS>(p, unit, rw, n_rows, lane);
  load_tile<T, D>(at(p.q, p.sq, two.a), two.a_ok, at(p.q, p.sq, two.b), two.b_ok, lane, qf);
  if (BIAS) fill_bias<T, 256>(bt, start, p, unit % p.H, tid);

  Rows<T, D> acc;
  acc.init();
  // This lane's places in slot 0; the slots lie at constant distances.
  const u16* kp[D / 16];
  const u16* vp[D / 32][2];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) kp[ks] = ring[0] + (row_lane<D>(c32, hw) ^ (8 * row_chunk(ks)));
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int h = 0; h < 2; ++h) vp[d][h] = ring[0] + KE + (col_lane<D>(lane) ^ (16 * h) ^ (32 * d));
  // Key minus query position of this lane's first key of tile 0.
  const int rel0 = 4 * hw - (ro.i + off);

  auto tile = [&](auto u, int t) {
    wait_vmem();
    const uint64_t keep = below(t * 64, n) & (p.key_mask ? __ballot(mb[u] != 0) : ~0ull);
    __syncthreads();
    if (t + 1 < t1) issue(integral_constant<int, 1 - u>{}, t + 1);
    if (keep != ~0ull) {
      if (keep == 0) return;
      clear_rows<D, 256>(ring[u] + KE, keep, fresh(tid));
      __syncthreads();
    }
    // A wave without rows, or whose rows come before all of these keys.
    if (rw >= n_rows || (BIAS && p.rb.causal && t * 64 > rw + 31 + off)) return;
    f32x16 x[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      x[g] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        x[g] = T::mfma(read_row<T>(kp[ks] + u * 2 * KE + 32 * g * D), qf[ks], x[g]);
    }
    if (BIAS) {
      const int far = p.rb.far, lo = t * 64 - (rw + 31 + off), hi = t * 64 + 63 - (rw + off);
      if (lo >= far || hi <= -far) {
        const float c = bt[lo >= far ? 2 * (far + kPad) : 0];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[g][e] = fmaf(x[g][e], p.sl2, c);
      } else {
        const float* at = bt + (row_ok ? rel0 + t * 64 : lo) + far + kPad;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[g][e] = fmaf(x[g][e], p.sl2, at[32 * g + 8 * (e >> 2) + (e & 3)]);
      }
    }
    if (keep != ~0ull) {
      const uint64_t mine = keep >> (4 * hw);
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!((mine >> (32 * g + 8 * (e >> 2) + (e & 3))) & 1)) x[g][e] = -INFINITY;
    }
    typename T::x8 pb[2][2];
    acc.weigh(x, BIAS ? 1.f : p.sl2, pb, t == t0);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int row = u * 128 + 16 * s;                  // a slot is two tiles of 64 rows
        acc.o[d] = T::mfma(read_cols<T>(vp[d][0] + row * D, vp[d][1] + (row + 8) * D), pb[s >> 1][s & 1], acc.o[d]);
      }
  };
  for (int t = t0; t < t1; t += 2) {
    tile(integral_constant<int, 0>{}, t);
    if (t + 1 < t1) tile(integral_constant<int, 1>{}, t + 1);
  }

  const float l = both_halves_sum(acc.l);
  const int64_t row = ((int64_t)ro.b * p.H + ro.h) * p.Lq + ro.i;
  if (p.splits > 1) {
    const int64_t at = (int64_t)split * p.B * p.H * p.Lq + row;
    store_tile_f32<D>(acc.o, p.part_o + at * D, row_ok, hw);
    if (row_ok && hw == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(acc.m, l);
    return;
  }
  store_tile<T, D>(acc.o, l == 0.f ? 0.f : 1.f / l, at(p.out, p.so, two.a), two.a_ok, at(p.out, p.so, two.b), two.b_ok,
                   lane);
  if (p.lse && row_ok && hw == 0) p.lse[row] = l == 0.f ? -INFINITY : (acc.m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Up to 32 rows at d 64: every wave takes the rows over blocks of 32 keys of its own,
// every fourth, with slots of its own in LDS and no barrier before the waves' sums
// are joined.  (With the tiles of cross_fwd_kernel one wave of four has the rows, and
// its walk, not HBM, bounds the call: one token of 16 x 24 heads over up to 2,049 keys
// with a bias, 143 MB, 40.5 us and so 33.6, new inputs each call; 20 rows of 48 heads
// over 100,000 keys 323 and 218.)  d 128 keeps cross_fwd_kernel: its slots would take
// all of LDS, and it reads at 5.9 TB/s there.
template <class T, int D, bool BIAS>
__global__ __launch_bounds__(256, 2) void cross_few_kernel(const CrossParams p) {
  constexpr int NW = 4, KE = 32 * D, CPR = D / 8, RPI = 64 / CPR;
  static_assert(RPI == 8, "two loads a period of the row order");
  __shared__ __attribute__((aligned(1024))) u16 ring[NW][2][2 * KE];   // per wave: slots [K | V]
  __shared__ float sm[NW][32], sl[NW][32];
  __shared__ uint16_t start[BIAS ? kMaxBucketSide : 1];
  extern __shared__ __attribute__((aligned(16))) float bt[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;

  const int n_rows = BIAS ? p.Lq : p.G * p.Lq;
  const Place place = place_of<BIAS>(p, BIAS ? p.H : p.Hk, 1, p.splits, true);
  const int unit = place.unit, split = place.split;
  const int b = BIAS ? unit / p.H : unit / p.Hk, hk = BIAS ? (unit % p.H) / p.G : unit % p.Hk;
  const int n = key_count(p, b), off = query_offset(p, n), far = BIAS ? p.rb.far : 0;
  int kend = n;
  if (BIAS && p.rb.causal) {
    const int64_t last = (int64_t)n_rows + off;          // past the last visible key
    kend = last < kend ? (last < 0 ? 0 : (int)last) : kend;
  }
  const int nb = (kend + 31) / 32;
  const int b0 = (int)((int64_t)nb * split / p.splits) + wave, b1 = (int)((int64_t)nb * (split + 1) / p.splits);

  const u16* kh = p.k + b * p.sk.b + hk * p.sk.h;
  const u16* vh = p.v + b * p.sv.b + hk * p.sv.h;
  uint32_t krel[2], vrel[2];                             // this lane's place in rows 0-7 and 8-15
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = 8 * j + lane / CPR, chunk = ((lane % CPR) ^ row_order<D>(row)) * 8;
    krel[j] = (uint32_t)(row * p.sk.t + chunk) * 2u;
    vrel[j] = (uint32_t)(row * p.sv.t + chunk) * 2u;
  }
  const uint32_t slots = lds_addr(ring[0][0]) + (uint32_t)wave * 8u * KE;
  int mb = 1;
  auto issue = [&](auto slot, int blk) {
    const int left = n - blk * 32;
    const u32x4 rk = TileLoad<D, 4, 32>::buffer(kh + (int64_t)blk * 32 * p.sk.t, p.sk.t, left);
    const u32x4 rv = TileLoad<D, 4, 32>::buffer(vh + (int64_t)blk * 32 * p.sv.t, p.sv.t, left);
    const uint32_t dst = slots + slot * 4 * KE;
    static_for<4>([&](auto j) {
      dma16<j * 1024>(rk, dst, krel[j & 1] + (uint32_t)(j / 2) * 32u * (uint32_t)p.sk.t, 0u);
      dma16<j * 1024>(rv, dst + 2 * KE, vrel[j & 1] + (uint32_t)(j / 2) * 32u * (uint32_t)p.sv.t, 0u);
    });
    if (p.key_mask) mb = blk * 32 + c32 < n ? p.key_mask[b * p.mask_stride + blk * 32 + c32] : 1;
  };
  if (b0 < b1) issue(integral_constant<int, 0>{}, b0);
  typename T::x8 qf[D / 16];
  const TwoRows two = two_rows<BIAS>(p, unit, 0, n_rows, lane);
  load_tile<T, D>(at(p.q, p.sq, two.a), two.a_ok, at(p.q, p.sq, two.b), two.b_ok, lane, qf);
  if (BIAS) {
    fill_bias<T, 256>(bt, start, p, unit % p.H, tid);
    __syncthreads();
  }
  Rows<T, D, 1> acc;
  acc.init();
  const int ra = row_lane<D>(c32, hw), ca = col_lane<D>(lane);
  auto block = [&](auto u, int blk) {
    // This block is there, and the other slot has been read.  (Both waits also keep
    // the compiler from moving LDS accesses past them: there is no barrier here.)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    const uint32_t keep = (uint32_t)below(blk * 32, n) & (p.key_mask ? (uint32_t)__ballot(mb != 0) : ~0u);
    u16* tK = ring[wave][u];
    u16* tV = tK + KE;
    if (blk + NW < b1) issue(integral_constant<int, 1 - u>{}, blk + NW);
    if (keep != ~0u) {
      if (keep == 0) return;
      for (int c = lane; c < 32 * CPR; c += 64)
        if (!((keep >> (c / CPR)) & 1)) *reinterpret_cast<u32x4*>(tV + c * 8) = u32x4{0, 0, 0, 0};
    }
    f32x16 x[1] = {f32x16{}};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) x[0] = T::mfma(read_row<T>(tK + (ra ^ (8 * row_chunk(ks)))), qf[ks], x[0]);
    if (BIAS) {
      const float* at = bt + bias_from(blk * 32 - (31 + off), far) + far + kPad + 31 + 4 * hw - c32;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[0][e] = fmaf(x[0][e], p.sl2, at[8 * (e >> 2) + (e & 3)]);
    }
    if (keep != ~0u) {
      const uint32_t mine = keep >> (4 * hw);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((mine >> (8 * (e >> 2) + (e & 3))) & 1)) x[0][e] = -INFINITY;
    }
    typename T::x8 pb[1][2];
    acc.weigh(x, BIAS ? 1.f : p.sl2, pb, blk == b0);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int s = 0; s < 2; ++s) acc.o[d] = T::mfma(read_col<T, D>(tV, ca, d, 16 * s), pb[0][s], acc.o[d]);
  };
  for (int blk = b0; blk < b1; blk += 2 * NW) {
    block(integral_constant<int, 0>{}, blk);
    if (blk + NW < b1) block(integral_constant<int, 1>{}, blk + NW);
  }

  // The waves' sums, through their slots: eight threads per row.
  float* mine = reinterpret_cast<float*>(ring[wave][0]);
  const float l = both_halves_sum(acc.l);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  store_tile_f32<D>(acc.o, mine + c32 * D, true, hw);
  if (hw == 0) {
    sm[wave][c32] = acc.m;
    sl[wave][c32] = l;
  }
  __syncthreads();
  const int r = tid >> 3, c = (tid & 7) * (D / 8);
  if (r >= n_rows) return;
  float m = sm[0][r], sum = 0.f, o[D / 8];
#pragma unroll
  for (int w = 1; w < NW; ++w) m = vmax(m, sm[w][r]);
#pragma unroll
  for (int j = 0; j < D / 8; ++j) o[j] = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float a = sm[w][r] == -INFINITY ? 0.f : fast_exp2(sm[w][r] - m);
    const float* from = reinterpret_cast<const float*>(ring[w][0]) + r * D + c;
    sum += a * sl[w][r];
#pragma unroll
    for (int j = 0; j < D / 8; ++j) o[j] += a * from[j];
  }
  const RowOf ro = row_of<BIAS>(p, unit, r);
  const int64_t row = ((int64_t)ro.b * p.H + ro.h) * p.Lq + ro.i;
  if (p.splits > 1) {
    const int64_t at = (int64_t)split * p.B * p.H * p.Lq + row;
#pragma unroll
    for (int j = 0; j < D / 8; j += 4)
      *reinterpret_cast<f32x4*>(p.part_o + at * D + c + j) = f32x4{o[j], o[j + 1], o[j + 2], o[j + 3]};
    if (c == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(m, sum);
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  u32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = T::pack(o[2 * j] * inv, o[2 * j + 1] * inv);
  *reinterpret_cast<u32x4*>(at(p.out, p.so, ro) + c) = v;
  if (p.lse && c == 0) p.lse[row] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Few keys, many rows: the keys and values of one (sample, key head) stay in
// LDS, and each wave walks row tiles on its own, without barriers; the next
// tile's queries are loaded while one is worked on.  What bounds it: the rows' way
// through memory beside products and weights (24 x 110,080 rows over 256 keys, d 128:
// 1.37 GB and 346 GFLOP in 409 us, 287 and 300 at a large copy's and product's rates;
// streaming the keys instead takes 577, and the first length that does not fit, 257,
// 582).
template <class T, int D>
__global__ __launch_bounds__(64 * kKeepWaves, kKeepWaves / 4) void cross_keep_kernel(const CrossParams p) {
  constexpr int NW = kKeepWaves, QR = keep_rows(D);
  extern __shared__ __attribute__((aligned(1024))) u16 keep_lds[];     // [K | V | 0 or -inf per key]
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;
  const int lid = xcd_remap(blockIdx.x, p.n_wg);
  const int unit = unit_at(p, lid / p.splits, p.Hk), chunk = lid % p.splits;
  const int b = unit / p.Hk, hk = unit % p.Hk, n = key_count(p, b);
  const int n_rows = p.G * p.Lq, n_rt = (n_rows + 32 * QR - 1) / (32 * QR);
  const int rt1 = (int)((int64_t)n_rt * (chunk + 1) / p.splits);
  int rt = (int)((int64_t)n_rt * chunk / p.splits) + wave;

  typename T::x8 qf[QR][D / 16];
  TileRegs<T, D> qn[QR];
  auto fetch = [&](int rt) {
#pragma unroll
    for (int r = 0; r < QR; ++r) {
      const TwoRows two = two_rows<false>(p, unit, (rt * QR + r) * 32, n_rows, lane);
      qn[r].load(at(p.q, p.sq, two.a), two.a_ok, at(p.q, p.sq, two.b), two.b_ok, lane);
    }
  };
  const KeptKeys<T, D> keys(p, b, hk, n, keep_lds, wave, lane, tid, [&]() {
    if (rt < rt1) fetch(rt);
  });
  for (; rt < rt1; rt += NW) {
#pragma unroll
    for (int r = 0; r < QR; ++r) qn[r].operands(qf[r]);
    if (rt + NW < rt1) fetch(rt + NW);
    Rows<T, D> acc[QR];
#pragma unroll
    for (int r = 0; r < QR; ++r) acc[r].init();
    static_for<KeptKeys<T, D>::TILES>([&](auto t) {
      if (t >= keys.nt) return;
      f32x16 x[QR][2];
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const typename T::x8 kf = read_row<T>(keys.kp[ks] + (64 * t + 32 * g) * D);
#pragma unroll
          for (int r = 0; r < QR; ++r) x[r][g] = T::mfma(kf, qf[r][ks], ks == 0 ? f32x16{} : x[r][g]);
        }
      if (!((keys.whole >> t) & 1)) {
        const float* at = keys.mask + t * 64 + 4 * hw;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int r = 0; r < QR; ++r) x[r][g][e] += at[32 * g + 8 * (e >> 2) + (e & 3)];
      }
      typename T::x8 pb[QR][2][2];
#pragma unroll
      for (int r = 0; r < QR; ++r) acc[r].weigh(x[r], p.sl2, pb[r], t == 0);
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int row = 64 * t + 16 * s;
          const typename T::x8 vf = read_cols<T>(keys.vp[d][0] + row * D, keys.vp[d][1] + (row + 8) * D);
#pragma unroll
          for (int r = 0; r < QR; ++r) acc[r].o[d] = T::mfma(vf, pb[r][s >> 1][s & 1], acc[r].o[d]);
        }
    });
#pragma unroll
    for (int r = 0; r < QR; ++r) {
      const float l = both_halves_sum(acc[r].l);
      const int r0 = (rt * QR + r) * 32;
      const TwoRows two = two_rows<false>(p, unit, r0, n_rows, fresh(lane));
      store_tile<T, D>(acc[r].o, l == 0.f ? 0.f : 1.f / l, at(p.out, p.so, two.a), two.a_ok, at(p.out, p.so, two.b),
                       two.b_ok, lane);
      // The rows of a unit are consecutive in lse.
      if (p.lse && r0 + c32 < n_rows && hw == 0)
        p.lse[(int64_t)unit * n_rows + r0 + c32] =
            l == 0.f ? -INFINITY : (acc[r].m + __builtin_amdgcn_logf(l)) * kLn2;
    }
  }
}

// Joins the ranges of a split call: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// NG groups of D / 4 threads share a row, take every NG-th range each and join
// their sums, all in a fixed order.  Many ranges come with few rows and want a
// workgroup per row (NG = 256 / (D / 4)); few ranges come with many rows, and one
// group per row then leaves no thread without a range (24,776 rows of d 64 in two
// ranges: 36 us with a workgroup per row, 5.7 so).  A chain of loads where rows are
// few (96 of 42 ranges: 4 us), else bound by its bytes.
template <class T, int D, int NG>
__global__ __launch_bounds__(256) void cross_join_kernel(const CrossParams p) {
  constexpr int TPR = D / 4;
  const int64_t rows = (int64_t)p.B * p.H * p.Lq, row = (int64_t)blockIdx.x * (256 / (TPR * NG)) + threadIdx.x / (TPR * NG);
  if (row >= rows) return;                                 // (with groups to join, never)
  const int t = threadIdx.x % TPR, grp = threadIdx.x / TPR % NG;
  float m = -INFINITY, l = 0.f;
#pragma unroll 4
  for (int s = grp; s < p.splits; s += NG) m = vmax(m, p.part_ml[2 * (s * rows + row)]);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = grp; s < p.splits; s += NG) {
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * (s * rows + row));
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_o + (s * rows + row) * D + 4 * t);
    const float w = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
    l += w * ml.y;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += w * v[j];
  }
  if constexpr (NG > 1) {
    __shared__ f32x4 so[NG][TPR];
    __shared__ float sm[NG], sl[NG];
    so[grp][t] = o;
    if (t == 0) {
      sm[grp] = m;
      sl[grp] = l;
    }
    __syncthreads();
    if (grp != 0) return;
    for (int g = 1; g < NG; ++g) m = vmax(m, sm[g]);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < NG; ++g) {
      const float w = sm[g] == -INFINITY ? 0.f : fast_exp2(sm[g] - m);
      const f32x4 v = so[g][t];
      l += w * sl[g];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += w * v[j];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int i = (int)(row % p.Lq), h = (int)(row / p.Lq % p.H), b = (int)(row / p.Lq / p.H);
  uint2 w;
  w.x = T::pack(o[0] * inv, o[1] * inv);
  w.y = T::pack(o[2] * inv, o[3] * inv);
  *reinterpret_cast<uint2*>(p.out + b * p.so.b + h * p.so.h + i * p.so.t + 4 * t) = w;
  if (p.lse && t == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

namespace {
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
}  // namespace

CrossPlan plan_fwd(const CrossParams& p, int D, bool bias) {
  CrossPlan c{};
  const int64_t units = (int64_t)p.B * (bias ? p.H : p.Hk), rows = bias ? p.Lq : (int64_t)p.G * p.Lq;
  const int64_t tiles = units * ((rows + kRows - 1) / kRows), nt = (p.Lk + 63) / 64;
  c.resident = keep_keys(p, D, bias, keep_rows(D));
  if (c.resident) {
    c.splits = keep_chunks(p, keep_rows(D));
    return c;
  }
  // Keys are split where the row tiles alone leave CUs without work, into
  // ranges of no less than four tiles; below 1,024 keys the join's launch and
  // scratch cost more than the shorter walk gains (us a call, whole and split: one
  // query over 512 keys, 32 heads, d 128 9 and 17.5).  And where all row tiles run at once but end apart, under
  // an order mask or at d 64 with one workgroup on some CUs and two on others
  // (causal 12 x 4,095 of d 128 113 and 101, 6 x 6,199 of d 64 118 and 73,
  // 12 x 8,191 194 and 175, but 32 x 4,096, 1,024 tiles, 126 and 138, and
  // 24 x 2,048 46 and 48; without order 6 x 6,199 of d 64 131 and 96, but
  // 12 x 4,095 of d 128 125 and 134).
  int64_t s = 1;
  if (tiles > 0 && tiles < 256 && nt >= 16) s = 512 / tiles;
  else if (nt >= 48 && (bias && p.rb.causal ? tiles < 1024 : D == 64 && tiles < 384)) s = D == 64 ? 4 : 2;
  s = s < nt / 4 ? s : nt / 4;
  c.splits = s < 1 ? 1 : (s > 128 ? 128 : (int)s);
  if (c.splits > 1) {
    const int64_t all = (int64_t)c.splits * p.B * p.H * p.Lq;
    c.part_ml = up256(all * D * 4);
    c.bytes = c.part_ml + up256(all * 8);
  }
  return c;
}

template <class T, int D>
static hipError_t run_fwd(CrossParams p, bool bias, const CrossPlan& c, hipStream_t st) {
  p.splits = c.splits;
  const int64_t units = (int64_t)p.B * (bias ? p.H : p.Hk), rows = bias ? p.Lq : (int64_t)p.G * p.Lq;
  if (c.resident) {
    p.n_wg = (int)(units * p.splits);
    hipLaunchKernelGGL((cross_keep_kernel<T, D>), dim3(p.n_wg), dim3(64 * kKeepWaves), keep_lds_bytes(p.Lk), st, p);
    return hipGetLastError();
  }
  p.n_wg = (int)(units * ((rows + kRows - 1) / kRows) * p.splits);
  if (p.n_wg == 0) return hipSuccess;
  const uint32_t lds = bias ? bias_entries(p.rb.far) * 4 : 0;
  bool few = false;
  if constexpr (D == 64) {
    few = rows <= 32;
    if (few && bias) hipLaunchKernelGGL((cross_few_kernel<T, D, true>), dim3(p.n_wg), dim3(256), lds, st, p);
    if (few && !bias) hipLaunchKernelGGL((cross_few_kernel<T, D, false>), dim3(p.n_wg), dim3(256), lds, st, p);
  }
  if (!few && bias) hipLaunchKernelGGL((cross_fwd_kernel<T, D, true>), dim3(p.n_wg), dim3(256), lds, st, p);
  if (!few && !bias) hipLaunchKernelGGL((cross_fwd_kernel<T, D, false>), dim3(p.n_wg), dim3(256), lds, st, p);
  if (p.splits > 1) {
    const int64_t all = (int64_t)p.B * p.H * p.Lq;
    constexpr int NG = 1024 / D;                           // a workgroup's groups
    if (p.splits > 8) hipLaunchKernelGGL((cross_join_kernel<T, D, NG>), dim3((uint32_t)all), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((cross_join_kernel<T, D, 1>), dim3((uint32_t)((all + NG - 1) / NG)), dim3(256), 0, st, p);
  }
  return hipGetLastError();
}

hipError_t launch_cross_fwd(CrossParams p, int D, bool f16, bool bias, const CrossPlan& c, hipStream_t st) {
  if (D == 64) return f16 ? run_fwd<FP16, 64>(p, bias, c, st) : run_fwd<BF16, 64>(p, bias, c, st);
  return f16 ? run_fwd<FP16, 128>(p, bias, c, st) : run_fwd<BF16, 128>(p, bias, c, st);
}

}  // namespace adaspa
