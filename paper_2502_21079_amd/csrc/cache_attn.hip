// Attention over a key/value cache in 8 bits (gfx950).
//
//   out_i = sum_j exp(S_ij - lse_i) v_j,  lse_i = log sum_j exp(S_ij),  S_ij = scale q_i . k_j
//
// over a sequence's keys j < n and, with an order, j <= n - queries + i; a row
// without any gives 0 and -inf.  Query heads that share a key head are rows of
// one problem: row r of a key head is query r / G of head hk G + r % G, so that
// neighbouring rows see almost the same keys.
//
// Keys enter the first product as codes, which 16 bits hold exactly, and their
// scale is part of the factor that the scores get anyway.  Values enter the second
// as code times scale in bf16, whose exponents hold every scale; so do the
// weights, as two values each (the second what the first leaves, 2^-16 of a weight are
// lost), so that no output type loses to their rounding.  The one exception is many rows
// with bf16 inputs: one value, which loses up to 2^-8 of a weight, as the result's own
// rounding does, since a second one is half as many matrix instructions again and leaves
// registers for half the waves (2,047 tokens over 17,664, 24 heads over 4 of d 128: 399 us,
// as two values, which fp16 inputs have, 655; the largest error against 64 bits 0.00170, with
// weights in fp32 0.00166).
#include "cache_tile.hpp"

namespace adaspa {

namespace {

// Weights are taken against a reference m (log2 units) that moves to a row's
// maximum only where a score is further above it: no weight exceeds 2^8, and most
// tiles rescale nothing.
constexpr float kAbove = 8.f;
// The same by sums: a lane's weights of one tile add up to no more.
constexpr float kSumLimit = 256.f;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Two weights as bf16, and what that leaves, as bf16 again.
__device__ __forceinline__ uint32_t split2(float a, float b, uint32_t& rest) {
  const uint32_t hi = BF16::pack(a, b);
  float ha, hb;
  BF16::unpack(hi, ha, hb);
  rest = BF16::pack(a - ha, b - hb);
  return hi;
}

// The query and head of a key head's row.
__device__ __forceinline__ RowOf cache_row(const CacheParams& p, int unit, int r) {
  RowOf o;
  o.b = unit / p.Hk;
  o.i = r / p.G;
  o.h = unit % p.Hk * p.G + (r - o.i * p.G);
  return o;
}

// Keys and queries of sequence b.
__device__ __forceinline__ int key_count(const CacheParams& p, int b) {
  return p.c.pages ? clamp_len(p.lens[b], p.c.max_pages * p.c.page) : 0;
}
struct Lens {
  int n, q;                                              // keys; queries, the last q of the positions
  __device__ __forceinline__ Lens(const CacheParams& p, int b) {
    n = __builtin_amdgcn_readfirstlane(key_count(p, b));
    q = p.new_lens ? clamp_len(__builtin_amdgcn_readfirstlane(p.new_lens[b]), p.L) : p.L;
  }
  // How many keys query i sees.
  __device__ __forceinline__ int seen(const CacheParams& p, int i) const {
    if (i >= q) return 0;
    if (!p.causal) return n;
    const int m = n - q + i + 1;
    return m < 0 ? 0 : m;
  }
};

template <bool BYPASS>
__device__ __forceinline__ u32x4 read16(const uint8_t* p) {
  const u32x4* from = reinterpret_cast<const u32x4*>(p);
  if constexpr (BYPASS) return __builtin_nontemporal_load(from);
  return *from;
}

__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32) |
                   (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x));
}

// The turns of all samples, and where share w of them begins (in LDS: sample, turn of
// that).  Share 0 also leaves the turns before each sample for the join.
struct Turns {
  int64_t total;
  int shares;                                            // no more than turns
  __device__ __forceinline__ Turns(const CacheParams& p, int tid, int wave, int lane, int w, int* place) {
    __shared__ int64_t sums[4];
    const int each = (p.B + 255) / 256, b0 = tid * each, b1 = b0 + each < p.B ? b0 + each : p.B;
    auto turns = [&](int b) { return (key_count(p, b) + 255) / 256; };
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += turns(b);
    int64_t upto = mine;                                   // of this wave's lanes up to this one
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int64_t x = __shfl_up(upto, s);
      if (lane >= s) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (x < wave) upto += sums[x];
      total += sums[x];
    }
    total = uniform(total);
    int64_t before = upto - mine;
    shares = (int)(total < p.shares ? total : p.shares);
    const int64_t from = shares == 0 ? 0 : total * w / shares;
    if (w == 0 || (from >= before && from < upto)) {
      for (int b = b0; b < b1; ++b) {
        const int t = turns(b);
        if (w == 0) p.before[b] = before;
        if (from >= before && from < before + t) {
          place[0] = b;
          place[1] = (int)(from - before);
        }
        before += t;
      }
      if (w == 0 && tid == 255) p.before[p.B] = total;
    }
    __syncthreads();
  }
};

}  // namespace

// Up to 16 NQ rows of a key head.  Every wave walks blocks of 64 keys of its own,
// from memory to registers in the places that the matrix instructions want: rows of
// the first product are keys ordered so that a lane's scores are those of 16
// neighbouring tokens, whose values of one channel lie side by side in the cache.
// So neither operand passes through LDS, and a block's loads are 16 bytes a lane.
//
// Work is counted in turns, 256 keys, a block for each wave.  SHARED: workgroup (w, key head)
// takes an equal share of the turns of all samples in their order, whatever their
// lengths; where a share ends inside a sequence, its sums go to the workspace (place 2 w for
// what begins inside one, 2 w + 1 for what begins with one) and cache_few_join_kernel joins
// them.  Else a workgroup takes a sequence: up to 2,048 keys that costs less than a second launch
// (2 key heads of 1,984 keys, d 64, us a call: 14.4 and 17.7; 4 of 4,096, d 128: 25.8 and 19.0.  A CU
// reads 50 GB/s, so eight waves instead of four gain nothing).
//
// Workgroups are few (one a CU; two where the next paragraph says so) and every wave has one or two
// blocks, 16 to 32 KB, on their way: more of them only spread the reads over memory.  The key heads of
// a share run side by side, since they lie side by side in a page.  BYPASS: keys and values that the
// last-level cache could not keep until the next call are read past it.  16 sequences of up to
// 17,664 tokens, 4 key heads of d 128 under 24, and 110,080 tokens of 24 heads, us a call: shares in
// the order samples, key heads, turns, 512 workgroups 53 and 129; key heads side by side 51 and 128;
// 256 workgroups 48 and 124; past the cache 46 and 113 (6.0 TB/s).
//
// Two tiles of rows, and three at d 64, have more to work on between a block's loads: two workgroups a CU,
// whose waves hold one block each (and so fit), work on one while the other's is on its way.  The same
// sequences, us: 18 rows 64 and 54.5, 48 rows of d 64 52 and 47; two of 6,000, 24 key heads, 20 rows 29.5 and
// 31; 48 rows of d 128 75 and 95 (they do not fit), 6 rows 48 and 47.5.
//
// Weights as two values for bf16 inputs too, us with one and with two: 16 sequences of up to 17,664
// tokens, 6 rows 46.4 and 47.7, 18 rows 58.9 and 59.5, 48 rows 74 and 79, 48 rows of d 64 42 and 47;
// 110,080 tokens of 24 heads 112.6 and 113.2.
constexpr bool one_block(int D, int tiles, bool shared) { return shared && (tiles == 2 || (tiles == 3 && D == 64)); }

template <class T, int D, int NQ, bool SHARED, bool BYPASS>
__global__ __launch_bounds__(256, !one_block(D, NQ, SHARED) && (NQ == 3 || (D == 128 && NQ == 2)) ? 1 : 2) void cache_few_kernel(const CacheParams p) {
  constexpr int NW = 4, STEP = 64 * NW, DT = D / 16, KJ = D / 64;          // channel tiles; 16-byte pieces of a key a lane
  __shared__ __attribute__((aligned(16))) float so[NW][NQ * 16 * D];
  __shared__ float sm[NW][NQ * 16], sl[NW][NQ * 16];
  __shared__ int place[2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int g = lane >> 4, c16 = lane & 15;
  const int n_rows = p.G * p.L, shift = 31 - __builtin_clz(p.c.page);
  const int hk = blockIdx.x % p.Hk, w = blockIdx.x / p.Hk;
  int b = w, left = 0;                                     // sample; turns of it before this share
  int64_t turn = 0, end = 1;                               // this workgroup's share of all turns
  if constexpr (SHARED) {
    const Turns all(p, tid, wave, lane, w, place);
    if (w >= all.shares) return;
    turn = all.total * w / all.shares;
    end = all.total * (w + 1) / all.shares;
    b = __builtin_amdgcn_readfirstlane(place[0]);
    left = __builtin_amdgcn_readfirstlane(place[1]);
  }
  for (bool first = true;; first = false) {
    const Lens len(p, b);
    const int turns = (len.n + STEP - 1) / STEP;
    if (SHARED && turns == 0) {                            // the next sample with keys (there is one)
      ++b;
      continue;
    }
    const int upto = !SHARED || turns - left <= end - turn ? turns : left + (int)(end - turn);
    const int k0 = left * STEP, k1 = upto * STEP < len.n ? upto * STEP : len.n;  // keys of this part of the share
    const int unit = b * p.Hk + hk;

    typename T::x8 qf[NQ][KJ][2];
    int seen[NQ];
    float m[NQ], l[NQ];
    f32x4 o[NQ][DT];
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const bool ok = r * 16 + c16 < n_rows;
      const RowOf ro = cache_row(p, unit, ok ? r * 16 + c16 : 0);
      const u16* q = at(p.q, p.sq, ro);
      seen[r] = ok ? len.seen(p, ro.i) : 0;
#pragma unroll
      for (int j = 0; j < KJ; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 w = {0, 0, 0, 0};
          if (ok) w = *reinterpret_cast<const u32x4*>(q + 64 * j + 16 * g + 8 * h);
          qf[r][j][h] = __builtin_bit_cast(typename T::x8, w);
        }
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[r][d] = f32x4{};
    }
    const int fewest = len.q < p.L ? 0 : len.seen(p, 0);     // keys that every row sees

    struct Block {
      u32x4 k[4][KJ], v[DT];
      float ks, vs;
      int live;                                              // tokens of this lane's 16 that are there
    };
    // What the table says of this wave's next 16 blocks (lane 4 i + j: sixteen j of block
    // i) and of the 16 after them, so that no load waits for another.  n > 0; behind the last
    // token the last one's page stands.
    auto look = [&](int k) {
      const int pos = k + (lane >> 2) * STEP + (lane & 3) * 16;
      return p.c.table[b * p.c.table_stride + ((pos < len.n - 1 ? pos : len.n - 1) >> shift)];
    };
    int pages = 0, later = 0, at_page = 0;
    // What is not there is read from the pool's first page and masked.
    auto load = [&](Block& x, int k) {
      if (at_page == 64) {
        pages = later;
        later = look(k + 16 * STEP);
        at_page = 0;
      }
      const int i0 = __builtin_amdgcn_readlane(pages, at_page), i1 = __builtin_amdgcn_readlane(pages, at_page + 1);
      const int i2 = __builtin_amdgcn_readlane(pages, at_page + 2), i3 = __builtin_amdgcn_readlane(pages, at_page + 3);
      at_page += 4;
      auto of = [&](int i) {                                 // (by bits: a choice would put them in memory)
        const int odd = -(i & 1), lo = i0 ^ ((i0 ^ i1) & odd), hi = i2 ^ ((i2 ^ i3) & odd);
        return (uint32_t)(lo ^ ((lo ^ hi) & -(i >> 1)));
      };
      // Keys: 16 rows of an instruction are tokens 4 t + c16 % 4 of sixteen number c16 / 4.
      const uint32_t kp = of(c16 >> 2), vp = of(g), all = p.c.pages, mask = p.c.page - 1;
      const int64_t ka = (int64_t)(kp < all ? kp : 0) * p.Hk + hk, va = (int64_t)(vp < all ? vp : 0) * p.Hk + hk;
      const uint8_t* kt = p.c.k + (ka << shift) * D + (((k + (c16 >> 2) * 16) & mask) + (c16 & 3)) * D + 16 * g;
      const uint8_t* vt = p.c.v + (va << shift) * D + ((k + g * 16) & mask) * D + 16 * c16;
      x.ks = p.c.k_scale[va];
      x.vs = p.c.v_scale[va];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < KJ; ++j) x.k[t][j] = read16<BYPASS>(kt + 4 * t * D + 64 * j);
#pragma unroll
      for (int d = 0; d < DT; ++d) x.v[d] = read16<BYPASS>(vt + 256 * d);
      const int left = len.n - (k + g * 16);
      x.live = vp < all ? (left < 16 ? left : 16) : 0;
    };
    auto work = [&](Block& x, int k) {
      const bool edge = k + 64 > fewest || __any(x.live < 16);
      if (edge) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) x.v[d][i] &= first_bytes(x.live - 4 * i);
        if (x.live <= 0) x.vs = 1.f;                         // no page's scale, and zeros
      }
      f32x4 s[NQ][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int r = 0; r < NQ; ++r) s[r][t] = f32x4{};
#pragma unroll
        for (int j = 0; j < KJ; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const typename T::x8 kf = decode8<T>(x.k[t][j][2 * h], x.k[t][j][2 * h + 1], 1.f);
#pragma unroll
            for (int r = 0; r < NQ; ++r) s[r][t] = mfma16(kf, qf[r][j][h], s[r][t]);
          }
      }
      const float a = x.ks * p.sl2;
      bf16x8 w[NQ][2], rest[NQ][2];
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        float top = -INFINITY;
        const int see = seen[r] - (k + 16 * g) < x.live ? seen[r] - (k + 16 * g) : x.live;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[r][t][e] *= a;
            if (edge && 4 * t + e >= see) s[r][t][e] = -INFINITY;
            top = vmax(top, s[r][t][e]);
          }
        const auto u = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = both_halves_max(vmax(__uint_as_float(u[0]), __uint_as_float(u[1])));
        if (__any(!(top <= m[r] + kAbove))) {                // NaN too: the row becomes NaN
          const float to = top <= m[r] ? m[r] : top;
          const float by = to == -INFINITY ? 1.f : fast_exp2(m[r] - to);
          m[r] = to;
          l[r] *= by;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][d][e] *= by;
        }
        const float ref = m[r] == -INFINITY ? 0.f : m[r];
        float sum = 0.f;
        u32x4 hi[2], lo[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float c = fast_exp2(s[r][t][e] - ref), d = fast_exp2(s[r][t][e + 1] - ref);
            sum += c + d;
            uint32_t left = 0;
            hi[t >> 1][(t & 1) * 2 + e / 2] = split2(c, d, left);
            lo[t >> 1][(t & 1) * 2 + e / 2] = left;
          }
        l[r] += sum;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          w[r][h] = __builtin_bit_cast(bf16x8, hi[h]);
          rest[r][h] = __builtin_bit_cast(bf16x8, lo[h]);
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 vf = decode8<BF16>(x.v[d][2 * h], x.v[d][2 * h + 1], x.vs);
#pragma unroll
          for (int r = 0; r < NQ; ++r) {
            o[r][d] = mfma16(vf, w[r][h], o[r][d]);
            o[r][d] = mfma16(vf, rest[r][h], o[r][d]);
          }
        }
    };
    int k = k0 + wave * 64;
    if (one_block(D, NQ, SHARED) && k < k1) {
      Block x;
      pages = look(k);
      later = look(k + 16 * STEP);
      for (;; k += STEP) {
        load(x, k);
        work(x, k);
        if (k + STEP >= k1) break;
      }
    }
    if (!one_block(D, NQ, SHARED) && k < k1) {
      Block x[2];
      // A block's loads go out before the one before it is worked on, also where it is past the
      // range (it is not worked on): behind a branch the compiler would wait for the newest.
      pages = look(k);
      later = look(k + 16 * STEP);
      load(x[0], k);
      // The queries are there (all but the newest 2 + 4 KJ + DT loads): left to the first product,
      // inside the loop, their wait would hold up every turn.
      constexpr int newest = 2 + 4 * KJ + DT;
      __builtin_amdgcn_s_waitcnt(0x0F70 | (newest & 15) | (newest >> 4 << 14));
      for (;; k += 2 * STEP) {
        load(x[1], k + STEP);
        work(x[0], k);
        if (k + STEP >= k1) break;
        load(x[0], k + 2 * STEP);
        work(x[1], k + STEP);
        if (k + 2 * STEP >= k1) break;
      }
    }

    // The waves' sums: lane c16 of a group of 16 has row c16, channels 16 d + 4 g on.
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const auto u = __builtin_amdgcn_permlane16_swap(__float_as_uint(l[r]), __float_as_uint(l[r]), false, false);
      l[r] = both_halves_sum(__uint_as_float(u[0]) + __uint_as_float(u[1]));
      if (g == 0) {
        sm[wave][r * 16 + c16] = m[r];
        sl[wave][r * 16 + c16] = l[r];
      }
      // A row that saw nothing has zeros, also where values that others saw are no numbers.
      const bool none = m[r] == -INFINITY;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<f32x4*>(&so[wave][(r * 16 + c16) * D + 16 * d + 4 * g]) = none ? f32x4{} : o[r][d];
    }
    __syncthreads();
    constexpr int TPR = D / 4;
    for (int i = tid; i < n_rows * TPR; i += 64 * NW) {
      const int r = i / TPR, c = i % TPR * 4;
      float top = sm[0][r], sum = 0.f;
#pragma unroll
      for (int w = 1; w < NW; ++w) top = sm[w][r] <= top ? top : sm[w][r];
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float by = sm[w][r] == -INFINITY ? 0.f : fast_exp2(sm[w][r] - top);
        const f32x4 y = *reinterpret_cast<const f32x4*>(&so[w][r * D + c]);
        sum += by * sl[w][r];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += by * y[e];
      }
      if (SHARED && (left > 0 || upto < turns)) {
        const int64_t to = ((2 * w + (first && left > 0 ? 0 : 1)) * (int64_t)p.Hk + hk) * n_rows + r;
        *reinterpret_cast<f32x4*>(p.part_o + to * D + c) = v;
        if (c == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * to) = make_float2(top, sum);
        continue;
      }
      const RowOf ro = cache_row(p, unit, r);
      const int64_t row = ((int64_t)ro.b * p.H + ro.h) * p.L + ro.i;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      *reinterpret_cast<uint2*>(at(p.out, p.so, ro) + c) =
          make_uint2(T::pack(v[0] * inv, v[1] * inv), T::pack(v[2] * inv, v[3] * inv));
      if (p.lse && c == 0) p.lse[row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    turn += upto - left;
    if (!SHARED || turn >= end) return;
    left = 0;
    ++b;
    __syncthreads();                                         // the waves' sums have been read
  }
}

// Joins the shares of key heads that several workgroups had, in their order, and writes
// the rows of sequences without tokens; the others were written already.  A workgroup per row.
template <class T, int D>
__global__ __launch_bounds__(256) void cache_few_join_kernel(const CacheParams p) {
  constexpr int TPR = D / 4, NG = 256 / TPR;
  __shared__ f32x4 so[NG][TPR];
  __shared__ float sm[NG], sl[NG];
  const int n_rows = p.G * p.L, unit = blockIdx.x / n_rows, r = blockIdx.x % n_rows;
  const RowOf ro = cache_row(p, unit, r);
  const int64_t from = p.before[ro.b], to = p.before[ro.b + 1], total = p.before[p.B];
  // Turn x is in share ((x + 1) shares - 1) / total.
  const int64_t shares = total < p.shares ? total : p.shares;
  const int w0 = from == to ? 0 : (int)(((from + 1) * shares - 1) / total);
  const int w1 = from == to ? -1 : (int)((to * shares - 1) / total);
  if (w0 == w1) return;
  const int t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  auto slot = [&](int w) { return ((2 * w + (w == w0 ? 1 : 0)) * (int64_t)p.Hk + unit % p.Hk) * n_rows + r; };
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int w = w0 + grp; w <= w1; w += NG) {
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * slot(w));
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_o + slot(w) * D + 4 * t);
    const float top = ml.x <= m ? m : ml.x;
    const float old = m == -INFINITY ? 0.f : fast_exp2(m - top), by = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
    m = top;
    l = l * old + by * ml.y;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] * old + by * v[j];
  }
  so[grp][t] = o;
  if (t == 0) {
    sm[grp] = m;
    sl[grp] = l;
  }
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int x = 1; x < NG; ++x) m = sm[x] <= m ? m : sm[x];
  l = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < NG; ++x) {
    const float w = sm[x] == -INFINITY ? 0.f : fast_exp2(sm[x] - m);
    const f32x4 v = so[x][t];
    l += w * sl[x];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += w * v[j];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(at(p.out, p.so, ro) + 4 * t) =
      make_uint2(T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv));
  if (p.lse && t == 0) p.lse[((int64_t)ro.b * p.H + ro.h) * p.L + ro.i] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Many rows: 32 NW of a key head, over tiles of 64 keys that are turned into 16 bits
// once for all of them on their way to LDS: raw codes are loaded into registers two
// tiles ahead (values: one), and written while an earlier tile is worked on.
//   keys: 16-byte pieces (8 channels) of the tile's 64 keys side by side, a piece
//   and one further apart each time, so that neither way meets a bank twice;
//   values: pieces of 8 tokens of a channel, in the order of the weights' places
//   in the second product, channels side by side.
// Every place that a lane reads is its own base plus a constant.
constexpr int kKeyPiece = 64 * 8 + 8;                      // elements from a piece of the keys to the next
// Waves of a workgroup, 32 rows each; two waves a SIMD (fp16 at d 128 one: its second values leave no
// more registers).  d 128: a tile's decoding and its way through LDS serve 256 rows; with four
// waves and two workgroups a CU 2,047 tokens over 17,664 (24 heads over 4) take 456 instead of 413 us, a
// prompt of 4,096 128 instead of 118.  At d 64 a tile has a piece of keys and of values for each of
// 256 threads.
// What bounds it: the matrix pipe at the clock that the card holds under it (busy 52% of the cycles, as
// vector units issue in 45%) and, for the example, 20 us of joining four ranges: 399 us in all, 1,050
// TFLOP/s where a product of 8,192^3 has 1,209; without ranges (4 x 16 heads, 4,096 over 16,384) 1,204.
// fp16 at d 128 655 us: six matrix instructions instead of four, and one wave a SIMD instead of two.
// d 64: 4,096 tokens of 24 heads over 4 74 us, 700 TFLOP/s: half the matrix instructions for a weight's
// same vector work (vector units issuing in 47% of the cycles, the matrix pipe busy in 28%).
constexpr int row_waves(bool f16, int D) { return f16 ? 4 : D / 16; }

// One step over tiles that every row sees whole: the scores of the next tile, the
// weights of this one, the output of the one before, in slots of one MFMA and a share of
// the weights' three stages (argument, exponential, rounding and sum), each a slot after
// the one it needs; a fence closes the slot, so that the matrix pipe and the vector units work side
// by side within a wave.  Scores and outputs alternate (with fp16 the output takes the weights'
// second values too); operands are read two slots ahead.  hook(i): the caller's share of slot i.
template <class T, int D, typename Hook>
__device__ __forceinline__ void rows_step(Hook&& hook, const u16* k, const u16* v, const typename T::x8 (&qf)[D / 16],
                                          const f32x16 (&s_cur)[2], const f32x4& a, float mc,
                                          const bf16x8 (&p_prev)[2][4], f32x16 (&s_next)[2], bf16x8 (&p_cur)[2][4],
                                          f32x16 (&o)[D / 32], float& sum) {
  constexpr int NK = D / 16, ND = D / 32, NM = 2 * NK + 4 * ND, PER = 32 / NM, AHEAD = 2;
  static_assert(2 * NK == 4 * ND && 32 % NM == 0, "slots alternate and share the weights evenly");
  u32x4 op[NM];
  auto fetch = [&](int i) {
    const int j = i >> 1;
    op[i] = *reinterpret_cast<const u32x4*>((i & 1) == 0 ? k + row_chunk(j % NK) * kKeyPiece + j / NK * 256
                                                         : v + (2 * (j / ND) * D + 32 * (j % ND)) * 8);
  };
  auto mfma = [&](int i) {
    const int j = i >> 1;
    if ((i & 1) == 0)
      s_next[j / NK] = T::mfma(__builtin_bit_cast(typename T::x8, op[i]), qf[j % NK],
                               j % NK == 0 ? f32x16{} : s_next[j / NK]);
    else o[j % ND] = mfma32(__builtin_bit_cast(bf16x8, op[i]), p_prev[0][j / ND], o[j % ND]);
  };
  float arg[32], ex[32], s0 = 0.f, s1 = 0.f;
  auto stage_arg = [&](int i) {
#pragma unroll
    for (int e = i * PER; e < (i + 1) * PER; ++e) {
      arg[e] = fmaf(s_cur[e >> 4][e & 15], a[e >> 3], -mc);
      pin(arg[e]);
    }
  };
  auto stage_exp = [&](int i) {
#pragma unroll
    for (int e = i * PER; e < (i + 1) * PER; ++e) {
      ex[e] = fast_exp2(arg[e]);
      pin(ex[e]);
    }
  };
  auto stage_sum = [&](int i) {
#pragma unroll
    for (int e = i * PER; e < (i + 1) * PER; ++e)
      if (e & 1) {
        uint32_t rest = 0;
        bf16x2 pr = __builtin_bit_cast(bf16x2, T::kHalf ? split2(ex[e - 1], ex[e], rest) : BF16::pack(ex[e - 1], ex[e]));
        pin(pr);
        p_cur[0][e >> 3][(e & 7) - 1] = pr[0];
        p_cur[0][e >> 3][e & 7] = pr[1];
        if constexpr (T::kHalf) {
          bf16x2 lo = __builtin_bit_cast(bf16x2, rest);
          pin(lo);
          p_cur[1][e >> 3][(e & 7) - 1] = lo[0];
          p_cur[1][e >> 3][e & 7] = lo[1];
        }
        s0 += ex[e - 1];
        s1 += ex[e];
        pin(s0);
        pin(s1);
      }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fetch(i);
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    if (i + AHEAD < NM) fetch(i + AHEAD);
    mfma(i);
    hook(i);
    stage_arg(i);
    if (i >= 1) stage_exp(i - 1);
    if (i >= 2) stage_sum(i - 2);
    __builtin_amdgcn_sched_barrier(0);
    if (T::kHalf && (i & 1)) {
      const int j = i >> 1;
      o[j % ND] = mfma32(__builtin_bit_cast(bf16x8, op[i]), p_prev[1][j / ND], o[j % ND]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  stage_exp(NM - 1);
  stage_sum(NM - 2);
  stage_sum(NM - 1);
  sum = s0 + s1;
}

// A barrier that waits for LDS alone: loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);                      // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <class T, int D>
__global__ __launch_bounds__(64 * row_waves(T::kHalf, D), T::kHalf && D == 128 ? 1 : 2) void cache_rows_kernel(const CacheParams p) {
  constexpr int NW = row_waves(T::kHalf, D), NR = 32 * NW, KP = kKeyPiece;
  constexpr int PER = 4 * D / (64 * NW);                   // 16-byte pieces of a thread, of a tile's keys and of its values
  __shared__ __attribute__((aligned(16))) u16 sk[2][D / 8 * KP];
  __shared__ __attribute__((aligned(16))) u16 sv[2][64 * D];
  __shared__ __attribute__((aligned(16))) float scale[4][4];   // factors on the scores of a tile's sixteens; below 0: not there
  __shared__ int again;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hw = lane >> 5, c32 = lane & 31;
  const int n_rows = p.G * p.L, n_rt = (n_rows + NR - 1) / NR;
  // All units' longest row tiles come first, and the short ones fill the gaps.
  const int around = p.n_wg / n_rt, lid = xcd_remap(blockIdx.x % around, around);
  const int unit = lid / p.chunks, range = lid % p.chunks, rt = n_rt - 1 - blockIdx.x / around;
  const int b = unit / p.Hk, hk = unit % p.Hk;
  const Lens len(p, b);
  if (range > 0 && range * p.chunk >= len.n) return;
  const int r0 = rt * NR, rw = r0 + wave * 32, r = rw + c32;
  const bool ok = r < n_rows;
  const RowOf ro = cache_row(p, unit, ok ? r : 0);
  const int seen = ok ? len.seen(p, ro.i) : 0;
  // The most keys that a row of [from, to] sees.
  auto most_of = [&](int from, int to) {
    const int i = to / p.G < len.q ? to / p.G : len.q - 1;
    return from > to || i < from / p.G ? 0 : len.seen(p, i);
  };
  const int end = most_of(r0, r0 + NR < n_rows ? r0 + NR - 1 : n_rows - 1);
  const int most = most_of(rw, rw + 32 < n_rows ? rw + 31 : n_rows - 1);
  const int k0 = range * p.chunk, k1 = end - k0 < p.chunk ? end : k0 + p.chunk;
  const int nt = k1 > k0 ? (k1 - k0 + 63) / 64 : 0;
  // Tiles that all rows which see anything see whole: the first row sees the fewest.  (Rows behind
  // the last query, and behind the last row, are worked on like it and count for nothing.)
  const int fewest = len.seen(p, r0 / p.G) - k0;
  // They are taken in pairs.
  int whole = fewest <= 0 ? 0 : (fewest / 64 < nt ? fewest / 64 : nt) & ~1;

  const int shift = 31 - __builtin_clz(p.c.page), mask = p.c.page - 1;
  // This thread's piece j of a tile, for keys and for values alike: of sixteen number six(j).
  const int in = tid % D;
  auto six = [&](int j) { return wave * 64 / D + j * 64 * NW / D; };
  auto place = [&](int t, int j) { return k0 + t * 64 + six(j) * 16; };
  // What the page table says of that sixteen in 64 tiles (a lane each) and the 64 after them.
  auto look = [&](int t, int j) {
    const int pos = place(t + lane, j);
    return p.c.table[b * p.c.table_stride + ((pos < len.n - 1 ? pos : len.n - 1) >> shift)];
  };
  int pages[PER], later[PER], id_k[PER], id_v[PER], id_between[PER];       // those of the tiles that rk and rv hold, and between
  u32x4 rk[PER], rv[PER];
  float ks[PER], vs[PER];
  bool gone = false;                                       // a page that is not there
  auto there = [&](int id, int pos) { return pos < len.n && (uint32_t)id < (uint32_t)p.c.pages; };
  auto offset = [&](int id, int pos) {                     // in the pool, of this thread's piece
    const int64_t a = (int64_t)(there(id, pos) ? id : 0) * p.Hk + hk;
    return (a << shift) * D + (pos & mask) * D + in * 16;
  };
  auto turn_pages = [&](int t) {                           // before tile t is fetched
    if ((t & 63) != 0 || t == 0) return;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      pages[j] = later[j];
      later[j] = look(t + 64, j);
    }
  };
  auto fetch_k = [&](int t) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      id_v[j] = id_between[j];
      id_between[j] = id_k[j];
      id_k[j] = __builtin_amdgcn_readlane(pages[j], t & 63);
      const int pos = place(t, j);
      rk[j] = *reinterpret_cast<const u32x4*>(p.c.k + offset(id_k[j], pos));
      ks[j] = p.c.k_scale[(int64_t)(there(id_k[j], pos) ? id_k[j] : 0) * p.Hk + hk];
    }
  };
  auto fetch_v = [&](int t, const int (&id)[PER]) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int pos = place(t, j);
      rv[j] = *reinterpret_cast<const u32x4*>(p.c.v + offset(id[j], pos));
      vs[j] = p.c.v_scale[(int64_t)(there(id[j], pos) ? id[j] : 0) * p.Hk + hk];
    }
  };
  auto put_k = [&](int t) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      u16* k = sk[t & 1] + in % (D / 16) * 2 * KP + (six(j) * 16 + in / (D / 16)) * 8;
      *reinterpret_cast<typename T::x8*>(k) = decode8<T>(rk[j][0], rk[j][1], 1.f);
      *reinterpret_cast<typename T::x8*>(k + KP) = decode8<T>(rk[j][2], rk[j][3], 1.f);
      // At least 2^-126, so that times minus infinity it hides.  (Every lane of the wave has the same.)
      const bool is = there(id_k[j], place(t, j));
      scale[t & 3][six(j)] = is ? fmaxf(ks[j] * p.sl2, 0x1p-126f) : -1.f;
      gone = gone || (!is && place(t, j) < len.n);
    }
  };
  // all: every token is there (or the tile is worked on again).
  auto put_v = [&](auto all, int t) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int live = there(id_v[j], place(t, j)) ? len.n - place(t, j) : 0;
      float by = vs[j];
      if (!all && live < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) rv[j][i] &= first_bytes(live - 4 * i);
        if (live <= 0) by = 1.f;                           // no page's scale, and zeros
      }
      u16* v = sv[t & 1] + (six(j) * 2 * D + in) * 8;
      *reinterpret_cast<bf16x8*>(v) = decode8<BF16>(rv[j][0], rv[j][2], by);
      *reinterpret_cast<bf16x8*>(v + D * 8) = decode8<BF16>(rv[j][1], rv[j][3], by);
    }
  };

  typename T::x8 qf[D / 16];
  auto two = [&](int ln) {
    TwoRows w;
    const int x = rw + (ln & 15);
    w.a_ok = x < n_rows;
    w.b_ok = x + 16 < n_rows;
    w.a = cache_row(p, unit, w.a_ok ? x : 0);
    w.b = cache_row(p, unit, w.b_ok ? x + 16 : 0);
    return w;
  };
  {
    TwoRows w = two(lane);
    // What lies behind a sample's last query is not read: it may be anything.
    w.a_ok = w.a_ok && w.a.i < len.q;
    w.b_ok = w.b_ok && w.b.i < len.q;
    load_tile<T, D>(at(p.q, p.sq, w.a), w.a_ok, at(p.q, p.sq, w.b), w.b_ok, lane, qf);
  }
  f32x16 o[D / 32];
  float m, l;
  const int kl = 2 * hw * KP + c32 * 8, vl = (hw * D + c32) * 8;       // this lane's places in a tile
  auto scores = [&](int t, f32x16 (&x)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = f32x16{};
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        x[h] = T::mfma(*reinterpret_cast<const typename T::x8*>(sk[t & 1] + kl + row_chunk(s) * KP + 256 * h), qf[s],
                         x[h]);
    }
  };
  auto output = [&](int t, const bf16x8 (&w)[4]) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        o[d] = mfma32(*reinterpret_cast<const bf16x8*>(sv[t & 1] + vl + (2 * s * D + 32 * d) * 8), w[s], o[d]);
  };
  auto rescale = [&](float by) {
    l *= by;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] *= by;
  };
  auto top_of = [&](const f32x16 (&x)[2], const f32x4& a) {
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = vmax(top, x[h][e] * a[2 * h + (e >> 3)]);
    return both_halves_max(top);
  };

  for (;;) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};
    m = -INFINITY;
    l = 0.f;
    if (nt == 0) break;
    if (tid == 0) again = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      pages[j] = look(0, j);
      later[j] = look(64, j);
      id_k[j] = id_v[j] = id_between[j] = 0;
    }
    __syncthreads();
    fetch_k(0);
    put_k(0);
    fetch_k(1);
    put_k(1);
    fetch_k(2);
    fetch_v(0, id_v);
    int t = 0;
    if (whole > 0) {
#pragma unroll
      for (int j = 0; j < 2 * PER; ++j)                    // the values before the first tile's
        *reinterpret_cast<u32x4*>(&sv[1][(tid + 64 * NW * j) * 8]) = u32x4{0, 0, 0, 0};
      lds_barrier();
      f32x16 s[2][2];
      bf16x8 w[2][2][4];                                 // of two tiles: weights, and with fp16 what they leave
#pragma unroll
      for (int i = 0; i < 4; ++i) w[1][0][i] = w[1][1][i] = bf16x8{};
      scores(0, s[0]);
      m = top_of(s[0], *reinterpret_cast<const f32x4*>(scale[0]));
      lds_barrier();                                     // the first step writes tile 2's keys over tile 0's
      bool bad = !(m < INFINITY && m > -INFINITY);
      if (bad) m = 0.f;
      auto step = [&](auto u) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(scale[t & 3]);
        float sum;
        turn_pages(t + 3);
        rows_step<T, D>([&](int i) {
          if (i == 1) put_k(t + 2);
          if (i == 3) put_v(integral_constant<bool, true>{}, t);
          if (i == 5) {
            fetch_k(t + 3);
            fetch_v(t + 1, id_v);
          }
        }, sk[1 - u] + kl, sv[1 - u] + vl, qf, s[u], a, m, w[1 - u], s[1 - u], w[u], o, sum);
        // A row's sum of this tile is far above its reference: what was taken against that, this
        // tile's weights too, moves by a power of two, exactly.
        const float most = both_halves_max(sum);
        if (__any(!(most <= kSumLimit))) {
          bad = bad || !(most <= 0x1p30f);
          const float by = most > kSumLimit ? __builtin_floorf(__builtin_amdgcn_logf(most)) : 0.f;
          const float f = fast_exp2(-by);
          m += by;
          sum *= f;
          rescale(f);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              w[u][0][i][e] = (__bf16)((float)w[u][0][i][e] * f);
              if (T::kHalf) w[u][1][i][e] = (__bf16)((float)w[u][1][i][e] * f);
            }
        }
        l += sum;
        ++t;
        lds_barrier();
      };
      while (t < whole) {
        step(integral_constant<int, 0>{});
        step(integral_constant<int, 1>{});
      }
      output(1, w[1][0]);                                // the last tile's
      if (T::kHalf) output(1, w[1][1]);
      if (bad || gone) again = 1;
    }
    for (; t < nt; ++t) {
      put_v(integral_constant<bool, false>{}, t);
      fetch_v(t + 1, id_between);
      lds_barrier();
      const int key0 = k0 + t * 64;
      if (key0 < most) {
        const f32x4 a4 = *reinterpret_cast<const f32x4*>(scale[t & 3]);
        f32x16 x[2];
        scores(t, x);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            // Minus infinity, once times the factor.
            if (key0 + 32 * h + 8 * (e >> 2) + 4 * hw + (e & 3) >= seen || a4[2 * h + (e >> 3)] < 0.f)
              x[h][e] = a4[2 * h + (e >> 3)] < 0.f ? INFINITY : -INFINITY;
        bf16x8 w[4], rest[4];
        auto weigh = [&]() {
          const float ref = m == -INFINITY ? 0.f : -m;
          float s0 = 0.f, s1 = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u32x4 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float c = fast_exp2(fmaf(x[i >> 1][(i & 1) * 8 + e], a4[i], ref));
              const float d = fast_exp2(fmaf(x[i >> 1][(i & 1) * 8 + e + 1], a4[i], ref));
              s0 += c;
              s1 += d;
              uint32_t left = 0;
              hi[e >> 1] = T::kHalf ? split2(c, d, left) : BF16::pack(c, d);
              lo[e >> 1] = left;
            }
            w[i] = __builtin_bit_cast(bf16x8, hi);
            rest[i] = __builtin_bit_cast(bf16x8, lo);
          }
          return s0 + s1;
        };
        float sum = weigh();
        const bool need = !(both_halves_max(sum) <= kSumLimit) || (m == -INFINITY && key0 < seen);
        if (__any(need)) {
          const float top = top_of(x, a4);
          const bool move = need && !(top <= m);           // NaN too: the row becomes NaN
          const float by = move ? fast_exp2(m - top) : 1.f;
          if (move) m = top;
          rescale(by);
          sum = weigh();
        }
        l += sum;
        output(t, w);
        if (T::kHalf) output(t, rest);
      }
      lds_barrier();
      put_k(t + 2);
      turn_pages(t + 3);
      fetch_k(t + 3);
    }
    // Scores too far above their row's first ones, or a page that is not there: once more, tile by tile.
    lds_barrier();
    if (whole == 0 || !again) break;
    whole = 0;
    __syncthreads();
  }
  if (seen <= k0) {                                        // no key here, or no query
    l = 0.f;
    m = -INFINITY;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};
  }

  l = both_halves_sum(l);
  const int64_t row = ((int64_t)ro.b * p.H + ro.h) * p.L + ro.i;
  if (p.chunks > 1) {
    const int64_t to = (int64_t)range * p.B * p.H * p.L + row;
    store_tile_f32<D>(o, p.part_o + to * D, ok, hw);
    if (ok && hw == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * to) = make_float2(l == 0.f ? -INFINITY : m, l);
    return;
  }
  const TwoRows w = two(lane);
  store_tile<T, D>(o, l == 0.f ? 0.f : 1.f / l, at(p.out, p.so, w.a), w.a_ok, at(p.out, p.so, w.b), w.b_ok, lane);
  if (p.lse && ok && hw == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Joins the ranges of a sequence's keys: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s,
// in their order.  Ranges are few (most often two to four) and rows many, so D / 4 threads have a
// row to themselves; bound by its bytes.
template <class T, int D>
__global__ __launch_bounds__(256) void cache_join_kernel(const CacheParams p) {
  constexpr int TPR = D / 4;
  const int64_t rows = (int64_t)p.B * p.H * p.L, row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (row >= rows) return;
  const int i = (int)(row % p.L), h = (int)(row / p.L % p.H), b = (int)(row / p.L / p.H), t = threadIdx.x % TPR;
  const int n = key_count(p, b);
  const int used = n > p.chunk ? (n + p.chunk - 1) / p.chunk : 1;          // the first range is always there
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < used; ++s) {
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * (s * rows + row));
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_o + (s * rows + row) * D + 4 * t);
    const float top = ml.x <= m ? m : ml.x;
    const float old = m == -INFINITY ? 0.f : fast_exp2(m - top), by = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
    m = top;
    l = l * old + by * ml.y;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] * old + by * v[j];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(p.out + b * p.so.b + h * p.so.h + i * p.so.t + 4 * t) =
      make_uint2(T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv));
  if (p.lse && t == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

namespace {
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
}  // namespace

CachePlan plan_cache_attn(const CacheParams& p, bool f16) {
  CachePlan c{};
  const int64_t units = (int64_t)p.B * p.Hk, rows = (int64_t)p.G * p.L, keys = (int64_t)p.c.max_pages * p.c.page;
  const int64_t steps = (keys + 255) / 256;
  // 33 to 48 rows too where keys are shared: 16 sequences of up to 17,664 tokens, 4 key heads of d 128
  // under 24, eight tokens each, 124 us over tiles of 256 rows, 79 here (fp16 125 and 79, d 64 54 and 47).
  // Not over less than 12 turns: 16 sequences of up to 2,304 tokens 28 and 35 (one of 3,000 24 and 21, 64 of
  // up to 4,096 107 and 96), 32 of up to 1,500 tokens, each a workgroup's, 40 rows, 23 and 27.
  // 49 to 64 rows gain nothing (60 of d 64: 20 and 20; 64 of d 128 over 100,000 tokens: 100 and 98).
  c.few = rows <= kFewRows || (rows <= kSharedRows && steps >= kSharedSteps);
  c.chunks = 1;
  c.chunk = 1 << 28;
  if (c.few) {
    // The last-level cache has 256 MB; from 192 on (217 MB: 42.6 and 38.4 us, 134 MB: 23.0 and 27.5).
    c.bypass = units * keys * 2 * p.D >= (int64_t)192 << 20;
    if (steps > kWholeSteps) {
      const int64_t room = one_block(p.D, (int)(rows + 15) / 16, true) ? 512 : 256;
      const int64_t n = p.Hk < room ? room / p.Hk : 1, most = p.B * steps;
      c.shares = (int)(n < most ? n : most);
      c.part_ml = up256(2 * c.shares * p.Hk * rows * p.D * 4);
      c.before = c.part_ml + up256(2 * c.shares * p.Hk * rows * 8);
      c.bytes = c.before + up256(((int64_t)p.B + 1) * 8);
    }
    return c;
  }
  // Ranges of the keys, so many that the workgroups (one a CU at d 128, two at d 64) end together.
  // A workgroup's start counts as six tiles and its sums' way through memory as eight.  Under an
  // order the rows of a sequence that is nearly all new differ in length: the short ones fill gaps, and
  // no more than the longest and an even share count; otherwise whole rounds do.
  const int NR = 32 * row_waves(f16, p.D), room = p.D == 128 ? 256 : 512;
  const int64_t tiles = units * ((rows + NR - 1) / NR), turns = (keys + 63) / 64;
  const bool uneven = p.causal && 2 * (int64_t)p.L > keys;
  int64_t n = 1, best = -1;
  // (Past 2^24 rows there is nothing to gain, and the join's grid has an end.)
  const int64_t most = (int64_t)p.B * p.H * p.L <= 1 << 24 ? 64 : 1;
  for (int64_t x = 1; x <= most && (x == 1 || turns / x >= 8); ++x) {
    const int64_t over = 6 + (x > 1 ? 8 : 0), each = (turns + x - 1) / x + over;
    int64_t cost = (tiles * x + room - 1) / room * each;
    if (uneven) {
      const int64_t share = tiles * (turns - p.L / 128 + x * over) / room + each / 4;
      cost = share > each ? share : each;
    }
    if (best < 0 || cost < best) {
      best = cost;
      n = x;
    }
  }
  const int64_t each = turns == 0 ? 1 : (turns + n - 1) / n;
  if (n > 1) c.chunk = (int)(each * 64);
  c.chunks = n > 1 ? (int)((turns + each - 1) / each) : 1;
  if (c.chunks > 1) {
    const int64_t all = (int64_t)c.chunks * p.B * p.H * p.L;
    c.part_ml = up256(all * p.D * 4);
    c.bytes = c.part_ml + up256(all * 8);
  }
  return c;
}

template <class T, int D, int NQ>
static void run_shared(const CacheParams& p, bool bypass, hipStream_t st) {
  if (bypass) hipLaunchKernelGGL((cache_few_kernel<T, D, NQ, true, true>), dim3(p.n_wg), dim3(256), 0, st, p);
  else hipLaunchKernelGGL((cache_few_kernel<T, D, NQ, true, false>), dim3(p.n_wg), dim3(256), 0, st, p);
}
template <class T, int D, int NQ>
static void run_few(const CacheParams& p, bool bypass, hipStream_t st) {
  if (p.shares) run_shared<T, D, NQ>(p, bypass, st);
  else if (bypass) hipLaunchKernelGGL((cache_few_kernel<T, D, NQ, false, true>), dim3(p.n_wg), dim3(256), 0, st, p);
  else hipLaunchKernelGGL((cache_few_kernel<T, D, NQ, false, false>), dim3(p.n_wg), dim3(256), 0, st, p);
}

template <class T, int D>
static hipError_t run_attn(CacheParams p, const CachePlan& c, hipStream_t st) {
  const int64_t rows = (int64_t)p.G * p.L, units = (int64_t)p.B * p.Hk;
  p.chunk = c.chunk;
  p.chunks = c.chunks;
  p.shares = c.shares;
  if (c.few) {
    p.n_wg = (c.shares ? c.shares : p.B) * p.Hk;
    if (rows <= 16) run_few<T, D, 1>(p, c.bypass, st);
    else if (rows <= 32) run_few<T, D, 2>(p, c.bypass, st);
    else run_shared<T, D, 3>(p, c.bypass, st);
    if (p.shares)
      hipLaunchKernelGGL((cache_few_join_kernel<T, D>), dim3((uint32_t)(units * rows)), dim3(256), 0, st, p);
    return hipGetLastError();
  }
  constexpr int NW = row_waves(T::kHalf, D);
  p.n_wg = (int)(units * p.chunks * ((rows + 32 * NW - 1) / (32 * NW)));
  hipLaunchKernelGGL((cache_rows_kernel<T, D>), dim3(p.n_wg), dim3(64 * NW), 0, st, p);
  if (p.chunks > 1)
    hipLaunchKernelGGL((cache_join_kernel<T, D>), dim3((uint32_t)((units * rows + 1024 / D - 1) / (1024 / D))), dim3(256),
                       0, st, p);
  return hipGetLastError();
}

hipError_t launch_cache_attn(CacheParams p, bool f16, const CachePlan& c, hipStream_t st) {
  if (p.D == 64) return f16 ? run_attn<FP16, 64>(p, c, st) : run_attn<BF16, 64>(p, c, st);
  return f16 ? run_attn<FP16, 128>(p, c, st) : run_attn<BF16, 128>(p, c, st);
}

}  // namespace adaspa
