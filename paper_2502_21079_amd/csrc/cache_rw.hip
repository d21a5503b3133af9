// A key/value cache in 8 bits: quantising new tokens into its pages, and
// reading sequences back (gfx950).
//
// A page and head has one scale for keys and one for values, the least power of
// two of which 448 times is the largest finite magnitude or more.  A page that
// holds tokens already keeps the larger of its scale and the new tokens'; where it
// grows, the codes that are there are brought to it.  As scales are powers of two,
// values divide exactly and codes change scale exactly, but for those that fall
// among e4m3's subnormal numbers.
#include "cache_tile.hpp"

namespace adaspa {

// One workgroup: the keys, or the values, of one page and head.  A thread holds
// its values in registers between the search for the largest and their rounding,
// so the new tokens are read once.
//   keys: 16-byte pieces of rows, 8 values each;
//   values: two channels of 16 tokens (8 at d 64), 4-byte pieces of rows, which
//   make rows of the page's layout without an exchange.
// Bound by bytes where there are many pages (8 prompts of up to 4,999 tokens, 12 heads of d 64, fp16,
// pages of 16: 147 MB in 37 us, 4.0 TB/s, vector units issuing 55% of the time), by a chain of four
// loads (length, page, scale, token) for single tokens: 64 sequences, 4 heads of d 128: 5.9 us.
template <class T, int D, int PAGE>
__global__ __launch_bounds__(PAGE * 4) void cache_write_kernel(const CacheParams p) {
  constexpr int NT = PAGE * 4, PER = D / 32;               // 8-value pieces of a thread
  __shared__ float wave_max[NT / 64];
  const int tid = threadIdx.x, hk = blockIdx.y >> 1, b = blockIdx.z;
  const bool values = blockIdx.y & 1;
  const int64_t start = p.lens[b];
  const int n = p.new_lens ? clamp_len(p.new_lens[b], p.L) : p.L;
  // A sample without new tokens leaves every page alone: its last one may be another's to write.
  if (start < 0 || n == 0) return;
  const int64_t index = start / PAGE + blockIdx.x, first = index * PAGE;
  if (first >= start + n || index >= p.c.max_pages) return;
  const int id = page_at(p.c, b, (int)index);
  if (id < 0) return;
  // Tokens [lo, hi) of the page are new, those below lo are kept.  Token i is row i + row0.
  const int lo = start > first ? (int)(start - first) : 0;
  const int hi = start + n - first < PAGE ? (int)(start + n - first) : PAGE;
  const int row0 = (int)(first - start);
  const int64_t at = (int64_t)id * p.Hk + hk;
  float* sp = (values ? p.c.v_scale : p.c.k_scale) + at;
  const float old = *sp;

  u32x4 x[PER];
  const int tok0 = values ? (D == 128 ? tid / 64 * 16 : tid / 64 * 16 + (tid & 32) / 4) : 0;
  const int dim = values ? (D == 128 ? tid % 64 : tid % 32) * 2 : 0;
  if (values) {
    const u16* v = p.v + b * p.sv.b + hk * p.sv.h + dim;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = tok0 + 4 * j + i;
        x[j][i] = t >= lo && t < hi ? *reinterpret_cast<const uint32_t*>(v + (row0 + t) * p.sv.t) : 0u;
      }
  } else {
    const u16* k = p.k + b * p.sk.b + hk * p.sk.h;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = tid + j * NT, t = i / (D / 8);
      x[j] = u32x4{0, 0, 0, 0};
      if (t >= lo && t < hi) x[j] = *reinterpret_cast<const u32x4*>(k + (row0 + t) * p.sk.t + i % (D / 8) * 8);
    }
  }
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, c;
      T::unpack(x[j][i], a, c);
      a = __builtin_fabsf(a);
      c = __builtin_fabsf(c);
      if (a < INFINITY && a > amax) amax = a;
      if (c < INFINITY && c > amax) amax = c;
    }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) amax = fmaxf(amax, __shfl_xor(amax, s));
  if ((tid & 63) == 0) wave_max[tid / 64] = amax;
  __syncthreads();                                         // every thread has read the old scale
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) amax = fmaxf(amax, wave_max[w]);
  float scale = scale_for(amax);
  if (lo > 0) scale = fmaxf(scale, old);
  if (tid == 0) *sp = scale;
  const float inv = 1.f / scale, by = old / scale;
  const bool moved = lo > 0 && old != scale;

  if (!values) {
    uint8_t* k = p.c.k + at * (PAGE * D);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = tid + j * NT, t = i / (D / 8);
      uint2* to = reinterpret_cast<uint2*>(k + i * 8);
      if (t >= lo && t < hi) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) T::unpack(x[j][e], f[2 * e], f[2 * e + 1]);
        *to = make_uint2(encode4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                         encode4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
      } else if (t < lo && moved) {
        const uint2 w = *to;
        *to = make_uint2(recode4(w.x, by), recode4(w.y, by));
      }
    }
    return;
  }
  // Tokens [tok0, tok0 + 4 PER) of channels dim and dim + 1.
  if (tok0 >= hi || (tok0 + 4 * PER <= lo && !moved)) return;
  uint8_t* v = p.c.v + at * (PAGE * D) + (tok0 / 16 * D + dim) * 16 + tok0 % 16;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t* to = reinterpret_cast<uint32_t*>(v + c * 16);
    uint32_t w[PER];
    if (tok0 < lo || tok0 + 4 * PER > hi) {
#pragma unroll
      for (int j = 0; j < PER; ++j) w[j] = to[j];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a, d;
        T::unpack(x[j][i], a, d);
        f[i] = (c ? d : a) * inv;
      }
      const uint32_t fresh = encode4(f[0], f[1], f[2], f[3]);
      const int t = tok0 + 4 * j;
      if (t >= lo && t + 4 <= hi) {
        w[j] = fresh;
      } else {
        const uint32_t kept = first_bytes(lo - t), upto = first_bytes(hi - t);
        w[j] = (w[j] & ~upto) | (fresh & upto & ~kept) | ((moved ? recode4(w[j], by) : w[j]) & kept);
      }
    }
    if constexpr (PER == 4) *reinterpret_cast<u32x4*>(to) = u32x4{w[0], w[1], w[2], w[3]};
    else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
  }
}

// One wave: 16 tokens of one head, keys and values.  Rows [0, L) of the output are
// positions starts[b] on; those at or past the sequence's length, or on no page of
// the pool, become zeros.  Keys are 8-byte reads and 16-byte writes; values 4-byte pieces of a
// channel's sixteen, which two of them turn into 4-byte writes of a token: a wave writes whole
// lines, and nothing passes through LDS.  Bound by its bytes, two in three of them written:
// 110,080 tokens of 24 heads of d 128 2.03 GB in 384 us, 5.3 TB/s (a large copy 5.05); two clips of
// up to 17,664 tokens, d 64, 309 MB in 62 us, 5.0 TB/s.
template <class T, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheParams p) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hk = blockIdx.y, b = blockIdx.z;
  const int64_t start = p.starts ? p.starts[b] : 0;
  // Tiles of 16 positions, from the one that holds the first row on.
  const int64_t pos0 = (start >> 4 << 4) + ((int64_t)blockIdx.x * 4 + wave) * 16;
  const int64_t row0 = pos0 - start;                       // row of the tile's first token
  if (row0 >= p.L) return;
  const int64_t most = (int64_t)p.c.max_pages * p.c.page;
  const int64_t n = clamp_len(p.lens[b], (int)most);
  int id = -1, in_page = 0;
  if (pos0 >= 0 && pos0 < n) {
    id = page_at(p.c, b, (int)(pos0 / p.c.page));
    in_page = (int)(pos0 % p.c.page);
  }
  const int live = id < 0 ? 0 : (int)(n - pos0 < 16 ? n - pos0 : 16);
  const int64_t at = (int64_t)(id < 0 ? 0 : id) * p.Hk + hk;
  const float ks = live ? p.c.k_scale[at] : 0.f, vs = live ? p.c.v_scale[at] : 0.f;
  const uint8_t* k = p.c.k + at * p.c.page * D + in_page * D;
  const uint8_t* v = p.c.v + at * p.c.page * D + in_page * D;
  u16* ko = p.k_out + b * p.sk.b + hk * p.sk.h;
  u16* vo = p.v_out + b * p.sv.b + hk * p.sv.h;
  const int first = row0 < 0 ? (int)-row0 : 0, last = p.L - row0 < 16 ? (int)(p.L - row0) : 16;

#pragma unroll
  for (int j = 0; j < D / 32; ++j) {                       // 8 values a lane
    const int i = lane + 64 * j, t = i / (D / 8), c = i % (D / 8) * 8;
    u32x4 w = {0, 0, 0, 0};
    if (t < live) {
      const uint2 x = *reinterpret_cast<const uint2*>(k + i * 8);
      float f[8];
      decode4(x.x, *reinterpret_cast<float(*)[4]>(f));
      decode4(x.y, *reinterpret_cast<float(*)[4]>(f + 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = T::pack(f[2 * e] * ks, f[2 * e + 1] * ks);
    }
    if (t >= first && t < last) *reinterpret_cast<u32x4*>(ko + (row0 + t) * p.sk.t + c) = w;
  }
  // Two channels of 16 tokens (8 at d 64).
  constexpr int PER = D / 32;
  const int tok0 = D == 128 ? 0 : (lane & 32) / 4, dim = (D == 128 ? lane : lane & 31) * 2;
  uint32_t w[2][PER];
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 0; j < PER; ++j) w[c][j] = 0;
  if (live) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        w[c][j] = *reinterpret_cast<const uint32_t*>(v + (dim + c) * 16 + tok0 + 4 * j);
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    float a[4], d[4];
    decode4(w[0][j], a);
    decode4(w[1][j], d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = tok0 + 4 * j + i;
      const uint32_t x = t < live ? T::pack(a[i] * vs, d[i] * vs) : 0u;
      if (t >= first && t < last) *reinterpret_cast<uint32_t*>(vo + (row0 + t) * p.sv.t + dim) = x;
    }
  }
}

template <class T, int D>
static void run_write(const CacheParams& p, hipStream_t st) {
  const dim3 grid((uint32_t)((p.L + p.c.page - 2) / p.c.page + 1), (uint32_t)p.Hk * 2, (uint32_t)p.B);
  switch (p.c.page) {
    case 16: hipLaunchKernelGGL((cache_write_kernel<T, D, 16>), grid, dim3(64), 0, st, p); break;
    case 32: hipLaunchKernelGGL((cache_write_kernel<T, D, 32>), grid, dim3(128), 0, st, p); break;
    case 64: hipLaunchKernelGGL((cache_write_kernel<T, D, 64>), grid, dim3(256), 0, st, p); break;
    default: hipLaunchKernelGGL((cache_write_kernel<T, D, 128>), grid, dim3(512), 0, st, p); break;
  }
}

hipError_t launch_cache_write(CacheParams p, bool f16, hipStream_t st) {
  if (p.B == 0 || p.L == 0 || p.c.max_pages == 0) return hipSuccess;
  if (p.D == 64) f16 ? run_write<FP16, 64>(p, st) : run_write<BF16, 64>(p, st);
  else f16 ? run_write<FP16, 128>(p, st) : run_write<BF16, 128>(p, st);
  return hipGetLastError();
}

hipError_t launch_cache_read(CacheParams p, bool f16, hipStream_t st) {
  if (p.B == 0 || p.L == 0) return hipSuccess;
  const dim3 grid((uint32_t)((p.L + 14) / 16 + 1 + 3) / 4, (uint32_t)p.Hk, (uint32_t)p.B);
  if (p.D == 64) {
    if (f16) hipLaunchKernelGGL((cache_read_kernel<FP16, 64>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((cache_read_kernel<BF16, 64>), grid, dim3(256), 0, st, p);
  } else {
    if (f16) hipLaunchKernelGGL((cache_read_kernel<FP16, 128>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((cache_read_kernel<BF16, 128>), grid, dim3(256), 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace adaspa
