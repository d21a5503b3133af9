// Rotary positions of queries and keys (gfx950).
//
//   (u, w) -> m (u cos a - w sin a, u sin a + w cos a),  a = position f_pair
//
// for the pairs (u, w) of the first 2 P elements of a head; the rest is copied.
// The backward pass turns the other way, by the same factor m.
#include "cross_tile.hpp"
#include "rotary.hpp"

namespace adaspa {

namespace {

// V elements of 16 bits, one access.
template <int V>
struct Vec {
  uint32_t w[(V + 1) / 2];
  __device__ __forceinline__ void load(const u16* p) {
    if constexpr (V == 1) w[0] = *p;
    else __builtin_memcpy(w, __builtin_assume_aligned(p, 2 * V), 2 * V);
  }
  __device__ __forceinline__ void store(u16* p) const {
    if constexpr (V == 1) *p = (u16)w[0];
    else __builtin_memcpy(__builtin_assume_aligned(p, 2 * V), w, 2 * V);
  }
};

}  // namespace

// A work item is V pairs (or 2 V of the elements that are copied) of one token,
// for all heads of a group, so that an angle's sine and cosine are formed once
// for many heads.  Angles: position times revolutions per position in fp64, whose
// nearest whole number is taken away exactly; in fp32 a position of 1e6 would
// leave 0.06 radians of doubt.  What is left, at most half a revolution, is what
// the sine and cosine units take.  Both vectors of a head are read before either is
// written, so the result may take the input's place.
//
// Bound by its bytes: q and k of 24 heads, 110,080 tokens, d 128 by three axes 541 us, 5.0 TB/s (a
// large copy 5.05); 4,999 tokens of 12 + 4 heads of d 64 by 40 elements (vectors of 4) 14 us.  A token
// of each of 64 sequences takes 3 us, a launch's own time.
template <class T, int V, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p) {
  constexpr int U = 4;                                     // heads on their way at a time
  const uint32_t blocks = gridDim.x / p.groups, group = blockIdx.x / blocks;
  const uint32_t item = (blockIdx.x % blocks) * 256 + threadIdx.x;
  if (item >= p.items) return;
  const int c = item % p.chunks, t = item / p.chunks % p.L, b = item / p.chunks / p.L;
  const bool turned = c * V < p.P;
  const int e0 = turned && !INTER ? c * V : 2 * c * V, e1 = turned && !INTER ? p.P + c * V : 2 * c * V + V;

  float cs[V], sn[V];
  if (turned) {
    const int64_t off = p.offset + (p.offsets ? p.offsets[b] : 0);
    const int32_t* at = p.positions + b * p.pos_b + t * p.pos_t;
    double pos[kMaxRotaryAxes];
    pos[0] = (double)(off + (p.positions ? at[0] : t));
#pragma unroll
    for (int a = 1; a < kMaxRotaryAxes; ++a) pos[a] = a < p.axes ? (double)(off + at[a]) : 0.0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int pair = c * V + e;
      double x = pos[0];
#pragma unroll
      for (int a = 1; a < kMaxRotaryAxes; ++a)
        if (a < p.axes && pair >= p.axis_end[a - 1]) x = pos[a];
      x *= p.turns[pair];
      const float turn = (float)(x - __builtin_rint(x));
      cs[e] = __builtin_amdgcn_cosf(turn) * p.cos_by;
      sn[e] = __builtin_amdgcn_sinf(turn) * p.sin_by;
    }
  }

  const int h0 = group * p.per_group, h1 = h0 + p.per_group;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const int before = which ? p.heads[0] : 0;
    const int lo = h0 > before ? h0 - before : 0, hi = h1 - before < p.heads[which] ? h1 - before : p.heads[which];
    const u16* x = p.x[which] + b * p.sx[which].b + t * p.sx[which].t;
    u16* y = p.y[which] + b * p.sy[which].b + t * p.sy[which].t;
    for (int h = lo; h < hi; h += U) {
      Vec<V> u[U], w[U];
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (h + i < hi) {
          u[i].load(x + (h + i) * p.sx[which].h + e0);
          w[i].load(x + (h + i) * p.sx[which].h + e1);
        }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (h + i < hi) {
          if (turned) {
            float f[2 * V];
            if constexpr (V == 1) {
              f[0] = T::load(&u[i].w[0], 0);
              f[1] = T::load(&w[i].w[0], 0);
            } else {
#pragma unroll
              for (int j = 0; j < V / 2; ++j) {
                T::unpack(u[i].w[j], f[2 * j], f[2 * j + 1]);
                T::unpack(w[i].w[j], f[V + 2 * j], f[V + 2 * j + 1]);
              }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const int k0 = INTER ? 2 * e : e, k1 = INTER ? 2 * e + 1 : V + e;
              const float a = f[k0], d = f[k1];
              f[k0] = a * cs[e] - d * sn[e];
              f[k1] = a * sn[e] + d * cs[e];
            }
            if constexpr (V == 1) {
              u[i].w[0] = T::pack(f[0], 0.f) & 0xFFFFu;
              w[i].w[0] = T::pack(f[1], 0.f) & 0xFFFFu;
            } else {
#pragma unroll
              for (int j = 0; j < V / 2; ++j) {
                u[i].w[j] = T::pack(f[2 * j], f[2 * j + 1]);
                w[i].w[j] = T::pack(f[V + 2 * j], f[V + 2 * j + 1]);
              }
            }
          }
          u[i].store(y + (h + i) * p.sy[which].h + e0);
          w[i].store(y + (h + i) * p.sy[which].h + e1);
        }
    }
  }
}

template <class T, int V>
static void run_rotary(const RotaryParams& p, bool interleaved, uint32_t n, hipStream_t st) {
  if (interleaved) hipLaunchKernelGGL((rotary_kernel<T, V, true>), dim3(n), dim3(256), 0, st, p);
  else hipLaunchKernelGGL((rotary_kernel<T, V, false>), dim3(n), dim3(256), 0, st, p);
}
template <class T>
static void run_rotary(const RotaryParams& p, bool interleaved, uint32_t n, hipStream_t st) {
  switch (rotary_vector(p.D, p.P)) {
    case 8: return run_rotary<T, 8>(p, interleaved, n, st);
    case 4: return run_rotary<T, 4>(p, interleaved, n, st);
    case 2: return run_rotary<T, 2>(p, interleaved, n, st);
    default: return run_rotary<T, 1>(p, interleaved, n, st);
  }
}

hipError_t launch_rotary(RotaryParams p, bool f16, bool interleaved, hipStream_t st) {
  const int heads = p.heads[0] + p.heads[1];
  p.chunks = p.D / 2 / rotary_vector(p.D, p.P);
  p.items = (uint32_t)((int64_t)p.B * p.L * p.chunks);
  if (p.items == 0 || heads == 0) return hipSuccess;
  // Few tokens: heads are divided until there are 65,536 threads, four waves a CU (500 tokens of 24 + 24
  // heads of d 128, us: 4.3; up to 16,384 threads 5.8, 262,144 4.8; 300 tokens of 64 + 8: 4.3, 5.9, 4.7).
  int64_t groups = (65536 + (int64_t)p.items - 1) / p.items;
  groups = groups < heads ? groups : heads;
  p.per_group = (int)((heads + groups - 1) / groups);
  p.groups = (heads + p.per_group - 1) / p.per_group;
  const uint32_t n = (p.items + 255) / 256 * (uint32_t)p.groups;
  if (f16) run_rotary<FP16>(p, interleaved, n, st);
  else run_rotary<BF16>(p, interleaved, n, st);
  return hipGetLastError();
}

}  // namespace adaspa
