// Rotary positions on three axes (gfx950).
//
// Every head's first R = dim_t + dim_y + dim_x channels are taken in R / 2 pairs, the
// first dim_t / 2 of them turned by the token's t, the next dim_y / 2 by its y, the rest
// by its x: pair i of an axis of d channels turns by a = pos * theta^(-2 i / d),
//     u' = u cos a - v sin a,  v' = u sin a + v cos a,
// and by -a in the inverse direction, which is the gradient's (the rotation is
// orthogonal). Pairs are neighbouring channels (2p, 2p + 1) or the two halves' channels
// (p, p + R / 2).
//
// The angle in turns, pos * theta^(-2 i / d) / 2 pi, is formed and reduced to [-1/2, 1/2]
// in 64 bits (positions of long streams reach 10^5 turns, of which 32 bits would keep
// two decimals), its sine and cosine are taken in 32 bits.
//
// Bound by memory: every element is read and written once (40 + 40 heads of 720p, 3.1 GB:
// 568 us, 5.45 TB/s; a plain copy of 1 GiB reaches 5.13). All heads of a token share its
// angles, so a thread owns eight pairs of one token, forms their sines and cosines once
// and goes through a group of heads with them in registers.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "fva_geometry.h"
#include "fva_internal.h"

namespace fva {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename V>
struct Elem;
template <>
struct Elem<bf16x8> { typedef __bf16 type; };
template <>
struct Elem<f16x8> { typedef _Float16 type; };
template <>
struct Elem<f32x8> { typedef float type; };

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 32;  // eight threads per token, each 16 channels in two vectors
constexpr int kRopeUnroll = 4;   // heads in flight per thread
// Tokens of a launch: 2^32 threads and more in a row of workgroups are cut to 32 bits without an
// error (2^29 + 5 tokens ran as 32).
constexpr int64_t kRopeMost = (int64_t)1 << 28;

struct RopeParams {
  RopeTensor q, k;
  int batch, tokens;
  int H, W, t0, y0, x0;
  int pt, py, pairs;  // pairs turned by t, by y, all pairs (R / 2)
  double log2_theta;
  double inv_t, inv_y, inv_x;  // 2 / d of each axis
  bool halves;
  double sign;
  const int32_t* ids;
  int64_t ids_stride;
  int heads_per_group;  // heads (of Q and K together) a workgroup goes through
  int n0;               // first token of the launch
};

// The products that are fused with the sum are named, so that every copy of the code the
// compiler makes (heads in and behind the unrolled loop) rounds alike.
__device__ __forceinline__ void turn(float u, float v, float c, float s, float& ru, float& rv) {
  ru = fmaf(u, c, -(v * s));
  rv = fmaf(u, s, v * c);
}

template <typename V, bool STREAM>
__device__ __forceinline__ void turn_heads(const RopeTensor& x, int b, int n, int h0, int h1, int ca, int cb, bool halves,
                                           const float (&c)[8], const float (&s)[8], uint32_t act) {
  typedef typename Elem<V>::type T;
  const int64_t base = (int64_t)b * x.sb + (int64_t)n * x.sn;
  for (int h = h0; h < h1; h += kRopeUnroll) {
    V va[kRopeUnroll], vb[kRopeUnroll];
#pragma unroll
    for (int u = 0; u < kRopeUnroll; ++u) {
      const T* p = static_cast<const T*>(x.in) + base + (int64_t)min(h + u, h1 - 1) * x.sh;
      va[u] = *reinterpret_cast<const V*>(p + ca);
      vb[u] = *reinterpret_cast<const V*>(p + cb);
    }
#pragma unroll
    for (int u = 0; u < kRopeUnroll; ++u) {
      if (h + u >= h1) break;
      const f32x8 fa = __builtin_convertvector(va[u], f32x8);
      const f32x8 fb = __builtin_convertvector(vb[u], f32x8);
      f32x8 ra = fa, rb = fb;
      if (halves) {
        // pair e: (a[e], b[e])
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (act >> e & 1) {
            float u, v;
            turn(fa[e], fb[e], c[e], s[e], u, v);
            ra[e] = u;
            rb[e] = v;
          }
        }
      } else {
        // pairs 0..3: (a[2e], a[2e + 1]), pairs 4..7: (b[2e], b[2e + 1])
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float u, v;
          if (act >> e & 1) {
            turn(fa[2 * e], fa[2 * e + 1], c[e], s[e], u, v);
            ra[2 * e] = u;
            ra[2 * e + 1] = v;
          }
          if (act >> (4 + e) & 1) {
            turn(fb[2 * e], fb[2 * e + 1], c[4 + e], s[4 + e], u, v);
            rb[2 * e] = u;
            rb[2 * e + 1] = v;
          }
        }
      }
      T* p = static_cast<T*>(x.out) + base + (int64_t)(h + u) * x.sh;
      if constexpr (STREAM) {
        __builtin_nontemporal_store(__builtin_convertvector(ra, V), reinterpret_cast<V*>(p + ca));
        __builtin_nontemporal_store(__builtin_convertvector(rb, V), reinterpret_cast<V*>(p + cb));
      } else {
        *reinterpret_cast<V*>(p + ca) = __builtin_convertvector(ra, V);
        *reinterpret_cast<V*>(p + cb) = __builtin_convertvector(rb, V);
      }
    }
  }
}

template <typename V, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeParams P) {
  const uint32_t nth = (uint32_t)P.n0 + blockIdx.x * kRopeTokens + (threadIdx.x >> 3);
  const int unit = threadIdx.x & 7;
  const int b = blockIdx.z;
  if (nth >= (uint32_t)P.tokens) return;
  const int n = (int)nth;
  const int id = P.ids ? P.ids[(int64_t)b * P.ids_stride + n] : n;

  // The thread's two vectors of eight channels and their eight pairs. Halves: unit u
  // below R / 16 holds channels 8u.. of the first half and of the second, the others 16
  // channels behind R. Pairs: channels 8u.. and 64 + 8u.., pairs 4u.. and 32 + 4u...
  int ca, cb, p0, p1;
  if (P.halves) {
    const int r8 = P.pairs >> 3;  // units that turn
    ca = unit < r8 ? 8 * unit : 2 * P.pairs + 16 * (unit - r8);
    cb = unit < r8 ? P.pairs + 8 * unit : ca + 8;
    p0 = unit < r8 ? 8 * unit : P.pairs;
    p1 = p0 + 4;
  } else {
    ca = 8 * unit;
    cb = 64 + 8 * unit;
    p0 = 4 * unit;
    p1 = 32 + 4 * unit;
  }
  const int hw = P.H * P.W;
  const int t = id / hw;
  const int rem = id - t * hw;
  const int y = rem / P.W;
  const double pos_t = (double)t + P.t0, pos_y = (double)y + P.y0, pos_x = (double)(rem - y * P.W) + P.x0;
  float c[8], s[8];
  uint32_t act = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int p = (e < 4 ? p0 : p1 - 4) + e;
    const bool is_t = p < P.pt, is_y = p < P.pt + P.py;
    const double pos = is_t ? pos_t : is_y ? pos_y : pos_x;
    const int i = is_t ? p : is_y ? p - P.pt : p - P.pt - P.py;
    const double inv = is_t ? P.inv_t : is_y ? P.inv_y : P.inv_x;
    // turns: pos * theta^(-2 i / d) / 2 pi, the whole ones taken off
    double turns = P.sign * pos * (exp2(-(double)i * inv * P.log2_theta) * 0.15915494309189533577);
    turns -= rint(turns);
    sincospif(2.0f * (float)turns, &s[e], &c[e]);
    act |= (p < P.pairs && id >= 0 ? 1u : 0u) << e;
  }
  const int h0 = blockIdx.y * P.heads_per_group;
  const int h1 = min(h0 + P.heads_per_group, P.q.heads + P.k.heads);
  if (h0 < P.q.heads) turn_heads<V, STREAM>(P.q, b, n, h0, min(h1, P.q.heads), ca, cb, P.halves, c, s, act);
  if (h1 > P.q.heads)
    turn_heads<V, STREAM>(P.k, b, n, max(h0, P.q.heads) - P.q.heads, h1 - P.q.heads, ca, cb, P.halves, c, s, act);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a) {
  (void)hipGetLastError();
  const int heads = a.q.heads + a.k.heads;
  if (a.batch == 0 || heads == 0) return hipSuccess;
  RopeParams P;
  P.q = a.q;
  P.k = a.k;
  P.batch = a.batch;
  P.tokens = a.tokens;
  P.H = a.H;
  P.W = a.W;
  P.t0 = a.t0;
  P.y0 = a.y0;
  P.x0 = a.x0;
  P.pt = a.dim_t / 2;
  P.py = a.dim_y / 2;
  P.pairs = (a.dim_t + a.dim_y + a.dim_x) / 2;
  P.log2_theta = a.log2_theta;
  P.inv_t = a.dim_t ? 2.0 / a.dim_t : 0.0;
  P.inv_y = a.dim_y ? 2.0 / a.dim_y : 0.0;
  P.inv_x = a.dim_x ? 2.0 / a.dim_x : 0.0;
  P.halves = a.halves;
  P.sign = a.inverse ? -1.0 : 1.0;
  P.ids = a.ids;
  P.ids_stride = a.ids_stride;
  // Heads in groups of kRopeUnroll: forming a token's angles again for every four heads is
  // cheaper than a workgroup that walks through all of them (40 + 40 heads of 720p: 580 us,
  // against 628 with all heads in one group and 596 in ten of eight).
  const int groups = (heads + kRopeUnroll - 1) / kRopeUnroll;
  P.heads_per_group = (heads + groups - 1) / groups;
  // Outputs that the 256 MB last-level cache would not keep for the next call leave it
  // alone: 580 -> 568 us at 720p (1.5 GB). Smaller ones stay (4680 tokens of 48 heads in
  // fp32, 115 MB: 41.4 us, 44.4 past the cache).
  const int64_t bytes = (int64_t)a.batch * heads * a.tokens * kHeadDim * (a.dtype == 2 ? 4 : 2);
  const bool stream = bytes > ((int64_t)128 << 20);
  auto launch = [&](auto small, auto large) {
    for (int64_t n0 = 0; n0 < a.tokens; n0 += kRopeMost) {
      const int64_t tiles = (std::min(a.tokens - n0, kRopeMost) + kRopeTokens - 1) / kRopeTokens;
      const dim3 grid((unsigned)tiles, (heads + P.heads_per_group - 1) / P.heads_per_group, a.batch);
      P.n0 = (int)n0;
      if (stream)
        large<<<grid, kRopeThreads, 0, a.stream>>>(P);
      else
        small<<<grid, kRopeThreads, 0, a.stream>>>(P);
    }
  };
  switch (a.dtype) {
    case 0: launch(rope_kernel<bf16x8, false>, rope_kernel<bf16x8, true>); break;
    case 1: launch(rope_kernel<f16x8, false>, rope_kernel<f16x8, true>); break;
    default: launch(rope_kernel<f32x8, false>, rope_kernel<f32x8, true>); break;
  }
  return hipGetLastError();
}

}  // namespace fva
