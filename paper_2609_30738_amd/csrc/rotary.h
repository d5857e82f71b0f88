// Rotation of rows by their positions (kv_rotate, kv_paged_append_rotated): the angles and the rotated rows.
//
// Of a pair of elements (a, b) at position p and frequency f: c = factor cos(p f), s = factor sin(p f),
//   a' = a c - b s,  b' = b c + a s.
// The angle is formed and reduced in 64 bits, since at far positions a 32-bit one has lost its fraction (2^24 radians are
// steps of 1), and so are its cosine and sine, by their power series on [-pi/4, pi/4]: remainders below 2^-47, so that what
// is rounded to 32 bits is off by half a step, and a rotation on its way into a cache gives the bits that one by itself gives.
// Their products with the row are rounded one by one in 32 bits, no two fused, for the same reason.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "paged.h"
#include "paged_codes.h"
#include "paged_rows.h"

namespace kv {

constexpr int kRotateThreads = 256;

// (factor cos, factor sin) of an angle in radians.
__device__ __forceinline__ float2 turn(double angle, float factor) {
  constexpr double kTwoOverPi = 0.6366197723675814;     // 2 / pi
  constexpr double kHalfPi = 1.5707963267948966;        // pi / 2, to 53 bits
  constexpr double kHalfPiRest = 6.123233995736766e-17;  // and what is left of it
  const double k = __builtin_rint(angle * kTwoOverPi);
  // (exact: k times the first part is taken in one fused step, and what is left has few bits)
  double r = __builtin_fma(-k, kHalfPi, angle);
  r = __builtin_fma(-k, kHalfPiRest, r);
  const double z = r * r;
  double s = -1.0 / 1307674368000.0;  // 1/15!
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  s = __builtin_fma(s * z, r, r);
  double c = -1.0 / 87178291200.0;  // 1/14!
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  // the quarter: k modulo 4
  const int q = (int)(k - 4.0 * __builtin_floor(k * 0.25));
  const double x = q & 1 ? s : c, y = q & 1 ? c : s;
  return make_float2((float)((q == 1 || q == 2 ? -x : x) * factor), (float)((q >= 2 ? -y : y) * factor));
}

// The turns of n tokens' pairs, tab[token][rot / 2], by the threads of a workgroup.
__device__ __forceinline__ void fill_turns(float2* tab, const Rotary& rot, const int32_t* pos, int n) {
  const int half = rot.rot >> 1;
  for (int i = threadIdx.x; i < n * half; i += kRotateThreads) {
    const int t = i / half, f = i - t * half;
    float2 cs = turn((double)pos[t] * rot.freq[f], rot.factor);
    cs.y *= rot.sign;
    tab[i] = cs;
  }
}

// The pairs (a[e], b[e]) turned by cs[e].
template <int N> __device__ __forceinline__ void turn_pairs(float (&a)[N], float (&b)[N], const float2 (&cs)[N]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float x = a[e] * cs[e].x, y = b[e] * cs[e].y, u = b[e] * cs[e].x, v = a[e] * cs[e].y;
    a[e] = x - y;
    b[e] = u + v;
  }
}

// A row's chunk (16 bytes) number c, turned: every lane of the wave calls it, the lanes of a row beside each other.  turns:
// those of the row's pairs.
template <int DT, int D> struct TurnChunk {
  static constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT;
  bool interleaved, in, low;
  int partner, first;  // the lane of the other halves of the pairs, and the first pair
  __device__ __forceinline__ explicit TurnChunk(const Rotary& rot) {
    const int lane = threadIdx.x & 63, c = lane % CH, half = rot.rot / EPT / 2;
    interleaved = rot.interleaved;
    in = c < 2 * half;
    low = c < half;
    partner = !in ? lane : low ? lane + half : lane - half;
    first = !in ? 0 : interleaved ? c * EPT / 2 : (low ? c : c - half) * EPT;
  }
  __device__ __forceinline__ void operator()(const u32x4_t& x, const float2* turns, float (&f)[EPT]) const {
#pragma clang fp contract(off)
    chunk_values<DT>(x, f);
    if (interleaved) {
      float a[EPT / 2], b[EPT / 2];
      float2 cs[EPT / 2];
#pragma unroll
      for (int e = 0; e < EPT / 2; ++e) {
        a[e] = f[2 * e];
        b[e] = f[2 * e + 1];
        cs[e] = turns[first + e];
      }
      turn_pairs(a, b, cs);
#pragma unroll
      for (int e = 0; e < EPT; ++e) f[e] = !in ? f[e] : e & 1 ? b[e / 2] : a[e / 2];
    } else {
      u32x4_t y;
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] = (uint32_t)__shfl((int)x[w], partner, 64);
      float g[EPT];
      chunk_values<DT>(y, g);
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        const float2 cs = turns[first + e];
        const float u = f[e] * cs.x, v = g[e] * cs.y;
        const float t = low ? u - v : u + v;
        f[e] = in ? t : f[e];
      }
    }
  }
};

// The tokens that a workgroup of kv_rotate takes at once: a lane has two chunks of a row, whose pairs lie in these two.
template <int DT, int D> constexpr int kRotateRows = 64 / (D * (int)sizeof(typename Elem<DT>::T) / 32);

// The heads of a group of kRotateRows tokens that fall to one part: waves and parts take heads in turn, kRotateBatch of them in
// flight.  tab: LDS of the group's turns.  Every thread of the workgroup calls it.
constexpr int kRotateBatch = 4;
template <int DT, int D> __device__ __forceinline__ void rotate_group(const RotateArgs& a, int64_t group, int part, float2* tab) {
  using E = typename Elem<DT>::T;
  constexpr int EPT = 16 / (int)sizeof(E), LPR = D / EPT / 2, RW = kRotateRows<DT, D>, kStep = kRotateThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane / LPR, j = lane % LPR;
  const int64_t t0 = group * RW;
  const int n = (int)(a.n_tok - t0 < RW ? a.n_tok - t0 : RW);
  const int half = a.rot.rot >> 1;
  const bool in = EPT * j < half, live = row < n;
  // half: chunks of the pairs' first and second elements; interleaved, and behind the rotated ones: neighbours
  const int c0 = in && !a.rot.interleaved ? j : 2 * j, c1 = in && !a.rot.interleaved ? j + half / EPT : 2 * j + 1;
  const int64_t t = t0 + (live ? row : 0);
  const E* x = static_cast<const E*>(a.x) + t * a.x_stride;
  E* out = static_cast<E*>(a.out) + t * a.out_stride;
  u32x4_t xa[kRotateBatch], xb[kRotateBatch];
  const int step = kStep * a.parts;
  int h0 = part * kStep + wave;
  auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kRotateBatch; ++i) {
      const int h = h0 + i * step;
      if (h < a.heads && live) {
        xa[i] = *reinterpret_cast<const u32x4_t*>(x + h * D + c0 * EPT);
        xb[i] = *reinterpret_cast<const u32x4_t*>(x + h * D + c1 * EPT);
      }
    }
  };
  load();
  fill_turns(tab, a.rot, a.pos + t0, n);
  __syncthreads();
  float2 cs[EPT];
#pragma unroll
  for (int e = 0; e < EPT; ++e) cs[e] = in && live ? tab[row * half + EPT * j + e] : make_float2(1.f, 0.f);
  for (; h0 < a.heads; h0 += kRotateBatch * step, load()) {
#pragma unroll
    for (int i = 0; i < kRotateBatch; ++i) {
      const int h = h0 + i * step;
      if (h >= a.heads || !live) continue;
      if (in) {
        float f[EPT], g[EPT];
        chunk_values<DT>(xa[i], f);
        chunk_values<DT>(xb[i], g);
        if (a.rot.interleaved) {
          float p[EPT], q[EPT];
#pragma unroll
          for (int e = 0; e < EPT; ++e) {
            p[e] = e < EPT / 2 ? f[2 * e] : g[2 * e - EPT];
            q[e] = e < EPT / 2 ? f[2 * e + 1] : g[2 * e + 1 - EPT];
          }
          turn_pairs(p, q, cs);
#pragma unroll
          for (int e = 0; e < EPT; ++e) {
            (e < EPT / 2 ? f[2 * e] : g[2 * e - EPT]) = p[e];
            (e < EPT / 2 ? f[2 * e + 1] : g[2 * e + 1 - EPT]) = q[e];
          }
        } else {
          turn_pairs(f, g, cs);
        }
        if constexpr (DT == kDtBf16) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            xa[i][w] = pack_bf16(f[2 * w], f[2 * w + 1]);
            xb[i][w] = pack_bf16(g[2 * w], g[2 * w + 1]);
          }
        } else {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            xa[i][w] = __float_as_uint(f[w]);
            xb[i][w] = __float_as_uint(g[w]);
          }
        }
      }
      *reinterpret_cast<u32x4_t*>(out + h * D + c0 * EPT) = xa[i];
      *reinterpret_cast<u32x4_t*>(out + h * D + c1 * EPT) = xb[i];
    }
  }
}

// Workgroups that share the heads of a group of tokens: as many as fill the chip.
inline int rotate_parts(int64_t groups, int heads) {
  const int most = (heads + kRotateThreads / 64 - 1) / (kRotateThreads / 64);
  const int64_t want = (2048 + groups - 1) / groups;
  return (int)(want < most ? want : most);
}

}  // namespace kv
