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

// Turns in LDS: those of a token's pairs two by two, 16 bytes, in the order that a wave's lanes read them without conflicts:
// with K of them to a lane, all lanes' first ones come first.  Tokens are kTurnPad apart beyond that.
constexpr int kTurnPad = 4;
struct Turns {
  float4* tab;
  int quads;   // of a token
  int lanes;   // that share them
  int stride;  // between two tokens
  int per, log_per;  // of a lane
  // EPT: elements of a chunk; a lane's chunk holds both elements of a pair (interleaved), or one of each of EPT pairs
  __device__ __forceinline__ Turns(float4* lds, const Rotary& rot, int pairs_of_lane) {
    tab = lds;
    quads = rot.rot >> 2;
    per = pairs_of_lane >> 1;
    log_per = per == 4 ? 2 : per == 2 ? 1 : 0;
    lanes = quads >> log_per;
    stride = quads + kTurnPad;
  }
  // n tokens' turns, by the threads of a workgroup: a thread keeps to two pairs, and takes every eighth token
  __device__ __forceinline__ void fill(const Rotary& rot, const int32_t* pos, int n) const {
    const int q = threadIdx.x & 31;
    if (q >= quads) return;
    const double f0 = rot.freq[2 * q], f1 = rot.freq[2 * q + 1];
    float4* to = tab + (q & (per - 1)) * lanes + (q >> log_per);
    int t = threadIdx.x >> 5;
    int next = t < n ? pos[t] : 0;
    for (; t < n; t += kRotateThreads / 32) {
      const double p = (double)next;
      if (t + kRotateThreads / 32 < n) next = pos[t + kRotateThreads / 32];
      const float2 x = turn(p * f0, rot.factor), y = turn(p * f1, rot.factor);
      to[t * stride] = make_float4(x.x, x.y * rot.sign, y.x, y.y * rot.sign);
    }
  }
  // those of lane l's pairs of token t
  template <int N> __device__ __forceinline__ void get(int t, int l, float2 (&cs)[N]) const {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      const float4 x = tab[t * stride + k * lanes + l];
      cs[2 * k] = make_float2(x.x, x.y);
      cs[2 * k + 1] = make_float2(x.z, x.w);
    }
  }
};
// LDS bytes of n tokens' turns.
inline size_t turn_bytes(int rot, int n) { return (size_t)n * (rot / 4 + kTurnPad) * sizeof(float4); }

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

// A row's chunk (16 bytes) turned: pairs of neighbours (interleaved), or of elements half the rotated ones apart, whose other
// halves another lane of the row holds.  Every lane of the wave calls it, the lanes of a row beside each other.
template <int DT, int D, bool INTERLEAVED> struct TurnChunk {
  static constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, PAIRS = INTERLEAVED ? EPT / 2 : EPT;
  bool in, all;       // whether the chunk is rotated, and every chunk is
  uint32_t flip;      // the sign bits of the other halves of the pairs
  int partner, mine;  // the lane that has these, and the lane's place among those that share a row's turns
  __device__ __forceinline__ explicit TurnChunk(const Rotary& rot) {
    const int lane = threadIdx.x & 63, c = lane % CH, half = rot.rot / EPT / 2;
    in = c < 2 * half;
    all = rot.rot == D;
    partner = !in ? lane : c < half ? lane + half : lane - half;
    flip = c < half ? (DT == kDtBf16 ? 0x80008000u : 0x80000000u) : 0u;
    mine = !in ? 0 : INTERLEAVED || c < half ? c : c - half;
  }
  __device__ __forceinline__ void operator()(const u32x4_t& x, const float2 (&cs)[PAIRS], float (&f)[EPT]) const {
#pragma clang fp contract(off)
    chunk_values<DT>(x, f);
    float t[EPT];
    if constexpr (INTERLEAVED) {
#pragma unroll
      for (int e = 0; e < EPT / 2; ++e) {
        const float a = f[2 * e] * cs[e].x, b = f[2 * e + 1] * cs[e].y, u = f[2 * e + 1] * cs[e].x, v = f[2 * e] * cs[e].y;
        t[2 * e] = a - b;
        t[2 * e + 1] = u + v;
      }
    } else {
      u32x4_t y;
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] = (uint32_t)__shfl((int)x[w], partner, 64) ^ flip;
      float g[EPT];
      chunk_values<DT>(y, g);
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        const float a = f[e] * cs[e].x, b = g[e] * cs[e].y;
        t[e] = a + b;
      }
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) f[e] = all || in ? t[e] : f[e];
  }
};

// The tokens that a workgroup of kv_rotate takes at once: a lane has two chunks of a row, whose pairs lie in these two.
template <int DT, int D> constexpr int kRotateRows = 64 / (D * (int)sizeof(typename Elem<DT>::T) / 32);

// The heads of a group of kRotateRows tokens that fall to one part: waves and parts take heads in turn, kRotateBatch of them in
// flight.  lds: of the group's turns.  Every thread of the workgroup calls it.
constexpr int kRotateBatch = 4;
template <int DT, int D> __device__ __forceinline__ void rotate_group(const RotateArgs& a, int64_t group, int part, float4* lds) {
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
  const Turns turns(lds, a.rot, EPT);
  turns.fill(a.rot, a.pos + t0, n);
  __syncthreads();
  float2 cs[EPT];
  turns.get(live ? row : 0, in ? j : 0, cs);
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

// Workgroups that share the heads of a group of tokens, each with the group's turns of its own: many short ones keep more
// loads in flight than as many as the chip holds.  31744 tokens of 32 heads 91 us with 16384 workgroups, 104 with 2048, 94 with
// 4096, 96 with a head to a wave; short calls take a head to a wave.
inline int rotate_parts(int64_t groups, int heads) {
  const int most = (heads + kRotateThreads / 64 - 1) / (kRotateThreads / 64);
  const int64_t want = (16384 + groups - 1) / groups;
  return (int)(want < most ? want : most);
}

}  // namespace kv
