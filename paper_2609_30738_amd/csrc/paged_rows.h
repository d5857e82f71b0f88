// Rows into the blocks of a paged cache: what the kernels that write them share (paged_store.hip, paged_rotated.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "common.h"
#include "paged.h"
#include "paged_codes.h"

namespace kv {

constexpr int kStoreThreads = 256;

typedef uint16_t __attribute__((ext_vector_type(2))) u16x2_t;

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// The values of a 16-byte chunk.
template <int DT> __device__ __forceinline__ void chunk_values(const u32x4_t& u, float (&f)[16 / sizeof(typename Elem<DT>::T)]) {
  if constexpr (DT == kDtBf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]);
  }
}

template <int QT, bool kFinite, int EPT> __device__ __forceinline__ void store_chunk(uint8_t* dst, const float (&f)[EPT], float inv) {
  if constexpr (EPT == 8) {
    u32x2_t u;
    u[0] = encode4<QT, kFinite>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
    u[1] = encode4<QT, kFinite>(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
    *reinterpret_cast<u32x2_t*>(dst) = u;
  } else {
    *reinterpret_cast<uint32_t*>(dst) = encode4<QT, kFinite>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
  }
}

// ---- 4 bits: a row's 32 elements are the chunks of 4 (bf16) or 8 (fp32) consecutive lanes.

struct F32x4 {
  float f[4];
};

// Largest over the aligned groups of N lanes.
template <int N> __device__ __forceinline__ uint32_t group_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < N; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// A chunk of fp32 values, number c of row r, into a block of R rows (live: else nothing is written).  Every lane of the
// wave calls it.
template <int D, int EPT>
__device__ __forceinline__ void store_chunk4(uint8_t* codes, uint8_t* scale, int r, int R, int c, bool live, const float (&x)[EPT]) {
  constexpr int LANES = kGroup4 / EPT;
  float f[EPT];
  uint32_t amax = 0;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const uint32_t u = __float_as_uint(x[e]) & 0x7FFFFFFFu;
    f[e] = u > 0x7F800000u ? 0.f : x[e];  // a NaN becomes 0, an infinity the largest code
    amax = max(amax, u < 0x7F800000u ? u : 0u);
  }
  const uint32_t b = scale_byte4(group_max<LANES>(amax));
  const float s = scale4(b);
  uint32_t u = encode2_f32<0>(0u, f[0], f[1], s);
  u = encode2_f32<1>(u, f[2], f[3], s);
  if constexpr (EPT == 8) {
    u = encode2_f32<2>(u, f[4], f[5], s);
    u = encode2_f32<3>(u, f[6], f[7], s);
  }
  if (live) {
    uint8_t* to = codes + r * (D / 2) + c * (EPT / 2);
    if constexpr (EPT == 8) *reinterpret_cast<uint32_t*>(to) = u;
    else *reinterpret_cast<uint16_t*>(to) = (uint16_t)u;
    if (c % LANES == 0) scale[c / LANES * R + r] = (uint8_t)b;
  }
}

// The same for eight bf16 values, converted as they are.
template <int D>
__device__ __forceinline__ void store_chunk4_bf16(uint8_t* codes, uint8_t* scale, int r, int R, int c, bool live, u32x4_t x) {
  constexpr int LANES = kGroup4 / 8;
  uint32_t top = 0;  // without the signs, two at a time
#pragma unroll
  for (int w = 0; w < 4; ++w)
    top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, top), __builtin_bit_cast(u16x2_t, x[w] & 0x7FFF7FFFu)));
  uint32_t amax = max(top << 16, top & 0xFFFF0000u);
  if (__ballot(amax >= 0x7F800000u)) {
    amax = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t u = (h ? x[w] & 0xFFFF0000u : x[w] << 16) & 0x7FFFFFFFu;
        if (u > 0x7F800000u) x[w] &= h ? 0x0000FFFFu : 0xFFFF0000u;
        amax = max(amax, u < 0x7F800000u ? u : 0u);
      }
  }
  const uint32_t b = scale_byte4(group_max<LANES>(amax));
  const uint32_t u = encode8_bf16(x, scale4(b));
  if (live) {
    *reinterpret_cast<uint32_t*>(codes + r * (D / 2) + c * 4) = u;
    if (c % LANES == 0) scale[c / LANES * R + r] = (uint8_t)b;
  }
}

// Codes and scales of a unit, a block's rows of one head.
template <int QT> using ScaleOf = std::conditional_t<QT == kQtE2m1, uint8_t, float>;
template <int QT, int D, int SHIFT> __device__ __forceinline__ uint8_t* unit_codes(uint8_t* pool, int64_t unit) {
  return pool + (unit << SHIFT) * (QT == kQtE2m1 ? D / 2 : D);
}
template <int QT, int D, int SHIFT> __device__ __forceinline__ ScaleOf<QT>* unit_scale(void* pool, int64_t unit) {
  return static_cast<ScaleOf<QT>*>(pool) + (QT == kQtE2m1 ? (unit << SHIFT) * (D / kGroup4) : unit);
}

// ---- rows of a block

// Chunks of a lane in a block of 1 << SHIFT rows.
template <int DT, int D, int SHIFT> constexpr int kChunks = ((D * (int)sizeof(typename Elem<DT>::T)) << SHIFT) / 1024;
// Chunks that a lane holds in registers; blocks of more (fp32, 128 rows of 128) are read twice: 89,000 fp32 rows (910 MB)
// 335 us, in blocks of 64 rows 279.
constexpr int kHeldChunks = 32;

// The scale of a block that holds row0 rows at scale `old` and gets rows whose own scale is s: the held codes move
// by whole binades where s is larger.  Every lane of the wave calls it.
template <int QT, int D> __device__ __forceinline__ float grown_scale(uint8_t* codes, int row0, float old, float s) {
  if (row0 == 0) return s;
  if (old >= s && old < INFINITY) return old;
  const float f = old > 0.f && old < s ? old * inv_scale(s) : 0.f;
  u32x4_t* at = reinterpret_cast<u32x4_t*>(codes);
  for (int i = threadIdx.x & 63; i < row0 * D / 16; i += 64) {
    u32x4_t u = at[i];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float y[4];
      decode4<QT>(u[w], y);
      u[w] = encode4<QT, false>(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
    }
    at[i] = u;
  }
  return s;
}

// store_rows for any values: read twice, infinities and NaNs apart.
template <int DT, int QT, int D, typename Load>
__device__ __forceinline__ void store_rows_any(uint8_t* codes, float* scale, int row0, int n, Load load) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH;
  const int lane = threadIdx.x & 63, c = lane % CH, rr = lane / CH;
  const float old = row0 > 0 ? *scale : 0.f;
  uint32_t amax = 0;
#pragma unroll 4
  for (int i = 0; i * RPP < n; ++i) {
    float f[EPT];
    chunk_values<DT>(load(i), f);
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const uint32_t u = __float_as_uint(f[e]) & 0x7FFFFFFFu;
      amax = max(amax, u < 0x7F800000u ? u : 0u);
    }
  }
  const float s = grown_scale<QT, D>(codes, row0, old, block_scale<QT>(wave_max_u32(amax))), inv = inv_scale(s);
#pragma unroll 4
  for (int i = 0; i * RPP < n; ++i) {
    float f[EPT];
    chunk_values<DT>(load(i), f);
    if (i * RPP + rr < n) store_chunk<QT, false>(codes + (row0 + i * RPP + rr) * D + c * EPT, f, inv);
  }
  if (lane == 0) *scale = s;
}

// Rows row0 .. row0 + n - 1 of one block and head, 4-bit: chunks as in store_rows, in batches of kBatch4, whose loads are in
// flight together.  Every lane of the wave calls it.
constexpr int kBatch4 = 8;
template <int DT, int D, int SHIFT, typename Load>
__device__ __forceinline__ void store_rows4(uint8_t* codes, uint8_t* scale, int row0, int n, Load load) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH;
  const int lane = threadIdx.x & 63, c = lane % CH, rr = lane / CH;
  constexpr int NC = kChunks<DT, D, SHIFT>, NB = NC < kBatch4 ? NC : kBatch4;
  for (int i0 = 0; i0 * RPP < n; i0 += NB) {
    u32x4_t x[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      x[i] = u32x4_t{0u, 0u, 0u, 0u};
      if ((i0 + i) * RPP < n) x[i] = load(i0 + i);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int r = (i0 + i) * RPP + rr;
      if ((i0 + i) * RPP >= n) break;
      if constexpr (DT == kDtBf16) store_chunk4_bf16<D>(codes, scale, row0 + r, 1 << SHIFT, c, r < n, x[i]);
      else store_chunk4<D, 4>(codes, scale, row0 + r, 1 << SHIFT, c, r < n, __builtin_bit_cast(F32x4, x[i]).f);
    }
  }
}

// Rows row0 .. row0 + n - 1 of one block and head; the block holds row0 rows already.  load(i): the lane's 16-byte
// chunk, number lane % CH of row i RPP + lane / CH of the new ones (zeros past the last).  Every lane of the wave
// calls it.
template <int DT, int QT, int D, int SHIFT, typename Load>
__device__ __forceinline__ void store_rows(uint8_t* codes, ScaleOf<QT>* scale, int row0, int n, Load load) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH;
  constexpr int NC = kChunks<DT, D, SHIFT>;
  if constexpr (QT == kQtE2m1) {
    store_rows4<DT, D, SHIFT>(codes, scale, row0, n, load);
  } else if constexpr (NC > kHeldChunks) {
    store_rows_any<DT, QT, D>(codes, scale, row0, n, load);
  } else {
    const int lane = threadIdx.x & 63, c = lane % CH, rr = lane / CH;
    const float old = row0 > 0 ? *scale : 0.f;
    u32x4_t x[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      x[i] = u32x4_t{0u, 0u, 0u, 0u};
      if (i * RPP < n) x[i] = load(i);
    }
    uint32_t amax = 0;  // without the signs; two bf16 at a time
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (DT == kDtBf16) {
          const u16x2_t u = __builtin_bit_cast(u16x2_t, x[i][w] & 0x7FFF7FFFu);
          amax = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, amax), u));
        } else {
          amax = max(amax, x[i][w] & 0x7FFFFFFFu);
        }
      }
    if constexpr (DT == kDtBf16) amax = max(amax << 16, amax & 0xFFFF0000u);
    amax = wave_max_u32(amax);
    if (amax >= 0x7F800000u) {  // an infinity or a NaN among them
      store_rows_any<DT, QT, D>(codes, scale, row0, n, load);
      return;
    }
    const float s = grown_scale<QT, D>(codes, row0, old, block_scale<QT>(amax)), inv = inv_scale(s);
    uint8_t* to = codes + row0 * D + rr * D + c * EPT;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      // (a value's conversion is not kept from the first pass over the chunks: registers)
      asm volatile("" : "+v"(x[i][0]), "+v"(x[i][1]), "+v"(x[i][2]), "+v"(x[i][3]));
      if (i * RPP + rr < n) {
        float f[EPT];
        chunk_values<DT>(x[i], f);
        store_chunk<QT, true>(to + i * RPP * D, f, inv);
      }
    }
    if (lane == 0) *scale = s;
  }
}

template <int V> using Int = std::integral_constant<int, V>;

// f(dtype, qtype, d, shift) of integral constants.
template <typename F> hipError_t dispatch(const Paged& pc, F f) {
  auto shift = [&](auto dt, auto qt, auto d) {
    switch (pc.shift) {
      case 4: return f(dt, qt, d, Int<4>{});
      case 5: return f(dt, qt, d, Int<5>{});
      case 6: return f(dt, qt, d, Int<6>{});
      default: return f(dt, qt, d, Int<7>{});
    }
  };
  auto d = [&](auto dt, auto qt) { return pc.d == 64 ? shift(dt, qt, Int<64>{}) : shift(dt, qt, Int<128>{}); };
  auto q = [&](auto dt) {
    if (pc.qtype == kQtE2m1) return d(dt, Int<kQtE2m1>{});
    return pc.qtype == kQtE4m3 ? d(dt, Int<kQtE4m3>{}) : d(dt, Int<kQtInt8>{});
  };
  return pc.dtype == kDtBf16 ? q(Int<kDtBf16>{}) : q(Int<kDtF32>{});
}

}  // namespace kv
