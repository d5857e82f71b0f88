// What the attention kernels over the paged cache share (paged_attention.hip, paged_attention4.hip, paged_prompt.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.h"
#include "paged.h"
#include "paged_codes.h"

namespace kv {

constexpr float kSlack = 8.f;           // octaves a logit may exceed its reference
constexpr float kSlackScale = 0x1p-8f;  // of the weights

typedef __bf16 __attribute__((ext_vector_type(8))) bf16x8v;

// Workgroups of the kernels for up to 32 columns.
constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / 64;
constexpr int kMaxSplitRows = 2048;  // the blocks of a split are held in LDS
constexpr int kMaxSplitBlocks = kMaxSplitRows / 16;

typedef float __attribute__((ext_vector_type(4))) f32x4v;

__device__ __forceinline__ f32x4v mfma16(const u32x4_t& a, const u32x4_t& b, const f32x4v& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), c,
                                                 0, 0, 0);
}

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

// Eight floats as N bf16 terms that add up to them (8 bits of each per term).
template <int N> __device__ __forceinline__ void split_terms(const float (&x)[8], u32x4_t (&t)[N]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t[n][i] = pack_bf16(r[2 * i], r[2 * i + 1]);
      if (n + 1 < N) {
        r[2 * i] -= bf16_lo(t[n][i]);
        r[2 * i + 1] -= bf16_hi(t[n][i]);
      }
    }
}

// Largest value and sum over the four lanes of a column (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float column_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float column_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A load with the non-temporal bit where one workgroup alone reads a row (up to 16 columns, one group of them):
// 32 caches of 32768 rows 335 us, 363 without it.
template <bool kOnce, typename T> __device__ __forceinline__ T load_code(const T* p) {
  return kOnce ? __builtin_nontemporal_load(p) : *p;
}

// Weight of a partial sum of reference m under the joint reference M: 0 where no finite logit came in.
__device__ __forceinline__ float part_weight(float m, float M) {
  return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
}

// A / S, 0 for a token that sees no row (a NaN stays one).
template <int DT> __device__ __forceinline__ void store_out(void* out, int64_t at, float A, float S) {
  const float o = S == 0.f ? 0.f : A / S;
  if constexpr (DT == kDtBf16) static_cast<__bf16*>(out)[at] = (__bf16)o;
  else static_cast<float*>(out)[at] = o;
}

// What a problem's call sees: its tokens, and the cache rows that the batch's table can reach.
struct Span {
  int tok0, n_tok, len, cap;
  // rows visible to token j
  __device__ __forceinline__ int visible(int j) const { return max(0, min(len - n_tok + j + 1, cap)); }
};
__device__ __forceinline__ Span span_of(const PagedAttnArgs& a, int p) {
  Span s;
  s.tok0 = a.tok_off ? a.tok_off[p] : p;
  const int end = a.tok_off ? a.tok_off[p + 1] : p + 1;
  // none where the offsets fall or leave the call's rows (compared before they are subtracted: a fall of more than
  // 2^27 tokens times 16 heads would come out positive)
  const bool ok = s.tok0 >= 0 && end >= s.tok0 && end <= a.n_tok && end - s.tok0 <= a.max_q;
  s.n_tok = ok ? end - s.tok0 : 0;
  s.len = max(a.pc.len[p], 0);
  s.cap = (int)min((int64_t)a.pc.table_stride << a.pc.shift, (int64_t)a.pc.max_len);
  return s;
}

}  // namespace kv
