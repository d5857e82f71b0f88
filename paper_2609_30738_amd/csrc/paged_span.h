// What the two attention kernels over the paged cache share (paged_attention.hip, paged_prompt.hip).
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

// Two floats as a bf16 pair, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2_t r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
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
