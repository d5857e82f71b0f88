// Rotation of rows by their positions (kv_rotate).
//
// rotate_kernel: one workgroup of four waves per (a few tokens, part of the heads).  The turns of the tokens' pairs are the
//   same for every head: the workgroup forms them once, in 64 bits, beside the first rows' loads, and keeps them in LDS; a
//   lane holds those of its chunks in registers while it goes over the heads.
//   Bound by HBM: 31744 tokens of 32 heads of 128 (520 MB read and written) 91 us, 5.7 TB/s; in fp32 186; 64 tokens 6.2, of
//   which the kernel takes 3.4.
#include "rotary.h"

namespace kv {

template <int DT, int D> __global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a) {
  extern __shared__ __align__(16) float4 lds[];
  rotate_group<DT, D>(a, blockIdx.x / a.parts, (int)(blockIdx.x % a.parts), lds);
}

namespace {

template <int DT, int D> hipError_t rotate(RotateArgs a, hipStream_t stream) {
  const int64_t groups = ((int64_t)a.n_tok + kRotateRows<DT, D> - 1) / kRotateRows<DT, D>;
  a.parts = rotate_parts(groups, a.heads);
  const size_t lds = turn_bytes(a.rot.rot, kRotateRows<DT, D>);
  rotate_kernel<DT, D><<<(unsigned)(groups * a.parts), kRotateThreads, lds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(int dtype, int d, const RotateArgs& a, hipStream_t stream) {
  if (dtype == kDtBf16) return d == 64 ? rotate<kDtBf16, 64>(a, stream) : rotate<kDtBf16, 128>(a, stream);
  return d == 64 ? rotate<kDtF32, 64>(a, stream) : rotate<kDtF32, 128>(a, stream);
}

}  // namespace kv
