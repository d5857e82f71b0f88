// The rows of a paged cache as contiguous keys and values (kv_paged_rows), in the layout that an eviction takes.
//
// paged_rows_kernel: one workgroup of four waves per (64 rows, kv head, problem), a wave 16 rows of K and of V, whose block
//   is the wave's.  A lane writes 16 bytes; the codes of all 16 rows are in flight together.
//   Bound by HBM: 44,400 rows of 8 heads of 128 from 4 bits (48 MB read, 182 MB written) 37 us, 6.2 TB/s, 15,400 rows 16.7;
//   24 caches of up to 131 rows 4.7: offsets, tables and lengths in one step of loads, codes and scales in another.  58,584 rows
//   from 8 bits 70 us, 5.2 TB/s (from 4 56), into fp32 121 (121), of 64 elements 28 (24).  Workgroups are launched for the bound on the
//   lengths: 2048 caches of 100 rows 233 us under a bound of 128, 2785 under 32768.
#include <math.h>

#include <algorithm>

#include "paged.h"
#include "paged_rows.h"
#include "paged_span.h"

namespace kv {

struct ReadArgs {
  Paged pc;
  const int64_t* row_off;  // [n_prob + 1]
  int64_t n_rows;
  void* k_out;  // either may be null
  void* v_out;
};

template <int DT, int QT, int D> __global__ __launch_bounds__(256) void paged_rows_kernel(ReadArgs a) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH, NC = 16 / RPP;
  constexpr int CB = QT == kQtE2m1 ? EPT / 2 : EPT;  // bytes of a chunk's codes
  const int g = blockIdx.y, p = blockIdx.z, lane = threadIdx.x & 63, c = lane % CH, rr = lane / CH;
  const int r0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 16, shift = a.pc.shift, j = r0 >> shift, in = r0 & ((1 << shift) - 1);
  // (loads beside each other)
  const int64_t off = a.row_off[p], end = a.row_off[p + 1];
  const int id = j < a.pc.table_stride ? a.pc.table[(int64_t)p * a.pc.table_stride + j] : -1;
  const int rows = a.pc.len[p];
  // none where the offsets fall or leave the output
  if (off < 0 || end < off || end > a.n_rows || end - off > a.pc.max_len) return;
  const int L = (int)(end - off);
  if (r0 >= L) return;
  const bool has = id >= 0 && id < a.pc.n_blocks;
  const int len = has ? min(max(rows, 0), L) : 0;  // rows from here on are zeros
  const int64_t unit = (int64_t)(has ? id : 0) * a.pc.h_kv + g;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    if (!(kv ? a.v_out : a.k_out)) continue;
    const uint8_t* codes = (kv ? a.pc.v : a.pc.k) + ((unit << shift) + in) * (CB * CH);
    uint32_t u[NC][CB <= 4 ? 1 : 2], b[NC];
    float s = 0.f;
    if constexpr (QT == kQtE2m1) {
      const uint8_t* sb = static_cast<const uint8_t*>(kv ? a.pc.v_scale : a.pc.k_scale) + (unit << shift) * (D / kGroup4) + in;
#pragma unroll
      for (int i = 0; i < NC; ++i) b[i] = sb[((c * EPT / kGroup4) << shift) + i * RPP + rr];
    } else {
      s = static_cast<const float*>(kv ? a.pc.v_scale : a.pc.k_scale)[unit];
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const uint8_t* at = codes + ((i * RPP + rr) * CH + c) * CB;
      if constexpr (CB == 8) {
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(at);
        u[i][0] = x[0];
        u[i][1] = x[1];
      } else if constexpr (CB == 4) {
        u[i][0] = *reinterpret_cast<const uint32_t*>(at);
      } else {
        u[i][0] = *reinterpret_cast<const uint16_t*>(at);
      }
    }
    u32x4_t* out = reinterpret_cast<u32x4_t*>(kv ? a.v_out : a.k_out) + (off * a.pc.h_kv + (int64_t)g * L + r0) * CH + lane;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int r = r0 + i * RPP + rr;
      u32x4_t x;
      if constexpr (QT == kQtE2m1) {
        const float sc = scale4(b[i]);
        if constexpr (DT == kDtBf16) {
          x = decode8_e2m1(u[i][0], sc);
        } else {
          const u32x2_t y = {decode2_e2m1<0>(u[i][0], sc), decode2_e2m1<1>(u[i][0], sc)};  // exact in bf16
          x = u32x4_t{y[0] << 16, y[0] & 0xFFFF0000u, y[1] << 16, y[1] & 0xFFFF0000u};
        }
      } else if constexpr (DT == kDtBf16) {
        float f[4], h[4];
        decode4<QT>(u[i][0], f);
        decode4<QT>(u[i][1], h);
        x = u32x4_t{pack_bf16(f[0] * s, f[1] * s), pack_bf16(f[2] * s, f[3] * s), pack_bf16(h[0] * s, h[1] * s),
                    pack_bf16(h[2] * s, h[3] * s)};
      } else {
        float f[4];
        decode4<QT>(u[i][0], f);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __float_as_uint(f[e] * s);
      }
      if (r < L) out[i * 64] = r < len ? x : u32x4_t{0u, 0u, 0u, 0u};
    }
  }
}

namespace {

template <int DT, int QT> hipError_t read(const ReadArgs& a, dim3 grid, hipStream_t stream) {
  if (a.pc.d == 64) paged_rows_kernel<DT, QT, 64><<<grid, 256, 0, stream>>>(a);
  else paged_rows_kernel<DT, QT, 128><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}
template <int DT> hipError_t read(const ReadArgs& a, dim3 grid, hipStream_t stream) {
  if (a.pc.qtype == kQtE2m1) return read<DT, kQtE2m1>(a, grid, stream);
  return a.pc.qtype == kQtE4m3 ? read<DT, kQtE4m3>(a, grid, stream) : read<DT, kQtInt8>(a, grid, stream);
}

}  // namespace

hipError_t launch_paged_rows(const Paged& pc, const int64_t* row_off, int64_t n_rows, void* k_out, void* v_out,
                             hipStream_t stream) {
  const ReadArgs a{pc, row_off, n_rows, k_out, v_out};
  const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(pc.max_len, n_rows));
  const dim3 grid((unsigned)((rows + 63) / 64), (unsigned)pc.h_kv, (unsigned)pc.n_prob);
  return pc.dtype == kDtBf16 ? read<kDtBf16>(a, grid, stream) : read<kDtF32>(a, grid, stream);
}

}  // namespace kv
