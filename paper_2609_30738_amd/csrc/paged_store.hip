// Rows into the 8-bit blocks of a paged cache: new tokens (kv_paged_append) and the rows that an
// eviction keeps (kv_paged_compact).
//
// A wave takes the rows of one (block, kv head) of K or of V: the largest |x| over them, the scale, the
// codes.  16-byte loads: a row is CH chunks, a pass 64 / CH rows.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "compact_rows.h"
#include "paged.h"
#include "paged_codes.h"

namespace kv {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

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

// Rows row0 .. row0 + n - 1 of one block and head from `source` (its i-th row's 16-byte chunks, or null: a
// row of zeros); the block holds row0 rows already, which move to a larger scale if these need one.
// Every lane of the wave calls it.
template <int DT, int QT, int D, typename Source>
__device__ __forceinline__ void store_rows(uint8_t* codes, float* scale, int row0, int n, Source source) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T);
  constexpr int CH = D / EPT;
  constexpr int RPP = 64 / CH;
  const int lane = threadIdx.x & 63, c = lane % CH, rr = lane / CH;
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  uint32_t amax = 0;
#pragma unroll 4
  for (int i = rr; i < n; i += RPP) {
    const u32x4_t* src = source(i);
    float f[EPT];
    chunk_values<DT>(src ? src[c] : zero, f);
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const uint32_t u = __float_as_uint(f[e]) & 0x7FFFFFFFu;
      amax = max(amax, u < 0x7F800000u ? u : 0u);
    }
  }
  float s = block_scale<QT>(wave_max_u32(amax));
  if (row0 > 0) {
    const float old = *scale;
    if (!(old >= s && old < INFINITY)) {  // the held codes move by whole binades
      const float f = old > 0.f && old < s ? old * inv_scale(s) : 0.f;
      u32x4_t* at = reinterpret_cast<u32x4_t*>(codes);
      for (int i = lane; i < row0 * D / 16; i += 64) {
        u32x4_t u = at[i];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float x[4];
          decode4<QT>(u[w], x);
          u[w] = encode4<QT>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
        }
        at[i] = u;
      }
    } else {
      s = old;
    }
  }
  const float inv = inv_scale(s);
#pragma unroll 4
  for (int i = rr; i < n; i += RPP) {
    const u32x4_t* src = source(i);
    float f[EPT];
    chunk_values<DT>(src ? src[c] : zero, f);
    uint8_t* dst = codes + (row0 + i) * D + c * EPT;
    if constexpr (EPT == 8) {
      u32x2_t u;
      u[0] = encode4<QT>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
      u[1] = encode4<QT>(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
      *reinterpret_cast<u32x2_t*>(dst) = u;
    } else {
      *reinterpret_cast<uint32_t*>(dst) = encode4<QT>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
    }
  }
  if (lane == 0) *scale = s;
}

}  // namespace

struct AppendArgs {
  Paged pc;
  const void* k_new;
  const void* v_new;
  int64_t tok_chunks;  // 16-byte chunks between two tokens' rows
  const int32_t* slots;
  int n_tok, n_share;  // waves that share the runs of 64 tokens
};

// A run: consecutive tokens in consecutive slots of one block.  A wave looks at 64 tokens' slots at once and
// takes every n_share-th of the runs that begin among them.
template <int DT, int QT, int D>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArgs a) {
  constexpr int CH = D * (int)sizeof(typename Elem<DT>::T) / 16;
  const int lane = threadIdx.x & 63;
  int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int kv = (int)(id & 1);
  id >>= 1;
  const int g = (int)(id % a.pc.h_kv);
  id /= a.pc.h_kv;
  const int share = (int)(id % a.n_share);
  const int64_t first = id / a.n_share * 64;
  if (first >= a.n_tok) return;
  const int R = 1 << a.pc.shift;
  const int n_slots = a.pc.n_blocks << a.pc.shift;
  const int t = (int)first + lane;
  const int slot = t < a.n_tok ? a.slots[t] : -1;
  const int before = t > 0 && t < a.n_tok ? a.slots[t - 1] : -1;
  const bool begins = slot >= 0 && slot < n_slots && (before < 0 || slot != before + 1 || (slot & (R - 1)) == 0);
  uint64_t runs = __ballot(begins);
  for (int rank = 0; runs; ++rank, runs &= runs - 1) {
    if (rank % a.n_share != share) continue;
    const int at = __ffsll((unsigned long long)runs) - 1;
    const int s0 = __builtin_amdgcn_readlane(slot, at);
    const int t0 = (int)first + at, row0 = s0 & (R - 1);
    int n = 0;  // tokens of the run
    while (true) {
      const int i = n + lane;
      const bool in = row0 + i < R && t0 + i < a.n_tok && a.slots[t0 + i] == s0 + i;
      const uint64_t m = ~__ballot(in);
      if (m) {
        n += __ffsll((unsigned long long)m) - 1;
        break;
      }
      n += 64;
    }
    const int64_t unit = (int64_t)(s0 >> a.pc.shift) * a.pc.h_kv + g;
    const u32x4_t* src = static_cast<const u32x4_t*>(kv ? a.v_new : a.k_new) + (int64_t)t0 * a.tok_chunks + g * CH;
    store_rows<DT, QT, D>((kv ? a.pc.v : a.pc.k) + unit * R * D, (kv ? a.pc.v_scale : a.pc.k_scale) + unit, row0, n,
                          [&](int i) { return src + i * a.tok_chunks; });
  }
}

struct PagedCompactArgs {
  Paged pc;
  const int32_t* lens;
  const int64_t* tok_off;
  const void* k;
  const void* v;
  const int32_t* sel_idx;
  int budget, keep_tail, wg_blocks;
  const int32_t* budgets;
};

// One workgroup per (wg_blocks blocks, kv head, problem): the admitted positions sorted in LDS, then a wave
// for each block of K and of V.
template <int DT, int QT, int D>
__global__ __launch_bounds__(kThreads) void paged_compact_kernel(PagedCompactArgs a) {
  constexpr int CH = D * (int)sizeof(typename Elem<DT>::T) / 16;
  extern __shared__ int32_t srt[];
  const int g = blockIdx.y, p = blockIdx.z, R = 1 << a.pc.shift;
  const int L = a.lens[p];
  const int bp = a.budgets ? min(a.budgets[p], a.budget) : a.budget;
  const int rows = bp + a.keep_tail;
  const int j0 = blockIdx.x * a.wg_blocks;
  if (j0 << a.pc.shift >= rows) return;
  int n2 = 1;
  while (n2 < bp) n2 <<= 1;
  const int32_t* sel = a.sel_idx + ((int64_t)p * a.pc.h_kv + g) * a.budget;
  for (int i = threadIdx.x; i < n2; i += kThreads) srt[i] = i < bp ? sel[i] : INT_MAX;
  __syncthreads();
  sort_positions(srt, n2, threadIdx.x, kThreads);
  const int64_t base = (a.tok_off[p] * a.pc.h_kv + (int64_t)g * L) * CH;
  const int blocks = min((rows + R - 1) >> a.pc.shift, a.pc.table_stride);
  for (int task = threadIdx.x >> 6; task < 2 * a.wg_blocks; task += kWaves) {
    const int j = j0 + (task >> 1), kv = task & 1;
    if (j >= blocks) break;
    const int block = a.pc.table[(int64_t)p * a.pc.table_stride + j];
    if (block < 0 || block >= a.pc.n_blocks) continue;
    const u32x4_t* src = static_cast<const u32x4_t*>(kv ? a.v : a.k) + base;
    const int64_t unit = (int64_t)block * a.pc.h_kv + g;
    const int r0 = j << a.pc.shift;
    store_rows<DT, QT, D>((kv ? a.pc.v : a.pc.k) + unit * R * D, (kv ? a.pc.v_scale : a.pc.k_scale) + unit, 0,
                          min(R, rows - r0), [&](int i) -> const u32x4_t* {
                            const int r = r0 + i;
                            const int pos = r < bp ? srt[r] : L - a.keep_tail + (r - bp);
                            return pos < 0 || pos >= L ? nullptr : src + (int64_t)pos * CH;
                          });
  }
}

namespace {

// f<dtype, qtype, d>()
template <typename F> hipError_t dispatch(const Paged& pc, F f) {
  auto d = [&](auto dt, auto qt) {
    return pc.d == 64 ? f(dt, qt, std::integral_constant<int, 64>{}) : f(dt, qt, std::integral_constant<int, 128>{});
  };
  auto q = [&](auto dt) {
    return pc.qtype == kQtE4m3 ? d(dt, std::integral_constant<int, kQtE4m3>{})
                               : d(dt, std::integral_constant<int, kQtInt8>{});
  };
  return pc.dtype == kDtBf16 ? q(std::integral_constant<int, kDtBf16>{}) : q(std::integral_constant<int, kDtF32>{});
}

}  // namespace

hipError_t launch_paged_append(const Paged& pc, const void* k_new, const void* v_new, int64_t tok_stride,
                               const int32_t* slots, int n_tok, hipStream_t stream) {
  AppendArgs a{pc, k_new, v_new, tok_stride / (pc.dtype == kDtBf16 ? 8 : 4), slots, n_tok, 1};
  const int64_t chunks = (n_tok + 63) / 64, units = chunks * pc.h_kv * 2;
  // single rows of many requests are runs of their own: as many waves to 64 tokens as fill the chip
  constexpr int64_t kFill = 16384;
  a.n_share = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(n_tok, 64), kFill / units));
  const unsigned wgs = (unsigned)((units * a.n_share + kWaves - 1) / kWaves);
  return dispatch(pc, [&](auto dt, auto qt, auto d) {
    paged_append_kernel<dt.value, qt.value, d.value><<<wgs, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_paged_compact(const Paged& pc, const int32_t* lens, const int64_t* tok_off, const void* k,
                                const void* v, const int32_t* sel_idx, int budget, const int32_t* budgets,
                                int keep_tail, hipStream_t stream) {
  PagedCompactArgs a{pc, lens, tok_off, k, v, sel_idx, budget, keep_tail, 1, budgets};
  const int blocks = (budget + keep_tail + (1 << pc.shift) - 1) >> pc.shift;
  a.wg_blocks = std::max(2, 128 >> pc.shift);
  int n2 = 1;
  while (n2 < budget) n2 <<= 1;
  const dim3 grid((unsigned)((blocks + a.wg_blocks - 1) / a.wg_blocks), (unsigned)pc.h_kv, (unsigned)pc.n_prob);
  return dispatch(pc, [&](auto dt, auto qt, auto d) {
    paged_compact_kernel<dt.value, qt.value, d.value><<<grid, kThreads, n2 * sizeof(int32_t), stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace kv
