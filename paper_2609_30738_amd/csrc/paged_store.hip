// Rows into the 8-bit blocks of a paged cache: new tokens (kv_paged_append) and the rows that an
// eviction keeps (kv_paged_compact).
//
// A wave takes the rows of one (block, kv head) of K or of V, 16 bytes a lane and load, and holds them in
// registers: the largest |x| over them, the scale, the codes.  So a row is read once, and the wave needs no other.
//   paged_append_kernel: 195,000 rows of 8 heads of 128 (bf16 to e4m3, K and V: 800 MB read, 400 MB written) 284 us,
//     4.2 TB/s of HBM, a copy's 4.7 (365 us with the rows' addresses per lane, 695 a row at a time); 64 single rows
//     6.6 us: a chain of loads (slots, the row and the block's scale) and the launch.
//   paged_compact_kernel: 96 rows of 32 layers and 8 heads 7.4 us (lengths, positions, their ranks and rows are a
//     chain of loads); 1792 to 256 rows of 32 layers of 32768, in int8, 63 us for 207 MB, read in rows of 256
//     bytes.
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

// Rows row0 .. row0 + n - 1 of one block and head; the block holds row0 rows already.  load(i): the lane's 16-byte
// chunk, number lane % CH of row i RPP + lane / CH of the new ones (zeros past the last).  Every lane of the wave
// calls it.
template <int DT, int QT, int D, int SHIFT, typename Load>
__device__ __forceinline__ void store_rows(uint8_t* codes, float* scale, int row0, int n, Load load) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH;
  constexpr int NC = kChunks<DT, D, SHIFT>;
  if constexpr (NC > kHeldChunks) {
    store_rows_any<DT, QT, D>(codes, scale, row0, n, load);
    return;
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

}  // namespace

struct AppendArgs {
  Paged pc;
  const void* k_new;
  const void* v_new;
  uint32_t tok_bytes;  // between two tokens' rows: at most 2^28
  const int32_t* slots;
  int n_tok, n_share;  // waves that share the runs of 64 tokens
};

// A run: consecutive tokens in consecutive slots of one block.  A wave looks at 64 tokens' slots at once and
// takes every n_share-th of the runs that begin among them.
template <int DT, int QT, int D, int SHIFT>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArgs a) {
  constexpr int CH = D * (int)sizeof(typename Elem<DT>::T) / 16, RPP = 64 / CH;
  const int lane = threadIdx.x & 63;
  int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int kv = (int)(id & 1);
  id >>= 1;
  const int g = (int)(id % a.pc.h_kv);
  id /= a.pc.h_kv;
  const int share = (int)(id % a.n_share);
  const int64_t first = id / a.n_share * 64;
  if (first >= a.n_tok) return;
  constexpr int R = 1 << SHIFT;
  const int n_slots = a.pc.n_blocks << SHIFT;
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
    const int64_t unit = (int64_t)(s0 >> SHIFT) * a.pc.h_kv + g;
    // a wave-uniform address and a lane's 32-bit offset
    const uint8_t* src = static_cast<const uint8_t*>(kv ? a.v_new : a.k_new) + (int64_t)t0 * a.tok_bytes + g * (CH * 16);
    const uint32_t mine = lane / CH * a.tok_bytes + lane % CH * 16;
    store_rows<DT, QT, D, SHIFT>((kv ? a.pc.v : a.pc.k) + unit * R * D, (kv ? a.pc.v_scale : a.pc.k_scale) + unit,
                                 row0, n, [&](int i) {
                                   u32x4_t x = {0u, 0u, 0u, 0u};
                                   if (i * RPP + lane / CH < n)
                                     x = *reinterpret_cast<const u32x4_t*>(src + (int64_t)i * RPP * a.tok_bytes + mine);
                                   return x;
                                 });
  }
}

struct PagedCompactArgs {
  Paged pc;
  const int32_t* lens;
  const int64_t* tok_off;
  const void* k;
  const void* v;
  const int32_t* sel_idx;
  int budget, keep_tail, wg_blocks, bitmap_words;
  const int32_t* budgets;
};

namespace {

// Budgets up to which a position's rank is counted against all others, and the longest problem whose positions
// are ranked through a bitmap (32 KB); beyond, or where a position is given twice, they are sorted.
// Counted and through the bitmap: 64 of 131072 positions 4.6 and 8.5 us, 250 of 4096 9.4 and 7.7, of 32768 (32 layers)
// 18.3 and 18.1, of 262144 9.4 and 22.9; sorted 7.4, 13.3, 22.2 and 13.3.  Bitmap and sorted, 1024 on average of
// 32768 (32 layers): 63 and 138 us.
constexpr int kCountBudget = 256;
constexpr int kCountLen = (1 << 24) - 1, kBitmapLen = 1 << 18;

// pos[0, n): the positions of rows first .. first + n - 1 of the unit, first + n <= bp: the ascending order of
// sel[0, bp).  lds: work space (see compact_lds).  Starts and ends synchronised.
__device__ __forceinline__ void kept_positions(const int32_t* sel, int bp, int L, int first, int n, int32_t* pos,
                                               int32_t* work, int words) {
  __shared__ int32_t sums[kWaves], below, twice;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (bp <= kCountBudget && L < kCountLen) {
    // keys of 24 bits of the position (below 0: the lowest, past the problem: the highest) and 8 of its place
    const int mine = tid < bp ? sel[tid] : INT_MAX;
    const uint32_t key = (uint32_t)(min(max(mine, -1), kCountLen - 1) + 1) << 8 | tid;
    uint32_t* keys = reinterpret_cast<uint32_t*>(work);
    keys[tid] = key;
    __syncthreads();
    int rank = 0;
    for (int j0 = 0; j0 < bp; j0 += 32) {  // (past bp: the highest, with later places)
#pragma unroll
      for (int j = j0; j < j0 + 32; j += 4) {
        const u32x4_t o = *reinterpret_cast<const u32x4_t*>(keys + j);
        rank += (o[0] < key) + (o[1] < key) + (o[2] < key) + (o[3] < key);
      }
    }
    if (tid < bp && rank >= first && rank < first + n) pos[rank - first] = mine;
    __syncthreads();
    return;
  }
  if (words > 0) {
    const int used = (L + 31) >> 5;
    for (int i = tid; i < used; i += kThreads) work[i] = 0;
    if (tid == 0) below = twice = 0;
    __syncthreads();
    int low = 0, again = 0;
    for (int i = tid; i < bp; i += kThreads) {
      const int x = sel[i];
      if (x < 0) ++low;
      else if (x < L) again |= (atomicOr(reinterpret_cast<uint32_t*>(work) + (x >> 5), 1u << (x & 31)) >> (x & 31)) & 1;
    }
    if (low) atomicAdd(&below, low);
    if (again) twice = 1;
    __syncthreads();
    if (!twice) {
      // positions below 0 first, then the bitmap's, then those past the problem: a thread takes consecutive words
      const int per = (used + kThreads - 1) / kThreads, w0 = min(tid * per, used), w1 = min(w0 + per, used);
      int count = 0;
      for (int w = w0; w < w1; ++w) count += __popc((uint32_t)work[w]);
      int incl = count;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(incl, o, 64);
        if (lane >= o) incl += u;
      }
      if (lane == 63) sums[wave] = incl;
      __syncthreads();
      int rank = below + incl - count, total = below;
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) rank += sums[w];
        total += sums[w];
      }
      if (rank < first + n && rank + count > first) {
        for (int w = w0; w < w1; ++w)
          for (uint32_t bits = (uint32_t)work[w]; bits; bits &= bits - 1, ++rank)
            if (rank >= first && rank < first + n) pos[rank - first] = 32 * w + __ffs((int)bits) - 1;
      }
      for (int i = tid; i < n; i += kThreads)
        if (first + i < below || first + i >= total) pos[i] = -1;
      __syncthreads();
      return;
    }
  }
  int n2 = 1;
  while (n2 < bp) n2 <<= 1;
  __syncthreads();
  for (int i = tid; i < n2; i += kThreads) work[i] = i < bp ? sel[i] : INT_MAX;
  __syncthreads();
  sort_positions(work, n2, tid, kThreads);
  for (int i = tid; i < n; i += kThreads) pos[i] = work[first + i];
  __syncthreads();
}

}  // namespace

// One workgroup per (wg_blocks blocks, kv head, problem): the ranks of the admitted positions, then a wave for
// each block of K and of V.
template <int DT, int QT, int D, int SHIFT>
__global__ __launch_bounds__(kThreads) void paged_compact_kernel(PagedCompactArgs a) {
  constexpr int CH = D * (int)sizeof(typename Elem<DT>::T) / 16, RPP = 64 / CH, R = 1 << SHIFT;
  const int lane = threadIdx.x & 63;
  extern __shared__ __align__(16) int32_t lds[];  // positions of the workgroup's rows, then work space
  const int g = blockIdx.y, p = blockIdx.z;
  const int L = a.lens[p];
  const int bp = a.budgets ? min(a.budgets[p], a.budget) : a.budget;
  const int rows = bp + a.keep_tail;
  const int j0 = blockIdx.x * a.wg_blocks, first = j0 << SHIFT;
  if (first >= rows) return;
  const int n = min(max(bp - first, 0), a.wg_blocks << SHIFT);  // admitted rows among the workgroup's
  if (n > 0)
    kept_positions(a.sel_idx + ((int64_t)p * a.pc.h_kv + g) * a.budget, bp, L, first, n, lds,
                   lds + (a.wg_blocks << SHIFT), L <= a.bitmap_words * 32 ? a.bitmap_words : 0);
  const int64_t base = (a.tok_off[p] * a.pc.h_kv + (int64_t)g * L) * CH;
  const int blocks = min((rows + R - 1) >> SHIFT, a.pc.table_stride);
  for (int task = threadIdx.x >> 6; task < 2 * a.wg_blocks; task += kWaves) {
    const int j = j0 + (task >> 1), kv = task & 1;
    if (j >= blocks) break;
    const int block = a.pc.table[(int64_t)p * a.pc.table_stride + j];
    if (block < 0 || block >= a.pc.n_blocks) continue;
    const u32x4_t* src = static_cast<const u32x4_t*>(kv ? a.v : a.k) + base;
    const int64_t unit = (int64_t)block * a.pc.h_kv + g;
    const int r0 = j << SHIFT;
    store_rows<DT, QT, D, SHIFT>((kv ? a.pc.v : a.pc.k) + unit * R * D, (kv ? a.pc.v_scale : a.pc.k_scale) + unit, 0,
                                 min(R, rows - r0), [&](int i) {
                                   // without a branch, so that the rows' loads are in flight together
                                   const int r = min(r0 + i * RPP + lane / CH, rows - 1);
                                   const int kept = n > 0 ? lds[min(r - first, n - 1)] : 0;
                                   const int pos = r < bp ? kept : L - a.keep_tail + (r - bp);
                                   const bool in = r0 + i * RPP + lane / CH < rows && (uint32_t)pos < (uint32_t)L;
                                   const u32x4_t x = src[(int64_t)(in ? pos : 0) * CH + lane % CH];
                                   return in ? x : u32x4_t{0u, 0u, 0u, 0u};
                                 });
  }
}

namespace {

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
  auto q = [&](auto dt) { return pc.qtype == kQtE4m3 ? d(dt, Int<kQtE4m3>{}) : d(dt, Int<kQtInt8>{}); };
  return pc.dtype == kDtBf16 ? q(Int<kDtBf16>{}) : q(Int<kDtF32>{});
}

}  // namespace

hipError_t launch_paged_append(const Paged& pc, const void* k_new, const void* v_new, int64_t tok_stride,
                               const int32_t* slots, int n_tok, hipStream_t stream) {
  AppendArgs a{pc, k_new, v_new, (uint32_t)(tok_stride * (pc.dtype == kDtBf16 ? 2 : 4)), slots, n_tok, 1};
  const int64_t chunks = ((int64_t)n_tok + 63) / 64, units = chunks * pc.h_kv * 2;
  // single rows of many requests are runs of their own: as many waves to 64 tokens as fill the chip.  4096 single rows
  // of 8 heads 34 us, with 2048 waves 49, with 8192 38; 60 prompts of up to 50 rows 5.4, 6.4 and 6.5
  constexpr int64_t kFill = 4096;
  a.n_share = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(n_tok, 64), kFill / units));
  const unsigned wgs = (unsigned)((units * a.n_share + kWaves - 1) / kWaves);
  return dispatch(pc, [&](auto dt, auto qt, auto d, auto shift) {
    paged_append_kernel<dt.value, qt.value, d.value, shift.value><<<wgs, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_paged_compact(const Paged& pc, const int32_t* lens, int max_len, const int64_t* tok_off,
                                const void* k, const void* v, const int32_t* sel_idx, int budget,
                                const int32_t* budgets, int keep_tail, hipStream_t stream) {
  PagedCompactArgs a{pc, lens, tok_off, k, v, sel_idx, budget, keep_tail, 1, 0, budgets};
  const int blocks = (budget + keep_tail + (1 << pc.shift) - 1) >> pc.shift;
  // a workgroup ranks for its blocks alone: few of them where ranking is short (96 rows 8.4 us, with one block 9.7
  // before ranks were counted by keys), else as many as pay for it (falling budgets 64 us; half the rows a workgroup 65,
  // twice 81)
  a.wg_blocks = budget <= kCountBudget ? 2 : std::max(2, 128 >> pc.shift);
  int work = kThreads;  // words: the counted positions, the bitmap, the sorted positions
  if (budget > kCountBudget) {
    if (max_len <= kBitmapLen) a.bitmap_words = (max_len + 31) / 32;
    int n2 = 1;
    while (n2 < budget) n2 <<= 1;
    work = std::max(a.bitmap_words, n2);
  }
  const size_t bytes = ((size_t)(a.wg_blocks << pc.shift) + work) * sizeof(int32_t);
  const dim3 grid((unsigned)((blocks + a.wg_blocks - 1) / a.wg_blocks), (unsigned)pc.h_kv, (unsigned)pc.n_prob);
  return dispatch(pc, [&](auto dt, auto qt, auto d, auto shift) {
    paged_compact_kernel<dt.value, qt.value, d.value, shift.value><<<grid, kThreads, bytes, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace kv
