// New rows into the blocks of a paged cache with the keys rotated on the way, and the rotated queries
// (kv_paged_append_rotated).
//
// paged_rotated_kernel: some workgroups rotate queries as kv_rotate does.  The others take runs of tokens in consecutive slots
//   of one block (as paged_append_kernel): the turns of the run's tokens go to LDS once, then a wave takes one head of K or
//   of V after the other.  A key's chunk is turned in registers, with the chunk of the other halves of its pairs from its
//   lane, and coded from the 32-bit values: it never reaches memory in another form.
#include <math.h>

#include <algorithm>

#include "paged.h"
#include "paged_rows.h"
#include "rotary.h"

namespace kv {

struct AppendRotatedArgs {
  Paged pc;
  RotateArgs rq;  // the queries; rot, pos and n_tok are the keys' too
  const void* k_new;
  const void* v_new;
  uint32_t tok_bytes;  // between two tokens' rows: at most 2^28
  const int32_t* slots;
  int64_t q_wgs;       // workgroups of the queries
  int n_share, parts;  // workgroups that share the runs of 64 tokens, and a run's heads
};

namespace {

// Rows row0 .. row0 + n - 1 of one block and head, turned; load as in store_rows, turns [n][half].
template <int DT, int QT, int D, int SHIFT, typename Load>
__device__ __forceinline__ void store_turned(uint8_t* codes, ScaleOf<QT>* scale, int row0, int n, const float2* turns, int half,
                                             const TurnChunk<DT, D>& turned, Load load) {
  constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH, NC = kChunks<DT, D, SHIFT>;
  const int lane = threadIdx.x & 63, c = lane % CH, rr = lane / CH;
  // the row's turns (the last row's past the end)
  auto of = [&](int i) { return turns + min(i * RPP + rr, n - 1) * half; };
  if constexpr (QT == kQtE2m1) {
    constexpr int NB = NC < kBatch4 ? NC : kBatch4;
    for (int i0 = 0; i0 * RPP < n; i0 += NB) {
      u32x4_t x[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        x[i] = u32x4_t{0u, 0u, 0u, 0u};
        if ((i0 + i) * RPP < n) x[i] = load(i0 + i);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        if ((i0 + i) * RPP >= n) break;
        float f[EPT];
        turned(x[i], of(i0 + i), f);
        const int r = (i0 + i) * RPP + rr;
        store_chunk4<D, EPT>(codes, scale, row0 + r, 1 << SHIFT, c, r < n, f);
      }
    }
  } else {
    // chunks that do not fit the registers are loaded again
    constexpr int NH = NC > kHeldChunks ? 1 : NC;
    const float old = row0 > 0 ? *scale : 0.f;
    u32x4_t x[NH];
    if constexpr (NH == NC) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        x[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (i * RPP < n) x[i] = load(i);
      }
    }
    uint32_t amax = 0;
    bool odd = false;  // an infinity or a NaN among the lane's values
    auto largest = [&](int i, const u32x4_t& y) __attribute__((always_inline)) {
      float f[EPT];
      turned(y, of(i), f);
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        const uint32_t u = __float_as_uint(f[e]) & 0x7FFFFFFFu;
        amax = max(amax, u < 0x7F800000u ? u : 0u);
        odd = odd || u >= 0x7F800000u;
      }
    };
    auto store = [&](int i, const u32x4_t& y, float inv, auto finite) __attribute__((always_inline)) {
      float f[EPT];
      turned(y, of(i), f);
      if (i * RPP + rr < n)
        store_chunk<QT, decltype(finite)::value>(codes + (row0 + i * RPP + rr) * D + c * EPT, f, inv);
    };
    auto each = [&](auto f) __attribute__((always_inline)) {
      if constexpr (NH == NC) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          // (a value is formed anew in each pass over the chunks: registers)
          asm volatile("" : "+v"(x[i][0]), "+v"(x[i][1]), "+v"(x[i][2]), "+v"(x[i][3]));
          if (i * RPP < n) f(i, x[i]);
        }
      } else {
        for (int i = 0; i * RPP < n; ++i) f(i, load(i));
      }
    };
    each(largest);
    const float s = grown_scale<QT, D>(codes, row0, old, block_scale<QT>(wave_max_u32(amax))), inv = inv_scale(s);
    if (__ballot(odd)) each([&](int i, const u32x4_t& y) { store(i, y, inv, std::false_type{}); });
    else each([&](int i, const u32x4_t& y) { store(i, y, inv, std::true_type{}); });
    if (lane == 0) *scale = s;
  }
}

}  // namespace

template <int DT, int QT, int D, int SHIFT>
__global__ __launch_bounds__(kStoreThreads) void paged_rotated_kernel(AppendRotatedArgs a) {
  constexpr int CH = D * (int)sizeof(typename Elem<DT>::T) / 16, RPP = 64 / CH, R = 1 << SHIFT, kWaves = kStoreThreads / 64;
  extern __shared__ __align__(16) float2 tab[];
  int64_t id = blockIdx.x;
  if (id < a.q_wgs) {
    rotate_group<DT, D>(a.rq, id / a.rq.parts, (int)(id % a.rq.parts), tab);
    return;
  }
  id -= a.q_wgs;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_tok = a.rq.n_tok;
  const int part = (int)(id % a.parts);
  id /= a.parts;
  const int share = (int)(id % a.n_share);
  const int64_t first = id / a.n_share * 64;
  if (first >= n_tok) return;
  const int n_slots = a.pc.n_blocks << SHIFT;
  const int t = (int)first + lane;
  const int slot = t < n_tok ? a.slots[t] : -1;
  const int before = t > 0 && t < n_tok ? a.slots[t - 1] : -1;
  const bool begins = slot >= 0 && slot < n_slots && (before < 0 || slot != before + 1 || (slot & (R - 1)) == 0);
  const TurnChunk<DT, D> turned(a.rq.rot);
  uint64_t runs = __ballot(begins);  // the same in every wave
  for (int rank = 0; runs; ++rank, runs &= runs - 1) {
    if (rank % a.n_share != share) continue;
    const int at = __ffsll((unsigned long long)runs) - 1;
    const int s0 = __builtin_amdgcn_readlane(slot, at);
    const int t0 = (int)first + at, row0 = s0 & (R - 1);
    int n = 0;  // tokens of the run
    while (true) {
      const int i = n + lane;
      const bool in = row0 + i < R && t0 + i < n_tok && a.slots[t0 + i] == s0 + i;
      const uint64_t m = ~__ballot(in);
      if (m) {
        n += __ffsll((unsigned long long)m) - 1;
        break;
      }
      n += 64;
    }
    fill_turns(tab, a.rq.rot, a.rq.pos + t0, n);
    __syncthreads();
    const uint32_t mine = lane / CH * a.tok_bytes + lane % CH * 16;
    for (int u = part * kWaves + wave; u < 2 * a.pc.h_kv; u += a.parts * kWaves) {
      const int kv = u & 1, g = u >> 1;
      const int64_t unit = (int64_t)(s0 >> SHIFT) * a.pc.h_kv + g;
      // a wave-uniform address and a lane's 32-bit offset
      const uint8_t* src = static_cast<const uint8_t*>(kv ? a.v_new : a.k_new) + (int64_t)t0 * a.tok_bytes + g * (CH * 16);
      auto load = [&](int i) {
        u32x4_t x = {0u, 0u, 0u, 0u};
        if (i * RPP + lane / CH < n) x = *reinterpret_cast<const u32x4_t*>(src + (int64_t)i * RPP * a.tok_bytes + mine);
        return x;
      };
      uint8_t* codes = unit_codes<QT, D, SHIFT>(kv ? a.pc.v : a.pc.k, unit);
      auto* scale = unit_scale<QT, D, SHIFT>(kv ? a.pc.v_scale : a.pc.k_scale, unit);
      if (kv) store_rows<DT, QT, D, SHIFT>(codes, scale, row0, n, load);
      else store_turned<DT, QT, D, SHIFT>(codes, scale, row0, n, tab, a.rq.rot.rot >> 1, turned, load);
    }
    __syncthreads();
  }
}

hipError_t launch_paged_append_rotated(const Paged& pc, const RotateArgs& rq, const void* k_new, const void* v_new,
                                       int64_t tok_stride, const int32_t* slots, hipStream_t stream) {
  AppendRotatedArgs a{pc, rq, k_new, v_new, (uint32_t)(tok_stride * (pc.dtype == kDtBf16 ? 2 : 4)), slots, 0, 1, 1};
  const int64_t windows = ((int64_t)rq.n_tok + 63) / 64;
  // single rows of many requests are runs of their own: as many workgroups to 64 tokens, and then to a run's heads, as
  // fill the chip
  constexpr int64_t kFill = 1024;
  a.n_share = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(rq.n_tok, 64), kFill / windows));
  const int most = (2 * pc.h_kv + 3) / 4;
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, kFill / (windows * a.n_share)));
  return dispatch(pc, [&](auto dt, auto qt, auto d, auto shift) {
    constexpr int RW = kRotateRows<dt.value, d.value>;
    if (rq.x) {
      const int64_t groups = ((int64_t)rq.n_tok + RW - 1) / RW;
      a.rq.parts = rotate_parts(groups, rq.heads);
      a.q_wgs = groups * a.rq.parts;
    }
    const size_t lds = (size_t)std::max(RW, 1 << shift.value) * (rq.rot.rot / 2) * sizeof(float2);
    const unsigned wgs = (unsigned)(a.q_wgs + windows * a.n_share * a.parts);
    paged_rotated_kernel<dt.value, qt.value, d.value, shift.value><<<wgs, kStoreThreads, lds, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace kv
