// New rows into the blocks of a paged cache with the keys rotated on the way, and the rotated queries
// (kv_paged_append_rotated).
//
// Bound by HBM: 44,400 tokens of 32 query heads and 8 of K and V into 8 bits (1.0 GB) 197 us, 5.1 TB/s, a copy's 5.5; K and V
// alone (273 MB) 72, 3.8 TB/s.  The same into 4 bits 198 and 66.  64 single tokens 8.4, 24 into 4 bits 6: a chain of loads (slots, then
// the block's scale), the turns and the launch.
//
// Some workgroups rotate queries as kv_rotate does.  The others form the turns of their tokens' pairs once, in LDS, and go
// over the heads with them; a key's chunk is turned in registers, with the chunk of the other halves of its pairs from its
// lane, and coded from the 32-bit values: it never reaches memory in another form.
//   paged_rotated_kernel (8 bits): runs of tokens in consecutive slots of one block (as paged_append_kernel), whose rows of a
//     head share a scale; a tile of rows of a few heads at a time, the scale through LDS.
//   paged_rotated4_kernel (4 bits): a few tokens, wherever their slots are, four rows at a time to a wave.
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
  int n_share, parts;  // workgroups that share the runs of 64 tokens, and the heads
};

namespace {

// The rows of a block in tiles.  Long runs: a tile's rows fall to the four waves, and a lane's chunks of a few heads are in
// registers together, kHeld of them, of at most four heads.  Short ones: a wave takes a head by itself.
// K and V of 44,400 tokens in blocks of 64 rows 72 us, with 4 chunks 74, with 16 77; of 128 rows 89, 122, 108; of 16 rows,
// four heads 67, eight 79.
constexpr int kHeld = 8;
template <int DT, int D, int SHIFT, bool LONG> struct Tiling {
  static constexpr int EPT = 16 / (int)sizeof(typename Elem<DT>::T), CH = D / EPT, RPP = 64 / CH, W = LONG ? kStoreThreads / 64 : 1;
  static constexpr int ROWS = RPP * W;  // of a tile
  static constexpr int TILES = (1 << SHIFT) > ROWS ? (1 << SHIFT) / ROWS : 1;
  static constexpr bool TWICE = !LONG || TILES > kHeld;  // runs of more than TB tiles are read twice
  static constexpr int TB = !LONG ? 1 : TWICE ? kHeld : TILES, HEADS = LONG ? std::min(kHeld / TB, 4) : 1;
};

// A workgroup's run: rows row0 .. row0 + n - 1 of a block, and the heads from g to end - 1 of K (KV 0, turned) or V.
struct Run {
  int row0, n;
  int64_t unit0;        // of the block's first head
  const uint8_t* rows;  // of the first token
  uint32_t tok_bytes;
};

template <int DT, int QT, int D, int SHIFT, bool INTERLEAVED, bool LONG, int KV>
__device__ __forceinline__ void store_heads(const Paged& pc, const Run& run, int g, int end, const Turns& turns,
                                            const TurnChunk<DT, D, INTERLEAVED>& turned, int& turn_of_sh) {
  using T = Tiling<DT, D, SHIFT, LONG>;
  using C = TurnChunk<DT, D, INTERLEAVED>;
  constexpr int EPT = T::EPT, CH = T::CH, HB = T::HEADS, TB = T::TB, W = T::W;
  __shared__ float sh_amax[2][W][kHeld];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % CH;
  const int r_lane = (LONG ? wave * T::RPP : 0) + lane / CH;
  uint8_t* const codes = unit_codes<QT, D, SHIFT>(KV ? pc.v : pc.k, run.unit0);
  float* const scales = unit_scale<QT, D, SHIFT>(KV ? pc.v_scale : pc.k_scale, run.unit0);
  for (; g < end; g += HB) {
    // past the last head and row: theirs again
    auto head = [&](int h) { return min(g + h, end - 1); };
    auto row = [&](int t) { return min(t * T::ROWS + r_lane, run.n - 1); };
    float v[HB][TB][EPT];
    auto take = [&](int t0) __attribute__((always_inline)) {
      u32x4_t x[HB][TB];
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const uint8_t* src = run.rows + (int64_t)row(t0 + t) * run.tok_bytes + c * 16;
#pragma unroll
        for (int h = 0; h < HB; ++h) x[h][t] = *reinterpret_cast<const u32x4_t*>(src + head(h) * (CH * 16));
      }
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        float2 cs[C::PAIRS];
        if constexpr (KV == 0) turns.get(row(t0 + t), turned.mine, cs);
#pragma unroll
        for (int h = 0; h < HB; ++h) {
          if constexpr (KV == 0) turned(x[h][t], cs, v[h][t]);
          else chunk_values<DT>(x[h][t], v[h][t]);
        }
      }
    };
    float amax[HB], odd = 0.f;  // odd: NaN where an infinity or a NaN is among the lane's values
#pragma unroll
    for (int h = 0; h < HB; ++h) amax[h] = 0.f;
    auto largest = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < HB; ++h)
#pragma unroll
        for (int t = 0; t < TB; ++t)
#pragma unroll
          for (int e = 0; e < EPT; ++e) {
            amax[h] = fmaxf(amax[h], fabsf(v[h][t][e]));
            odd = fmaf(v[h][t][e], 0.f, odd);
          }
    };
    // the finite values' largest, of values that are not all finite
    auto largest_finite = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < HB; ++h)
#pragma unroll
        for (int t = 0; t < TB; ++t)
#pragma unroll
          for (int e = 0; e < EPT; ++e) amax[h] = fmaxf(amax[h], fabsf(v[h][t][e]) < INFINITY ? fabsf(v[h][t][e]) : 0.f);
    };
    bool any = T::TWICE;
    const bool once = run.n <= TB * T::ROWS;
    if constexpr (T::TWICE) {
      for (int t0 = 0; t0 * T::ROWS < run.n; t0 += TB) {
        take(t0);
        largest_finite();
      }
    } else {
      take(0);
      largest();
      any = __ballot(!(odd == 0.f)) != 0;
      if (any) {
#pragma unroll
        for (int h = 0; h < HB; ++h) amax[h] = 0.f;
        largest_finite();
      }
    }
    float old[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) old[h] = run.row0 > 0 ? scales[head(h)] : 0.f;
    const int turn = turn_of_sh;
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      amax[h] = wave_max_uniform(amax[h]);
      if (LONG && lane == h) sh_amax[turn][wave][h] = amax[h];
    }
    if constexpr (LONG) {
      __syncthreads();
      turn_of_sh ^= 1;
    }
    float inv[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      float m = amax[h];
      if constexpr (LONG) {
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, sh_amax[turn][w][h]);
      }
      float s = block_scale<QT>(__float_as_uint(m));
      if (run.row0 > 0) {
        // the block's rows in use move to a larger scale by one wave
        if (g + h < end && (!LONG || h % W == wave)) grown_scale<QT, D>(codes + ((int64_t)(g + h) << SHIFT) * D, run.row0, old[h], s);
        if (old[h] >= s && old[h] < INFINITY) s = old[h];
      }
      if ((LONG ? threadIdx.x : lane) == 0 && g + h < end) scales[g + h] = s;
      inv[h] = inv_scale(s);
    }
    auto put = [&](int t0, auto finite) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const int r = (t0 + t) * T::ROWS + r_lane;
#pragma unroll
        for (int h = 0; h < HB; ++h)
          if (r < run.n && g + h < end)
            store_chunk<QT, decltype(finite)::value>(codes + (((int64_t)(g + h) << SHIFT) + run.row0 + r) * D + c * EPT, v[h][t], inv[h]);
      }
    };
    if constexpr (T::TWICE) {
      for (int t0 = 0; t0 * T::ROWS < run.n; t0 += TB) {
        if (!once) take(t0);
        put(t0, std::false_type{});
      }
    } else if (any) {
      put(0, std::false_type{});
    } else {
      put(0, std::true_type{});
    }
  }
}

}  // namespace

template <int DT, int QT, int D, int SHIFT, bool INTERLEAVED, bool LONG>
__global__ __launch_bounds__(kStoreThreads) void paged_rotated_kernel(AppendRotatedArgs a) {
  using C = TurnChunk<DT, D, INTERLEAVED>;
  constexpr int R = 1 << SHIFT;
  extern __shared__ __align__(16) float4 lds[];
  int64_t id = blockIdx.x;
  if (id < a.q_wgs) {
    rotate_group<DT, D>(a.rq, id / a.rq.parts, (int)(id % a.rq.parts), lds);
    return;
  }
  id -= a.q_wgs;
  const int lane = threadIdx.x & 63, n_tok = a.rq.n_tok;
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
  const C turned(a.rq.rot);
  const Turns turns(lds, a.rq.rot, C::PAIRS);
  const int per = (a.pc.h_kv + a.parts - 1) / a.parts, g0 = part * per, g1 = min(g0 + per, a.pc.h_kv);
  int turn = 0;
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
    turns.fill(a.rq.rot, a.rq.pos + t0, n);
    __syncthreads();
    Run run{row0, n, (int64_t)(s0 >> SHIFT) * a.pc.h_kv, static_cast<const uint8_t*>(a.k_new) + (int64_t)t0 * a.tok_bytes, a.tok_bytes};
    const uint8_t* v_rows = static_cast<const uint8_t*>(a.v_new) + (int64_t)t0 * a.tok_bytes;
    if constexpr (LONG) {
      store_heads<DT, QT, D, SHIFT, INTERLEAVED, true, 0>(a.pc, run, g0, g1, turns, turned, turn);
      run.rows = v_rows;
      store_heads<DT, QT, D, SHIFT, INTERLEAVED, true, 1>(a.pc, run, g0, g1, turns, turned, turn);
    } else {
      for (int u = 2 * g0 + (threadIdx.x >> 6); u < 2 * g1; u += kStoreThreads / 64) {
        const int g = __builtin_amdgcn_readfirstlane(u >> 1);
        if (u & 1) {
          Run v = run;
          v.rows = v_rows;
          store_heads<DT, QT, D, SHIFT, INTERLEAVED, false, 1>(a.pc, v, g, g + 1, turns, turned, turn);
        } else {
          store_heads<DT, QT, D, SHIFT, INTERLEAVED, false, 0>(a.pc, run, g, g + 1, turns, turned, turn);
        }
      }
    }
    __syncthreads();
  }
}

// Tokens of a workgroup of paged_rotated4_kernel: a wave's 64 chunks of 16 bytes are whole rows of a head.
template <int DT, int D> constexpr int kRotatedRows4 = kStoreThreads * 16 / (D * (int)sizeof(typename Elem<DT>::T));

template <int DT, int D, bool INTERLEAVED>
__global__ __launch_bounds__(kStoreThreads) void paged_rotated4_kernel(AppendRotatedArgs a) {
  using C = TurnChunk<DT, D, INTERLEAVED>;
  constexpr int EPT = C::EPT, CH = C::CH, RPP = 64 / CH, ROWS = kRotatedRows4<DT, D>, kBatch = 8;
  extern __shared__ __align__(16) float4 lds[];
  int64_t id = blockIdx.x;
  if (id < a.q_wgs) {
    rotate_group<DT, D>(a.rq, id / a.rq.parts, (int)(id % a.rq.parts), lds);
    return;
  }
  id -= a.q_wgs;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane % CH, part = (int)(id % a.parts);
  const int64_t t0 = id / a.parts * ROWS;
  const int n = (int)min((int64_t)ROWS, a.rq.n_tok - t0), r = wave * RPP + lane / CH;
  const int slot = r < n ? a.slots[t0 + r] : -1, R = 1 << a.pc.shift;
  const bool live = slot >= 0 && (slot >> a.pc.shift) < a.pc.n_blocks;
  const int64_t unit0 = (int64_t)(live ? slot >> a.pc.shift : 0) * a.pc.h_kv;  // of the block's first head
  const int row = live ? slot & (R - 1) : 0;
  // consecutive heads fall to a part: rows of a token lie beside each other
  const int per = (a.pc.h_kv + a.parts - 1) / a.parts, g0 = part * per, g1 = min(g0 + per, a.pc.h_kv);
  const int64_t mine = (t0 + (r < n ? r : 0)) * (int64_t)a.tok_bytes + c * 16;
  u32x4_t x[kBatch];
  auto load = [&](const void* rows, int g) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (g + i < g1) x[i] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint8_t*>(rows) + mine + (g + i) * (CH * 16));
  };
  load(a.k_new, g0);
  const Turns turns(lds, a.rq.rot, C::PAIRS);
  turns.fill(a.rq.rot, a.rq.pos + t0, n);
  __syncthreads();
  const C turned(a.rq.rot);
  float2 cs[C::PAIRS];
  turns.get(min(r, n - 1), turned.mine, cs);
  auto put = [&](int kv, int g, const float (&f)[EPT]) __attribute__((always_inline)) {
    const int64_t unit = (unit0 + g) << a.pc.shift;
    store_chunk4<D, EPT>((kv ? a.pc.v : a.pc.k) + unit * (D / 2), static_cast<uint8_t*>(kv ? a.pc.v_scale : a.pc.k_scale) + unit * (D / kGroup4),
                         row, R, c, live, f);
  };
  for (int g = g0; g < g1; g += kBatch) {
    if (g > g0) load(a.k_new, g);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (g + i >= g1) break;
      float f[EPT];
      turned(x[i], cs, f);
      put(0, g + i, f);
    }
    load(a.v_new, g);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (g + i >= g1) break;
      if constexpr (DT == kDtBf16) {
        const int64_t unit = (unit0 + g + i) << a.pc.shift;
        store_chunk4_bf16<D>(a.pc.v + unit * (D / 2), static_cast<uint8_t*>(a.pc.v_scale) + unit * (D / kGroup4), row, R, c, live, x[i]);
      } else {
        float f[EPT];
        chunk_values<DT>(x[i], f);
        put(1, g + i, f);
      }
    }
  }
}

namespace {

// Whether 8-bit appending takes the runs as long ones: by the tokens to a request, a padded batch's among them, for the whole
// call.  In us as short and as long ones, in blocks of 16 / 64 / 128 rows:
//   with queries: 2000 single rows 28 / 28 / 42 and 103 / 382 / 367; five rows of 64 requests 12 / 12 / 13 and 23 / 64 / 61;
//     one prompt of 2048 tokens beside 255 requests without rows 33 / 94 / 152 and 15 / 17 / 22, beside 255 single rows
//     33 / 80 / 151 and 94 / 331 / 316;
//   without: 20 rows of 64 requests 19 / 28 / 23 and 14 / 25 / 24, four prompts of 300 tokens 17 / 50 / 95 and 12 / 16 / 18.
// A workgroup takes the runs that fall to it one after the other, and in blocks of 64 rows all runs of 64 tokens fall to one.
// So requests of 5 to about 16 rows each would be faster as short runs, where a prompt that brings a call to as many rows to a
// request is faster as long ones; a prompt beside single rows is slow either way (kv_rotate of both and kv_paged_append:
// 32 / 41 / 52).
bool is_long(const Paged& pc, int n_tok) { return n_tok > 4 * (int64_t)pc.n_prob; }

template <int DT, int D, bool INTERLEAVED> hipError_t append4(AppendRotatedArgs a, hipStream_t stream) {
  constexpr int ROWS = kRotatedRows4<DT, D>;
  const int64_t groups = ((int64_t)a.rq.n_tok + ROWS - 1) / ROWS;
  // parts of the heads, up to 1024 workgroups (15,400 tokens into 4 bits 22 us, with 2048 23; single ones the same)
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(a.pc.h_kv, 1024 / groups));
  const size_t lds = turn_bytes(a.rq.rot.rot, std::max(ROWS, kRotateRows<DT, D>));
  paged_rotated4_kernel<DT, D, INTERLEAVED><<<(unsigned)(a.q_wgs + groups * a.parts), kStoreThreads, lds, stream>>>(a);
  return hipGetLastError();
}

template <int DT, int QT, int D, int SHIFT, bool INTERLEAVED, bool LONG> hipError_t append(AppendRotatedArgs a, hipStream_t stream) {
  const int64_t windows = ((int64_t)a.rq.n_tok + 63) / 64;
  // a run to a workgroup: those of a prompt, or single rows of many requests (up to 1024 workgroups: 2000 single rows 28.6 us,
  // with 512 37.8, with 2048 35.4); then parts of its heads, each of which forms the run's turns: 2048 workgroups of long runs
  // (72.1, with 1024 77.7, with 4096 73.5), 256 of short ones (256 single rows 10.5, with 1024 13.9; 128 8.7 and 9.4)
  constexpr int64_t kFill = LONG ? 2048 : 256;
  a.n_share = LONG ? std::max(1, 64 >> SHIFT) : (int)std::max<int64_t>(1, std::min<int64_t>(std::min(a.rq.n_tok, 64), 1024 / windows));
  constexpr int HEADS = LONG ? Tiling<DT, D, SHIFT, true>::HEADS : 2;
  const int most = (a.pc.h_kv + HEADS - 1) / HEADS;
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, kFill / (windows * a.n_share)));
  const size_t lds = turn_bytes(a.rq.rot.rot, std::max(kRotateRows<DT, D>, 1 << SHIFT));
  auto kernel = paged_rotated_kernel<DT, QT, D, SHIFT, INTERLEAVED, LONG>;
  if (lds > (64 << 10)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<(unsigned)(a.q_wgs + windows * a.n_share * a.parts), kStoreThreads, lds, stream>>>(a);
  return hipGetLastError();
}
template <int DT, int QT, int D, int SHIFT, bool INTERLEAVED> hipError_t append(const AppendRotatedArgs& a, hipStream_t stream) {
  return is_long(a.pc, a.rq.n_tok) ? append<DT, QT, D, SHIFT, INTERLEAVED, true>(a, stream)
                                   : append<DT, QT, D, SHIFT, INTERLEAVED, false>(a, stream);
}

}  // namespace

hipError_t launch_paged_append_rotated(const Paged& pc, const RotateArgs& rq, const void* k_new, const void* v_new,
                                       int64_t tok_stride, const int32_t* slots, hipStream_t stream) {
  AppendRotatedArgs a{pc, rq, k_new, v_new, (uint32_t)(tok_stride * (pc.dtype == kDtBf16 ? 2 : 4)), slots, 0, 1, 1};
  return dispatch(pc, [&](auto dt, auto qt, auto d, auto shift) {
    constexpr int RW = kRotateRows<dt.value, d.value>;
    if (rq.x) {
      const int64_t groups = ((int64_t)rq.n_tok + RW - 1) / RW;
      a.rq.parts = rotate_parts(groups, rq.heads);
      a.q_wgs = groups * a.rq.parts;
    }
    if constexpr (qt.value == kQtE2m1) {
      return rq.rot.interleaved ? append4<dt.value, d.value, true>(a, stream) : append4<dt.value, d.value, false>(a, stream);
    } else {
      return rq.rot.interleaved ? append<dt.value, qt.value, d.value, shift.value, true>(a, stream)
                                : append<dt.value, qt.value, d.value, shift.value, false>(a, stream);
    }
  });
}

}  // namespace kv
