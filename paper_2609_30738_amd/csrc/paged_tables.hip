// Block tables and slots of a paged cache from request lengths (kv_paged_tables).
//
// tables_scan_kernel: prefix sums of the new rows and of the new blocks over the problems, 1024 at a time, in
//   every workgroup for itself, the offsets and lengths written by the first; then each workgroup takes its
//   share of the rows' slots and of the blocks' table entries, finding the problem by bisection in LDS.
//   Inputs that are outputs too (lengths in place, the count of taken blocks in blk_off or taken_out) allow one
//   workgroup: the others' sums would read what it writes.  In the one, a value is read before the barrier that
//   its overwriting follows, or by the thread that overwrites it.  Many slots are then filled by a second launch,
//   tables_fill_kernel, from the first one's offsets, where a wave takes kWaveRows rows and finds the first one's
//   problem by looking at 64 offsets at a time.
//   Bound by latency: a step of 256 requests 5.6 us, 64 prompts of 1.1 million rows 9.3 us (as two launches 10.7;
//   four rows a thread instead of one 7.4 and 10.0).
#include <algorithm>

#include "paged.h"

namespace kv {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kFillThreads = 256;
constexpr int kWaveRows = 256;  // of a wave of the fill kernel, four a lane
constexpr int kMaxRows = 1 << 24;  // of a problem
// Slots up to which one workgroup fills them where lengths are updated in place, a launch less (4096 slots of 64
// requests 6.9 us, of 1024 requests 8.5, by two launches 9.5 and 12.5; 16384 of 1024 requests 20.7 and 13.8), and slots
// for each further workgroup where they are not.
constexpr int kFillInScan = 4096, kScanRows = 2048;

__device__ __forceinline__ int64_t wave_scan(int64_t v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

__device__ __forceinline__ int saturate(int64_t x) { return (int)min(x, (int64_t)INT32_MAX); }

// Entry `at` of the free list, -1 where there is none.
__device__ __forceinline__ int free_block(const Paged& pc, const TablesArgs& a, int64_t at) {
  if (at < 0 || at >= a.n_free) return -1;
  const int block = a.free_blocks ? a.free_blocks[at] : (int)at;
  return block < 0 || block >= pc.n_blocks ? -1 : block;
}

// Slot of row `row` of problem p.  have: the blocks it had before, base: the free list's place of its first new one.
__device__ __forceinline__ int slot_of(const Paged& pc, const TablesArgs& a, int p, int row, int have, int base) {
  const int j = row >> pc.shift;
  if ((uint32_t)j >= (uint32_t)pc.table_stride) return -1;
  const int block = j < have ? pc.table[(int64_t)p * pc.table_stride + j] : free_block(pc, a, (int64_t)base + (j - have));
  return block < 0 || block >= pc.n_blocks ? -1 : (block << pc.shift) + (row & ((1 << pc.shift) - 1));
}

// The table's entry of the new block at place `at` of the free list.
__device__ __forceinline__ void enter(const Paged& pc, const TablesArgs& a, int p, int at, int have, int base) {
  const int64_t j = (int64_t)have + (at - base);
  if (j >= 0 && j < pc.table_stride) pc.table[(int64_t)p * pc.table_stride + j] = free_block(pc, a, at);
}

// The last of offsets[0 .. n) that is at most i, by bisection (offsets[0] <= i).
__device__ __forceinline__ int last_at_most(const int32_t* offsets, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace

template <bool kFill>
__global__ __launch_bounds__(kThreads) void tables_scan_kernel(Paged pc, TablesArgs a) {
  __shared__ int64_t sum_rows[kWaves], sum_blocks[kWaves];
  __shared__ int32_t first_row[kThreads], first_block[kThreads], old_rows[kThreads];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t id = (int64_t)blockIdx.x * kThreads + tid, ids = (int64_t)gridDim.x * kThreads;
  const int R = 1 << pc.shift;
  const int64_t cap = (int64_t)pc.table_stride << pc.shift;
  int64_t rows0 = 0, blocks0 = a.taken_in ? a.taken_in[0] : 0;
  for (int base = 0; base < pc.n_prob; base += kThreads) {
    const int p = base + tid;
    int old = 0, add = 0;
    if (p < pc.n_prob) {
      old = a.len_in ? min(max(a.len_in[p], 0), kMaxRows) : 0;
      add = a.add ? min(max(a.add[p], 0), kMaxRows) : 1;
    }
    const int64_t have = (min((int64_t)old, cap) + R - 1) >> pc.shift;
    const int64_t need = (min((int64_t)old + add, cap) + R - 1) >> pc.shift;
    const int64_t r = wave_scan(add), b = wave_scan(need - have);
    if (lane == 63) {
      sum_rows[wave] = r;
      sum_blocks[wave] = b;
    }
    __syncthreads();
    int64_t rb = rows0, bb = blocks0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) {
        rb += sum_rows[w];
        bb += sum_blocks[w];
      }
      rows0 += sum_rows[w];
      blocks0 += sum_blocks[w];
    }
    const int row = saturate(rb + r - add), block = saturate(bb + b - (need - have));
    if (p < pc.n_prob && blockIdx.x == 0) {
      a.tok_off[p] = row;
      a.blk_off[p] = block;
      pc.len[p] = old + add;
    }
    if constexpr (kFill) {
      first_row[tid] = row;
      first_block[tid] = block;
      old_rows[tid] = old;
      __syncthreads();
      const int n = min(pc.n_prob - base, kThreads), end = saturate(rows0);
      for (int64_t i = first_row[0] + id; i < min(end, a.n_slots); i += ids) {
        const int q = last_at_most(first_row, n, (int)i);
        a.slots[i] = slot_of(pc, a, base + q, old_rows[q] + ((int)i - first_row[q]), (old_rows[q] + R - 1) >> pc.shift,
                             first_block[q]);
      }
      for (int64_t i = first_block[0] + id; i < saturate(blocks0); i += ids) {
        const int q = last_at_most(first_block, n, (int)i);
        enter(pc, a, base + q, (int)i, (old_rows[q] + R - 1) >> pc.shift, first_block[q]);
      }
    }
    __syncthreads();
  }
  if (id == 0) {
    a.tok_off[pc.n_prob] = saturate(rows0);
    a.blk_off[pc.n_prob] = saturate(blocks0);
    if (a.taken_out) a.taken_out[0] = saturate(blocks0);
  }
  if constexpr (kFill)
    for (int64_t i = rows0 + id; i < a.n_slots; i += ids) a.slots[i] = -1;
}

namespace {

// The last of offsets[0 .. n) that is at most i (offsets[0] <= i), by a whole wave: 64 evenly spaced ones at a time.
__device__ __forceinline__ int wave_last_at_most(const int32_t* offsets, int n, int64_t i) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const bool in = lane * step < n && offsets[lo + lane * step] <= i;
    const int k = __popcll(__ballot(in)) - 1;  // the first is
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

}  // namespace

__global__ __launch_bounds__(kFillThreads) void tables_fill_kernel(Paged pc, TablesArgs a) {
  const int lane = threadIdx.x & 63, R = 1 << pc.shift;
  const int64_t wave = (int64_t)blockIdx.x * (kFillThreads / 64) + (threadIdx.x >> 6);
  const int64_t waves = (int64_t)gridDim.x * (kFillThreads / 64);
  const int total = a.tok_off[pc.n_prob];
  auto rows_before = [&](int p) { return pc.len[p] - (a.tok_off[p + 1] - a.tok_off[p]); };
  for (int64_t first = wave * kWaveRows; first < a.n_slots; first += waves * kWaveRows) {
    const int p = first < total ? wave_last_at_most(a.tok_off, pc.n_prob, first) : 0;
    if (first < total && first + kWaveRows <= a.tok_off[p + 1]) {  // all of one problem
      const int old = rows_before(p), have = (old + R - 1) >> pc.shift, base = a.blk_off[p];
      const int64_t i = first + 4 * lane;
      const int row = old + (int)(i - a.tok_off[p]);
      int32_t s[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] = slot_of(pc, a, p, row + k, have, base);
      if (i + 4 <= a.n_slots && a.slots_aligned) {
        *reinterpret_cast<int4*>(a.slots + i) = make_int4(s[0], s[1], s[2], s[3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k < a.n_slots) a.slots[i + k] = s[k];
      }
      continue;
    }
    for (int64_t i = first + lane; i < min(first + kWaveRows, (int64_t)a.n_slots); i += 64) {
      int slot = -1;  // behind the last row
      if (i < total) {
        const int q = p + last_at_most(a.tok_off + p, pc.n_prob - p, (int)i), old = rows_before(q);
        slot = slot_of(pc, a, q, old + ((int)i - a.tok_off[q]), (old + R - 1) >> pc.shift, a.blk_off[q]);
      }
      a.slots[i] = slot;
    }
  }
  const int64_t end = a.blk_off[pc.n_prob];
  for (int64_t first = a.blk_off[0] + wave * 64; first < end; first += waves * 64) {
    const int p = wave_last_at_most(a.blk_off, pc.n_prob, first);
    if (first + lane >= end) continue;
    const int i = (int)first + lane, q = p + last_at_most(a.blk_off + p, pc.n_prob - p, i);
    enter(pc, a, q, i, (rows_before(q) + R - 1) >> pc.shift, a.blk_off[q]);
  }
}

hipError_t launch_paged_tables(const Paged& pc, const TablesArgs& a, hipStream_t stream) {
  if (!a.in_place || a.n_slots <= kFillInScan) {
    const int wgs = a.in_place ? 1 : std::max(1, std::min((a.n_slots + kScanRows - 1) / kScanRows, 256));
    tables_scan_kernel<true><<<(unsigned)wgs, kThreads, 0, stream>>>(pc, a);
    return hipGetLastError();
  }
  tables_scan_kernel<false><<<1, kThreads, 0, stream>>>(pc, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int kWgRows = kWaveRows * (kFillThreads / 64);
  const int wgs = std::min((a.n_slots + kWgRows - 1) / kWgRows, 4096);
  tables_fill_kernel<<<(unsigned)wgs, kFillThreads, 0, stream>>>(pc, a);
  return hipGetLastError();
}

}  // namespace kv
