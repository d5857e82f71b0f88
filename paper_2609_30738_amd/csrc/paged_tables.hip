// Block tables and slots of a paged cache from request lengths (kv_paged_tables).
//
// tables_scan_kernel: one workgroup takes the prefix sums of the new rows and of the new blocks over the
//   problems, 1024 at a time, and writes the offsets and the new lengths; for few slots it also fills
//   them.  tables_fill_kernel: one thread per new row finds its problem by bisection of the row offsets,
//   its block from the free list (or the table, for a block in use), and writes its slot; the thread
//   of a block's first row writes the table's entry.  Everything a thread of the second step reads is the
//   first step's output, so len_in may be the cache's own lengths.
#include <algorithm>

#include "paged.h"

namespace kv {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kFillThreads = 256;
constexpr int kMaxRows = 1 << 24;  // of a problem
// Slots up to which the scan's workgroup fills them itself, a launch less.
constexpr int kFillInScan = 4096;

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

// Slot (and at a block's first row the table's entry) of new row i of the batch.
__device__ __forceinline__ void fill_row(const Paged& pc, const TablesArgs& a, int i) {
  int lo = 0, hi = pc.n_prob;  // the last problem with tok_off <= i
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.tok_off[mid] <= i) lo = mid;
    else hi = mid;
  }
  const int p = lo, first = a.tok_off[p];
  const int old = pc.len[p] - (a.tok_off[p + 1] - first);
  const int row = old + (i - first), j = row >> pc.shift, R = 1 << pc.shift;
  int block = -1;
  if (j < pc.table_stride) {
    int32_t* entry = pc.table + (int64_t)p * pc.table_stride + j;
    const int have = (old + R - 1) >> pc.shift;
    if (j < have) {
      block = *entry;
    } else {
      const int64_t at = (int64_t)a.blk_off[p] + (j - have);
      if (at >= 0 && at < a.n_free) block = a.free_blocks ? a.free_blocks[at] : (int)at;
      if (block < 0 || block >= pc.n_blocks) block = -1;
      if ((row & (R - 1)) == 0) *entry = block;
    }
    if (block < 0 || block >= pc.n_blocks) block = -1;
  }
  if (i < a.n_slots) a.slots[i] = block < 0 ? -1 : (block << pc.shift) + (row & (R - 1));
}

// Rows first, first + stride, ... of the batch, then -1 in the slots behind the last one.
__device__ __forceinline__ void fill_rows(const Paged& pc, const TablesArgs& a, int64_t first, int64_t stride) {
  const int total = a.tok_off[pc.n_prob];
  for (int64_t i = first; i < total; i += stride) fill_row(pc, a, (int)i);
  for (int64_t i = first; i < a.n_slots; i += stride)
    if (i >= total) a.slots[i] = -1;
}

}  // namespace

__global__ __launch_bounds__(kThreads) void tables_scan_kernel(Paged pc, TablesArgs a, bool fill) {
  __shared__ int64_t sum_rows[kWaves], sum_blocks[kWaves];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
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
    if (p < pc.n_prob) {
      a.tok_off[p] = saturate(rb + r - add);
      a.blk_off[p] = saturate(bb + b - (need - have));
      pc.len[p] = old + add;
    }
    __syncthreads();
  }
  if (tid == 0) {
    a.tok_off[pc.n_prob] = saturate(rows0);
    a.blk_off[pc.n_prob] = saturate(blocks0);
    if (a.taken_out) a.taken_out[0] = saturate(blocks0);
  }
  if (fill) {
    __threadfence_block();
    __syncthreads();
    fill_rows(pc, a, tid, kThreads);
  }
}

__global__ __launch_bounds__(kFillThreads) void tables_fill_kernel(Paged pc, TablesArgs a) {
  fill_rows(pc, a, (int64_t)blockIdx.x * kFillThreads + threadIdx.x, (int64_t)gridDim.x * kFillThreads);
}

hipError_t launch_paged_tables(const Paged& pc, const TablesArgs& a, hipStream_t stream) {
  const bool one = a.n_slots <= kFillInScan;
  tables_scan_kernel<<<1, kThreads, 0, stream>>>(pc, a, one);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  const int wgs = std::min((a.n_slots + kFillThreads - 1) / kFillThreads, 8192);
  tables_fill_kernel<<<(unsigned)wgs, kFillThreads, 0, stream>>>(pc, a);
  return hipGetLastError();
}

}  // namespace kv
