// The paged cache of 8- or 4-bit codes on the host's side: its description as the kernels take it, and the
// launchers.  Arguments are validated by the C ABI layer before any of these is called.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace kv {

constexpr int kQtE4m3 = 0;
constexpr int kQtInt8 = 1;
constexpr int kQtE2m1 = 4;  // 4 bits, two to a byte

// Pools [n_blocks][h_kv][1 << shift][d] of codes and [n_blocks][h_kv] of scales (e2m1: d / 2 bytes to a row, and
// scale bytes [n_blocks][h_kv][d / 32][1 << shift]); row r of problem p is row r % R of block table[p][r / R],
// R = 1 << shift.
struct Paged {
  int dtype, qtype;
  int n_prob, h_q, h_kv, d;
  int shift;
  int n_blocks, table_stride, max_len;
  uint8_t* k;
  uint8_t* v;
  void* k_scale;
  void* v_scale;
  int32_t* table;
  int32_t* len;
  int group() const { return h_q / h_kv; }
};

// Block tables and slots (paged_tables.hip).
struct TablesArgs {
  const int32_t* len_in;  // [n_prob], null: 0
  const int32_t* add;     // [n_prob], null: 1
  const int32_t* free_blocks;  // [n_free], null: block i is i
  int n_free;
  const int32_t* taken_in;  // [1], null: 0
  int32_t* taken_out;       // [1], nullable
  int32_t* tok_off;         // [n_prob + 1]
  int32_t* blk_off;         // [n_prob + 1]
  int32_t* slots;           // [n_slots]
  int n_slots;
  bool slots_aligned;       // 16 bytes
  bool in_place;            // len_in, add or taken_in is written as an output
};
hipError_t launch_paged_tables(const Paged& pc, const TablesArgs& a, hipStream_t stream);

// Rows into the blocks (paged_store.hip).  tok_stride: elements between the rows of two tokens.
hipError_t launch_paged_append(const Paged& pc, const void* k_new, const void* v_new, int64_t tok_stride,
                               const int32_t* slots, int n_tok, hipStream_t stream);
hipError_t launch_paged_compact(const Paged& pc, const int32_t* lens, int max_len, const int64_t* tok_off,
                                const void* k, const void* v, const int32_t* sel_idx, int budget,
                                const int32_t* budgets, int keep_tail, hipStream_t stream);

// A rotation by positions (kv_rotary): freq [rot / 2] radians a position.
struct Rotary {
  bool interleaved;
  int rot;       // rotated elements of a head
  float sign;    // -1: by the opposite angle
  float factor;  // of the rotated elements
  const double* freq;
};
// Rows of `heads` heads of d elements, out (nullable) and their rotation; strides in elements between two tokens.
struct RotateArgs {
  Rotary rot;
  const void* x;
  void* out;
  int64_t x_stride, out_stride;
  const int32_t* pos;  // [n_tok]
  int n_tok, heads;
  int parts;  // workgroups that share the heads of a group of tokens
};
hipError_t launch_rotate(int dtype, int d, const RotateArgs& a, hipStream_t stream);
// Rows into the blocks with K rotated, and the rotated rows of q (rq.x null: none) in the same launch (paged_rotated.hip).
hipError_t launch_paged_append_rotated(const Paged& pc, const RotateArgs& rq, const void* k_new, const void* v_new,
                                       int64_t tok_stride, const int32_t* slots, hipStream_t stream);
// The caches' rows, contiguous (paged_read.hip).
hipError_t launch_paged_rows(const Paged& pc, const int64_t* row_off, int64_t n_rows, void* k_out, void* v_out,
                             hipStream_t stream);

// Attention over the blocks (paged_attention.hip).
struct PagedAttnArgs {
  Paged pc;
  const void* q;          // token t, head h: q_stride t + h d elements
  int64_t q_stride;
  const int32_t* tok_off;  // [n_prob + 1], null: one token per problem
  int n_tok, max_q;
  float c;  // softmax scale * log2(e)
  void* out;  // [n_tok][h_q][d], the queries' type
  int split_rows, n_split;
  float* part;  // [n_tok][h_q][n_split][d + 2] when n_split > 1
  // up to 32 columns over 4-bit blocks: workgroups that share a unit's rounds (0: one for each problem), and their prefix sums
  int shares;
  int32_t* prefix;
  int32_t* first;  // the problems that the shares begin in (null: not wanted)
  int group;           // h_q / h_kv, and its reciprocal in units of 2^-32, rounded up (0: a group of one)
  uint32_t group_inv;
};
// prompt_waves: 0 for paged_attention.hip's kernel, else the waves of paged_prompt.hip's (32 columns each).
struct PagedPlan {
  int split_rows, n_split, prompt_waves;
  int shares;  // of paged_attention4.hip's kernel, 0: whole problems
};
PagedPlan paged_plan(const Paged& pc, int max_q);
// Workgroups along the grid axis that the columns are on: the second one of paged_prompt.hip's kernel, with its splits,
// the first one of paged_attention.hip's, with the kv heads.  At most 65535: the limit of a second axis, and on the
// first what keeps the join's launch (256 threads a column) far below 2^32 threads.
int64_t paged_grid_groups(const Paged& pc, int max_q, const PagedPlan& plan);
size_t paged_ws_bytes(const Paged& pc, int n_tok, int max_q, const PagedPlan& plan);
hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedPlan& plan, hipStream_t stream);
// Up to 32 columns at a time over 4-bit blocks (paged_attention4.hip).
int paged4_shares(const Paged& pc, int max_q);
size_t paged4_prefix_bytes(const Paged& pc, int max_q, int shares);
size_t paged4_ws_bytes(const Paged& pc, int max_q, int shares);
hipError_t launch_paged_attention4(PagedAttnArgs a, hipStream_t stream);
// Blocks of a split that the prompt kernel of so many waves holds in LDS beside its tiles
// (two workgroups of four waves share a CU's 160 KB, one of eight has it alone).
constexpr int prompt_split_blocks(int waves) { return waves == 4 ? 256 : 4096; }
hipError_t launch_paged_prompt(const PagedAttnArgs& a, int waves, hipStream_t stream);

}  // namespace kv
