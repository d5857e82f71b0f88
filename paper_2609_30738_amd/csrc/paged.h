// The 8-bit paged cache on the host's side: its description as the kernels take it, and the
// launchers.  Arguments are validated by the C ABI layer before any of these is called.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace kv {

constexpr int kQtE4m3 = 0;
constexpr int kQtInt8 = 1;

// Pools [n_blocks][h_kv][1 << shift][d] of codes and [n_blocks][h_kv] of scales; row r of problem p is
// row r % R of block table[p][r / R], R = 1 << shift.
struct Paged {
  int dtype, qtype;
  int n_prob, h_q, h_kv, d;
  int shift;
  int n_blocks, table_stride, max_len;
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
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
};
// prompt_waves: 0 for paged_attention.hip's kernel, else the waves of paged_prompt.hip's (32 columns each).
struct PagedPlan {
  int split_rows, n_split, prompt_waves;
};
PagedPlan paged_plan(const Paged& pc, int max_q);
// Workgroups along the grid axis that the columns are on: the second one of paged_prompt.hip's kernel, with its splits,
// the first one of paged_attention.hip's, with the kv heads.  At most 65535: the limit of a second axis, and on the
// first what keeps the join's launch (256 threads a column) far below 2^32 threads.
int64_t paged_grid_groups(const Paged& pc, int max_q, const PagedPlan& plan);
size_t paged_ws_bytes(const Paged& pc, int n_tok, const PagedPlan& plan);
hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedPlan& plan, hipStream_t stream);
// Blocks of a split that the prompt kernel of so many waves holds in LDS beside its tiles
// (two workgroups of four waves share a CU's 160 KB, one of eight has it alone).
constexpr int prompt_split_blocks(int waves) { return waves == 4 ? 256 : 4096; }
hipError_t launch_paged_prompt(const PagedAttnArgs& a, int waves, hipStream_t stream);

}  // namespace kv
