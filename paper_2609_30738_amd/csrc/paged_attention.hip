// Attention of the last tokens of every problem over its 8-bit paged cache (kv_paged_attention), and the join of the
// splits of every paged cache.
//
// paged_attn_kernel: one workgroup of four waves per (kv head and group of columns, split of the rows,
//   problem).  A column is a (token, query head) pair of the kv head; a wave takes 16 NT of them
//   against 32 rows a step:
//     S^T = K Q^T by v_mfma_f32_16x16x32_bf16, 16 rows a tile: the codes are exact in bf16, and the
//   block's scale multiplies the logits, not the keys.  Lane l of the accumulator holds column l % 16 and
//   four rows, so the column's running maximum and sum stay in the lane, and the eight weights of a
//   step's two tiles are exactly the eight of the lane's operand of
//     O^T = V^T P^T.
//   Row 4 j + l / 16 of a tile stands for row l / 16 * 4 + j of the accumulator, so that a load of V reads
//   four whole consecutive rows; the lane's operand of V is transposed in registers.
//   fp32 queries and weights are taken as three bf16 terms each (24 bits): the matrix products lose nothing
//   of the operands beyond that, and accumulate in fp32.  With bf16 queries the weights are two terms for up
//   to 16 columns, where the second one is free beside the loads, and one for more (2^-9 of each, a step of
//   the output; five tokens of 16 requests 59 us, with two terms 64; now 48).
//   The reference of a column's weights is raised, and the sums rescaled, only when a logit exceeds it by
//   more than kSlack octaves; weights are 2^(t - m - kSlack), so that none exceeds 1.
//   The grid's fastest axis is the kv head, so that every XCD gets as many of the splits that reach past a cache's end
//   as the others (with the splits fastest, 16 of them put each on an XCD of its own: 64 caches of up to 8000 rows
//   151 us, now 121, 16 of up to 32768 146, now 118).
//   The four waves are merged through LDS; with several splits the partial sums go to the workspace and
//   paged_combine_kernel joins them.
//   Bound by the cache's reads: one token over 32 caches of 32768 rows (e4m3, 8 heads of 128, 2.0 GB) 335 us, 6.0 TB/s
//   of the 6.9 that streaming reads reach here; 24 ragged ones of up to 24001 rows (int8, eight query heads to a
//   kv head, 0.66 GB) 137 us, 4.8 TB/s: the last splits of unequal caches leave CUs idle; over 32 caches of 100 rows
//   6.0 us, fp32 over four of 4097 rows 11.7 us with the join: latency.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "paged.h"
#include "paged_codes.h"
#include "paged_span.h"

namespace kv {

namespace {

constexpr int kThreads = kAttnThreads;
constexpr int kWaves = kAttnWaves;
constexpr int kStep = 32;               // rows of a wave's step

// Waves per SIMD that the registers are held to: as many as run without spills.
template <int DT, int D, int NT> constexpr int kMinWaves = (NT == 1 ? 3 : 2) - (DT == kDtF32 && D == 128 ? 1 : 0);

}  // namespace

template <int DT, int QT, int D, int NT>
__global__ __launch_bounds__(kThreads, (kMinWaves<DT, D, NT>)) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int NS = D / 32;                       // matrix steps over the head dimension
  constexpr int NI = D / 16;                       // 16-wide tiles of the output
  constexpr int KH = D / 64;                       // 16-byte loads of a key
  constexpr int VW = D / 64;                       // words of a value row that a lane loads
  constexpr int QN = DT == kDtBf16 ? 1 : 3;        // bf16 terms of a query
  constexpr int PN = DT == kDtF32 ? 3 : (NT == 1 ? 2 : 1);  // and of a weight
  constexpr int COLS = 16 * NT;
  __shared__ int32_t sh_block[kMaxSplitBlocks];
  __shared__ float sh_ks[kMaxSplitBlocks], sh_vs[kMaxSplitBlocks];
  __shared__ float sh_m[kWaves][16], sh_s[kWaves][16];
  extern __shared__ __align__(16) float sh_acc[];  // [kWaves][up to 16 columns][D]

  const int p = blockIdx.z, g = blockIdx.x % a.pc.h_kv, cg = blockIdx.x / a.pc.h_kv, G = a.pc.h_q / a.pc.h_kv;
  // (the problems' splits start one further each: with fewer heads than XCDs, these take long caches' ends in turn)
  const int split = a.n_split > 1 ? (int)((blockIdx.y + (uint32_t)p) % (uint32_t)a.n_split) : 0;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = lane & 15, kg = lane >> 4;
  const int shift = a.pc.shift, R = 1 << shift;
  const int r0 = split * a.split_rows;
  // the split's table entries load beside the lengths
  const int entry = (r0 >> shift) + tid;
  const int id = tid << shift < a.split_rows && entry < a.pc.table_stride
                     ? a.pc.table[(int64_t)p * a.pc.table_stride + entry] : -1;
  const Span sp = span_of(a, p);
  const int col0 = cg * COLS;
  const int n_cols = min(sp.n_tok * G - col0, COLS);
  if (n_cols <= 0) return;
  const int vis_max = sp.visible((col0 + n_cols - 1) / G);
  const int vis_min = sp.visible(col0 / G);
  const int r1 = min(vis_max, r0 + a.split_rows);
  if (r0 >= r1 && a.n_split > 1) return;  // the join reads the splits below a column's last row

  // blocks and scales of the split's rows: the scales arrive beside the first codes
  const bool has = tid << shift < r1 - r0 && id >= 0 && id < a.pc.n_blocks;
  if (tid < kMaxSplitBlocks) sh_block[tid] = has ? id : -1;
  __syncthreads();
  const int64_t scale_at = (int64_t)(has ? id : 0) * a.pc.h_kv + g;
  const float my_ks = has ? static_cast<const float*>(a.pc.k_scale)[scale_at] * a.c : 0.f, my_vs = has ? static_cast<const float*>(a.pc.v_scale)[scale_at] : 0.f;

  // the codes of 32 rows: row 16 t + 4 j + kg for V, and for K the row that holds the accumulator's row n
  u32x4_t xk[2][KH];
  uint32_t xv[2][4][VW];
  // a wave-uniform address and a lane's 32-bit offset
  const uint32_t k_lane = (4 * (n & 3) + (n >> 2)) * D + 16 * kg, v_lane = kg * D + n * (4 * VW);
  auto tile_at = [&](int rb, int t) {
    const int r = min(rb + 16 * t, (r1 - 1) & ~15) - r0;
    const int64_t id = max(__builtin_amdgcn_readfirstlane(sh_block[r >> shift]), 0);
    return ((id * a.pc.h_kv + g) << shift) * D + ((r & (R - 1)) * D);
  };
  auto load_k = [&](int rb) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t* ks = a.pc.k + tile_at(rb, t);
#pragma unroll
      for (int i = 0; i < KH; ++i) xk[t][i] = load_code<NT == 1>(reinterpret_cast<const u32x4_t*>(ks + (k_lane + 64 * i)));
    }
  };
  auto load_v = [&](int rb) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t* vs = a.pc.v + tile_at(rb, t);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (VW == 2) {
          const u32x2_t u = load_code<NT == 1>(reinterpret_cast<const u32x2_t*>(vs + (v_lane + 4 * j * D)));
          xv[t][j][0] = u[0];
          xv[t][j][1] = u[1];
        } else {
          xv[t][j][0] = load_code<NT == 1>(reinterpret_cast<const uint32_t*>(vs + (v_lane + 4 * j * D)));
        }
      }
    }
  };

  constexpr int kRound = kWaves * kStep;
  const int rb0 = r0 + wave * kStep;
  if (rb0 < r1) {
    load_k(rb0);
    load_v(rb0);
  }
  // the queries' operand: column n, elements 64 (s / 2) + 16 kg + 8 (s % 2) .. + 7 (D = 64: 16 kg + 8 s)
  u32x4_t qf[NT][NS][QN];
  int vis[NT];
#pragma unroll
  for (int ct = 0; ct < NT; ++ct) {
    const int col = col0 + 16 * ct + n;
    const bool live = 16 * ct + n < n_cols;
    const int j = live ? col / G : 0, h = live ? col % G : 0;
    vis[ct] = live ? sp.visible(j) : 0;
    const int64_t at = (int64_t)(sp.tok0 + j) * a.q_stride + (int64_t)(g * G + h) * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int e = 64 * (s >> 1) + 16 * kg + 8 * (s & 1);
      if constexpr (DT == kDtBf16) {
        qf[ct][s][0] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.q) + at + e);
      } else {
        const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at + e);
        const float4 x = src[0], y = src[1];
        const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        split_terms<QN>(f, qf[ct][s]);
      }
    }
  }
  if (tid < kMaxSplitBlocks) {
    sh_ks[tid] = my_ks;
    sh_vs[tid] = my_vs;
  }
  __syncthreads();

  float m[NT], mu[NT], sum[NT];  // mu: m, or 0 before the first finite logit
  f32x4v acc[NT][NI];
#pragma unroll
  for (int ct = 0; ct < NT; ++ct) {
    m[ct] = -INFINITY;
    mu[ct] = 0.f;
    sum[ct] = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) acc[ct][i] = f32x4v{0.f, 0.f, 0.f, 0.f};
  }

  // A step of 32 rows; the codes of the step at `next` (if any) load as this one's are used up.
  auto step = [&](int rb, int next) __attribute__((always_inline)) {
    int blk[2];
    float ksc[2], vsc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = (min(rb + 16 * t, (r1 - 1) & ~15) - r0) >> shift;
      blk[t] = __builtin_amdgcn_readfirstlane(sh_block[i]);
      ksc[t] = sh_ks[i];
      vsc[t] = sh_vs[i];
    }
    // its rows are not all visible to every column, or a block is missing
    const bool masked = rb + kStep > vis_min || (blk[0] | blk[1]) < 0;
    uint64_t nan_rows = 0;
    if (masked) {
      // a row without a column that sees it holds anything: zero its values, so that 0 times them is 0
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = blk[t] >= 0 && rb + 16 * t + 4 * j + kg < r1;
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            xv[t][j][w] = in ? xv[t][j][w] : 0u;
            if constexpr (QT == kQtE4m3) {
              const uint32_t u = (xv[t][j][w] & 0x7F7F7F7Fu) + 0x01010101u;  // 0x80 in a byte of 0x7F
              nan_rows |= __ballot((u & 0x80808080u) != 0);
            }
          }
        }
    }

    float lg[NT][8];
    // (codes are converted here, not where they were loaded a step before: registers)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < KH; ++i)
        asm volatile("" : "+v"(xk[t][i][0]), "+v"(xk[t][i][1]), "+v"(xk[t][i][2]), "+v"(xk[t][i][3]));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4v s4[NT];
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) s4[ct] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const u32x2_t lo = decode4_bf16<QT>(xk[t][s >> 1][2 * (s & 1)]);
        const u32x2_t hi = decode4_bf16<QT>(xk[t][s >> 1][2 * (s & 1) + 1]);
        const u32x4_t kf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
        for (int ct = 0; ct < NT; ++ct)
#pragma unroll
          for (int q = QN - 1; q >= 0; --q) s4[ct] = mfma16(kf, qf[ct][s][q], s4[ct]);
      }
#pragma unroll
      for (int ct = 0; ct < NT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float l = s4[ct][j] * ksc[t];
          if (masked && (blk[t] < 0 || rb + 16 * t + 4 * j + kg >= vis[ct])) l = -INFINITY;
          lg[ct][4 * t + j] = l;
        }
    }
    if (next < r1) load_k(next);
    u32x4_t pf[NT][PN];
    bool over = false;
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      float tm = lg[ct][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) tm = fmaxf(tm, lg[ct][e]);
      over = over || tm > m[ct] + kSlack;
    }
    if (__ballot(over)) {
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        float tm = lg[ct][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) tm = fmaxf(tm, lg[ct][e]);
        const float mn = fmaxf(m[ct], column_max(tm));
        const float f = m[ct] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[ct] - mn);
        m[ct] = mn;
        mu[ct] = mn == -INFINITY ? 0.f : mn;
        sum[ct] *= f;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[ct][i][j] *= f;
      }
    }
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = __builtin_amdgcn_exp2f(lg[ct][e] - mu[ct]) * kSlackScale;
        sum[ct] += w[e];
        w[e] *= vsc[e >> 2];
      }
      split_terms<PN>(w, pf[ct]);
    }

    if (QT == kQtE4m3 && nan_rows) {
      // a NaN counts for the columns that see its row alone: these are marked by a product of indicators,
      // and it leaves the codes
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        u32x4_t seen;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const int r = rb + 16 * (e >> 2) + 4 * (e & 3) + kg;
          seen[e >> 1] = (r < vis[ct] ? 0x3F80u : 0u) | (r + 4 < vis[ct] ? 0x3F800000u : 0u);
        }
#pragma unroll
        for (int w = 0; w < VW; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u32x4_t nf;
#pragma unroll
            for (int e = 0; e < 8; e += 2)
              nf[e >> 1] = ((xv[e >> 2][e & 3][w] >> (8 * i) & 0x7Fu) == 0x7Fu ? 0x3F80u : 0u) |
                           ((xv[e >> 2][(e & 3) + 1][w] >> (8 * i) & 0x7Fu) == 0x7Fu ? 0x3F800000u : 0u);
            const f32x4v hit = mfma16(nf, seen, f32x4v{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (hit[j] > 0.f) acc[ct][4 * w + i][j] = NAN;
          }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            const uint32_t u = (((xv[t][j][w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
            xv[t][j][w] &= ~(u * 0xFFu);
          }
    }
    // V^T: eight rows' words of four elements, transposed to four elements' operands
#pragma unroll
    for (int w = 0; w < VW; ++w) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        asm volatile("" : "+v"(xv[t][0][w]), "+v"(xv[t][1][w]), "+v"(xv[t][2][w]), "+v"(xv[t][3][w]));
      uint32_t b[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i % 2 == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            b[e] = i == 0 ? decode2_bf16<QT, 0>(xv[e >> 2][e & 3][w]) : decode2_bf16<QT, 1>(xv[e >> 2][e & 3][w]);
        }
        u32x4_t vf;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          vf[e] = __builtin_amdgcn_perm(b[2 * e + 1], b[2 * e], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int ct = 0; ct < NT; ++ct)
#pragma unroll
          for (int q = PN - 1; q >= 0; --q) acc[ct][4 * w + i] = mfma16(vf, pf[ct][q], acc[ct][4 * w + i]);
      }
    }
    if (next < r1) load_v(next);
  };

  for (int rb = rb0; rb < r1; rb += kRound) step(rb, rb + kRound);  // the waves' steps in turn

  // merge of the waves, 16 columns at a time: element 4 VW (4 kg + j) + 4 w + i of column n
#pragma unroll
  for (int ct = 0; ct < NT; ++ct) {
    const int cols = min(n_cols - 16 * ct, 16);
    if (cols <= 0) break;
    const float s = column_sum(sum[ct]);
    if (kg == 0) {
      sh_m[wave][n] = m[ct];
      sh_s[wave][n] = s;
    }
    if (n < cols) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < VW; ++w)
          *reinterpret_cast<float4*>(&sh_acc[(wave * cols + n) * D + (4 * kg + j) * 4 * VW + 4 * w]) =
              make_float4(acc[ct][4 * w][j], acc[ct][4 * w + 1][j], acc[ct][4 * w + 2][j], acc[ct][4 * w + 3][j]);
    }
    __syncthreads();
    for (int idx = tid; idx < cols * D; idx += kThreads) {
      const int cc = idx / D, e = idx % D;
      float M = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) M = fmaxf(M, sh_m[i][cc]);
      float S = 0.f, A = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float f = part_weight(sh_m[i][cc], M);
        S = fmaf(sh_s[i][cc], f, S);
        A = fmaf(sh_acc[(i * cols + cc) * D + e], f, A);
      }
      const int col = col0 + 16 * ct + cc;
      const int64_t row = (int64_t)(sp.tok0 + col / G) * a.pc.h_q + g * G + col % G;
      if (a.n_split == 1) {
        store_out<DT>(a.out, row * D + e, A, S);
      } else {
        float* pt = a.part + (row * a.n_split + split) * (D + 2);
        if (e == 0) {
          pt[0] = M;
          pt[1] = S;
        }
        pt[2 + e] = A;
      }
    }
    if (ct + 1 < NT) __syncthreads();
  }
}

// One workgroup per (column, kv head, problem): the splits below the column's last visible row, the waves' in
// turn, kJoin at a time in flight.
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void paged_combine_kernel(PagedAttnArgs a) {
  constexpr int E = D / 64, kJoin = 4;
  __shared__ float sh_a[kWaves][D], sh_m[kWaves], sh_s[kWaves];
  const int col = blockIdx.x, g = blockIdx.y, p = blockIdx.z, G = a.pc.h_q / a.pc.h_kv;
  const Span sp = span_of(a, p);
  if (col >= sp.n_tok * G) return;
  const int64_t row = (int64_t)(sp.tok0 + col / G) * a.pc.h_q + g * G + col % G;
  const int n_split = (sp.visible(col / G) + a.split_rows - 1) / a.split_rows;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const float* part = a.part + row * a.n_split * (D + 2);
  float m = -INFINITY, S = 0.f, A[E];
#pragma unroll
  for (int e = 0; e < E; ++e) A[e] = 0.f;
  for (int i = wave; i < n_split; i += kJoin * kWaves) {
    float xm[kJoin], xs[kJoin], xa[kJoin][E];
#pragma unroll
    for (int j = 0; j < kJoin; ++j) {
      const bool in = i + j * kWaves < n_split;
      const float* x = part + (int64_t)(in ? i + j * kWaves : i) * (D + 2);
      xm[j] = in ? x[0] : -INFINITY;
      xs[j] = in ? x[1] : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) xa[j][e] = in ? x[2 + E * lane + e] : 0.f;
    }
    float mn = m;
#pragma unroll
    for (int j = 0; j < kJoin; ++j) mn = fmaxf(mn, xm[j]);
    const float f = part_weight(m, mn);
    S *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) A[e] *= f;
#pragma unroll
    for (int j = 0; j < kJoin; ++j) {
      const float w = part_weight(xm[j], mn);
      S = fmaf(xs[j], w, S);
#pragma unroll
      for (int e = 0; e < E; ++e) A[e] = fmaf(xa[j][e], w, A[e]);
    }
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) sh_a[wave][E * lane + e] = A[e];
  if (lane == 0) {
    sh_m[wave] = m;
    sh_s[wave] = S;
  }
  __syncthreads();
  if (tid >= D) return;
  float M = -INFINITY, total = 0.f, out = 0.f;
#pragma unroll
  for (int q = 0; q < kWaves; ++q) M = fmaxf(M, sh_m[q]);
#pragma unroll
  for (int q = 0; q < kWaves; ++q) {
    const float f = part_weight(sh_m[q], M);
    total = fmaf(sh_s[q], f, total);
    out = fmaf(sh_a[q][tid], f, out);
  }
  store_out<DT>(a.out, row * D + tid, out, total);
}

namespace {

// 16-wide column tiles of a wave: one for up to 16 columns, else two.
int column_tiles(int max_q, int group) { return max_q * group <= 16 ? 1 : 2; }
int column_groups(int max_q, int group) {
  const int w = 16 * column_tiles(max_q, group);
  return (int)(((int64_t)max_q * group + w - 1) / w);
}

}  // namespace

PagedPlan paged_plan(const Paged& pc, int max_q) {
  const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(pc.max_len, (int64_t)pc.table_stride << pc.shift));
  const int64_t cols = (int64_t)max_q * pc.group();
  PagedPlan plan;
  plan.prompt_waves = plan.shares = 0;
  int64_t n = 1, units;
  if (pc.dtype == kDtBf16 && cols > 32) {  // (20 columns 51 us in paged_attn_kernel, 85 in the other)
    plan.prompt_waves = cols <= 128 ? 4 : 8;
    units = (int64_t)pc.n_prob * pc.h_kv * ((cols + 32 * plan.prompt_waves - 1) / (32 * plan.prompt_waves));
    // one round of 256 workgroups in splits of at least 512 rows: more splits cost more in the join than they even
    // out (2048 tokens of one prompt 70 us whole, 153 in two splits; 40 tokens over 32768 rows 47 us in 32 splits,
    // 61 in 64)
    n = std::max<int64_t>(1, std::min<int64_t>(256 / units, (rows + 511) / 512));
  } else {
    // Up to 512 rows a unit stays whole (500 rows of 64 units 8.2 us whole, 9.1 split and joined; of 512 units 15.1
    // and 22.3).  Longer ones get 2304 workgroups in splits of at least 512 rows.  That is three rounds of the 768 that
    // fit the chip with one column tile (bf16, d = 128), so that caches of unequal length even out: 24 of up to 16001
    // rows 91 us, with 1536 104, 64 of up to 16384 and 2 heads 64 and 71, 32 of up to 4000 37.5 and 41.1; caches of one
    // length pay for it, 24 of 13000 rows 109 and 105.  Two column tiles let 512 fit, fp32 512 and 256, d = 64 more.  The
    // number is the same for all: five tokens over 16 caches of up to 6001 rows 42 us, as with 768 to 3456 (fp32 80, with
    // 768 74), over 24 of up to 24001 168 and with 1536 167, over 24 of 13000 150 and 137, one fp32 token over 24 of up
    // to 16001 100 and 104.  Where the splits are few, 512 workgroups of at least 256 rows (8 units of 2000 rows 9.4 us, in splits of 512 rows 12.0; of 32768 rows in
    // 128 splits 25.9 us, in 64 20.2).
    units = (int64_t)pc.n_prob * pc.h_kv * column_groups(max_q, pc.group());
    auto splits = [&](int64_t wgs, int64_t least) { return std::min(wgs / units, (rows + least - 1) / least); };
    if (rows > 512) n = std::max<int64_t>(1, std::max(splits(2304, 512), splits(512, 256)));
  }
  int64_t split = ((rows + n - 1) / n + 127) / 128 * 128;
  split = std::min<int64_t>(split, plan.prompt_waves ? (int64_t)prompt_split_blocks(plan.prompt_waves) << pc.shift : kMaxSplitRows);
  plan.split_rows = (int)split;
  plan.n_split = (int)((rows + split - 1) / split);
  if (pc.qtype == kQtE2m1 && !plan.prompt_waves && plan.n_split > 1) plan.shares = paged4_shares(pc, max_q);
  return plan;
}

int64_t paged_grid_groups(const Paged& pc, int max_q, const PagedPlan& plan) {
  const int64_t cols = (int64_t)max_q * pc.group();
  if (plan.prompt_waves) return (cols + 32 * plan.prompt_waves - 1) / (32 * plan.prompt_waves) * plan.n_split;
  return (int64_t)pc.h_kv * column_groups(max_q, pc.group());
}

size_t paged_ws_bytes(const Paged& pc, int n_tok, int max_q, const PagedPlan& plan) {
  if (plan.shares) return paged4_ws_bytes(pc, max_q, plan.shares);
  if (plan.n_split == 1) return 0;
  return (size_t)n_tok * pc.h_q * plan.n_split * (pc.d + 2) * sizeof(float);
}

namespace {

template <int DT, int QT, int D> hipError_t attend(const PagedAttnArgs& a, hipStream_t stream) {
  const int G = a.pc.group(), nt = column_tiles(a.max_q, G), groups = column_groups(a.max_q, G);
  const dim3 grid((unsigned)(a.pc.h_kv * groups), (unsigned)a.n_split, (unsigned)a.pc.n_prob);
  const size_t lds = (size_t)kWaves * std::min(a.max_q * G, 16) * D * sizeof(float);
  if (nt == 1) paged_attn_kernel<DT, QT, D, 1><<<grid, kThreads, lds, stream>>>(a);
  else paged_attn_kernel<DT, QT, D, 2><<<grid, kThreads, lds, stream>>>(a);
  return hipGetLastError();
}

template <int DT, int D> hipError_t combine(const PagedAttnArgs& a, hipStream_t stream) {
  const dim3 cols((unsigned)(a.max_q * a.pc.group()), (unsigned)a.pc.h_kv, (unsigned)a.pc.n_prob);
  paged_combine_kernel<DT, D><<<cols, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedPlan& plan, hipStream_t stream) {
  const bool bf16 = a.pc.dtype == kDtBf16;
  auto d = [&](auto dt, auto qt) {
    return a.pc.d == 64 ? attend<dt.value, qt.value, 64>(a, stream) : attend<dt.value, qt.value, 128>(a, stream);
  };
  auto q = [&](auto dt) {
    return a.pc.qtype == kQtE4m3 ? d(dt, std::integral_constant<int, kQtE4m3>{})
                                 : d(dt, std::integral_constant<int, kQtInt8>{});
  };
  if (a.pc.qtype == kQtE2m1 && !plan.prompt_waves) return launch_paged_attention4(a, stream);
  const hipError_t e = plan.prompt_waves ? launch_paged_prompt(a, plan.prompt_waves, stream)
                       : bf16            ? q(std::integral_constant<int, kDtBf16>{})
                                         : q(std::integral_constant<int, kDtF32>{});
  if (e != hipSuccess || a.n_split == 1) return e;
  if (bf16) return a.pc.d == 64 ? combine<kDtBf16, 64>(a, stream) : combine<kDtBf16, 128>(a, stream);
  return a.pc.d == 64 ? combine<kDtF32, 64>(a, stream) : combine<kDtF32, 128>(a, stream);
}

}  // namespace kv
