// Attention of the last tokens of every problem over its 4-bit paged cache (kv_paged_attention on a cache of e2m1
// codes, up to 32 columns at a time; a column is a (token, query head) pair of the kv head).
//
// paged_attn4_kernel: columns, references and weights as in paged_attention.hip's kernel.
//     S^T = K Q^T,  O^T = V^T P^T  by v_mfma_f32_16x16x32_bf16.
//   Weights of bf16 queries: two bf16 terms for up to 16 columns (as close to 64 bits as fp32 weights), one for more, 2^-9 of
//   each.  Up to five tokens of 16 requests, root mean square over the output's: 0.00165 from 64 bits, of which 0.00159 is
//   the output's own rounding; with two terms 0.00159, and 28.7 us for 26.3.
//   Codes.  The scales belong to a row and 32 of its elements, so they go into the operands, where the conversion from four
//   bits applies them at no cost (a code times its scale is exact in bf16).  A lane's operand of K is a quarter of a row: at
//   d = 128 one 16-byte load and one scale.  For V a lane takes D / 16 elements of each of its rows, a word at d = 128, and
//   the scales of 16 rows in one load, a byte of which one turn brings to a float's exponent; pairs of rows are put together
//   by byte permutations once converted.  The weights' sum comes from a row of ones in the same products.
//   Shares.  Caches of more than a split's rows are one long axis of rounds of 128 rows, problem after problem, that every
//   unit's workgroups share equally, as many as the chip holds at once: unequal caches cost no idle CUs, and a workgroup
//   begins once.  The parts of problems that fall to several shares are joined by paged_join4_kernel.
//   Bound by the cache's reads: one token over 32 caches of up to 32768 rows (1.07 GB) 183 us, 5.8 TB/s, of which this kernel
//   takes 172 to 177 (at an earlier step, of 188 us, the loads alone took 175).
//   24 ragged ones of up to 24001 rows in blocks of 16 (0.41 GB, eight query heads to a kv head) 79 us, 5.1 TB/s (in splits of
//   2048 rows 86), this kernel 73: the scales of 16 rows are half a line; in blocks of 64 74 in all.  Up to five tokens of 16 requests of up to 6001
//   rows 26, in splits 34: latency of the rounds, and 5 for the join; over 32 caches of 100 rows 6.2, latency.
//   Measured and left: K's codes as they are against e4m3 terms of the queries by v_mfma_scale_f32_16x16x128 (the same for
//   long caches, 10 us more for five tokens: the queries have to be taken apart first), four tiles a step (the same), two
//   steps of loads ahead (179 and 25.8, and 1 us more for short calls), four waves a SIMD for up to 16 columns (200), three for
//   32 (their registers spill: 49 for five tokens), the next problem's lengths beside the merge (the same).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "paged.h"
#include "paged_codes.h"
#include "paged_shares.h"
#include "paged_span.h"

namespace kv {

namespace {

constexpr int kThreads = kAttnThreads;
constexpr int kWaves = kAttnWaves;

// Tiles of 16 rows in a wave's step, and the waves per SIMD that the registers are held to.
constexpr int kTiles4 = 2;
template <int DT, int D, int NT> constexpr int kMinWaves4 = (NT == 1 ? 3 : 2) - (DT == kDtF32 && D == 128 ? 1 : 0);

constexpr int kRound4 = kWaves * 16 * kTiles4;  // rows of a workgroup's round

typedef const __attribute__((address_space(4))) int32_t* uniform_ints;  // read by scalar loads

// The token of a column, column / group: by the group's reciprocal, exact below 2^28.
__device__ __forceinline__ int token_of(const PagedAttnArgs& a, int col) {
  return a.group_inv ? (int)__umulhi((uint32_t)col, a.group_inv) : col;
}

// Rounds of a problem's rows for the columns from col0 on (at least one if it has such columns).
__device__ __forceinline__ int rounds_of(const PagedAttnArgs& a, const Span& sp, int col0, int cols, int G) {
  const int n = min(sp.n_tok * G - col0, cols);
  return n <= 0 ? 0 : max(1, (int)((uint32_t)(sp.visible(token_of(a, col0 + n - 1)) + kRound4 - 1) / kRound4));
}

// Place of a share's part of a unit's column: slot 0 of a problem that begins before the share, 1 of one that ends behind it.
__device__ __forceinline__ int64_t part4_at(int unit, int share, int slot, int col, int cols, int shares) {
  return (((int64_t)unit * shares + share) * 2 + slot) * cols + col;
}

// store_out of four elements.
template <int DT> __device__ __forceinline__ void store_out4(void* out, int64_t at, const f32x4v& A, float S) {
  float o[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = S == 0.f ? 0.f : A[k] / S;
  if constexpr (DT == kDtBf16)
    *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(out) + at) = u32x2_t{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
  else
    *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(o[0], o[1], o[2], o[3]);
}

// A wave's view of 256 problems, four consecutive ones to a lane: what they see, their rounds, and the rounds before them.
struct Shares {
  Span sp[4];
  int rounds[4], before[4], total;
  __device__ __forceinline__ void of(const PagedAttnArgs& a, int q0, int col0, int cols, int G) {
    const int lane = threadIdx.x & 63;
    int sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int q = q0 + 4 * lane + k;
      sp[k] = span_of(a, min(q, a.pc.n_prob - 1));
      rounds[k] = q < a.pc.n_prob ? rounds_of(a, sp[k], col0, cols, G) : 0;
      sum += rounds[k];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(incl, o, 64);
      if (lane >= o) incl += u;
    }
    total = __builtin_amdgcn_readlane(incl, 63);
    int at = incl - sum;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      before[k] = at;
      at += rounds[k];
    }
  }
};

}  // namespace

template <int DT, int D, int NT, bool SHARES>
__global__ __launch_bounds__(kThreads, (kMinWaves4<DT, D, NT>)) void paged_attn4_kernel(PagedAttnArgs a) {
  constexpr int NS = D / 32;                       // matrix steps over the head dimension
  constexpr int NI = D / 16;                       // 16-wide tiles of the output, elements of V that a lane takes
  constexpr int KW = D / 32;                       // words of a key that a lane takes
  constexpr int RB = D / 2, NG = D / kGroup4;      // bytes and scales of a row
  constexpr int TS = kTiles4, STEP = 16 * TS;
  constexpr int QN = DT == kDtBf16 ? 1 : 3;        // bf16 terms of a query
  constexpr int PN = DT == kDtF32 ? 3 : (NT == 1 ? 2 : 1);  // bf16 terms of a weight
  constexpr int COLS = 16 * NT;
  constexpr int kStride = D + 4;                   // of a column in LDS: its lanes' writes fall on all banks
  __shared__ float sh_m[kWaves][16], sh_s[kWaves][16];
  extern __shared__ __align__(16) float sh_acc[];  // [kWaves][up to 16 columns][kStride]

  const int g = blockIdx.x, cg = blockIdx.y, G = a.group, col0 = cg * COLS;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int shift = a.pc.shift, R = 1 << shift;

  // the share: rounds `at` to `end` of all problems' one after the other, from problem p on, whose first one is `base`
  const int share = SHARES ? (int)blockIdx.z : 0;
  int p = SHARES ? 0 : (int)blockIdx.z, base = 0, at = 0, end = 1;
  Span sp;
  if constexpr (SHARES) {
    // every wave by itself
    Shares s;
    s.of(a, 0, col0, COLS, G);
    int T = s.total;
    for (int q = 256; q < a.pc.n_prob; q += 256) {
      s.of(a, q, col0, COLS, G);
      T += s.total;
    }
    const int S = share_of(T, a.shares);
    at = share_begin(T, S, share);
    end = share_end(T, S, at);
    const bool writes = share == 0 && g == 0 && wave == 0;  // the sums, for the join
    if (at >= end && !writes) return;
    int32_t* prefix = a.prefix + (int64_t)cg * (a.pc.n_prob + 1);
    if (a.pc.n_prob > 256) s.of(a, 0, col0, COLS, G);
    bool found = false;
    for (int q = 0, before = 0; q < a.pc.n_prob; q += 256) {
      if (q > 0) s.of(a, q, col0, COLS, G);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int mine = before + s.before[k];
        const uint64_t has = __ballot(at >= mine && at < mine + s.rounds[k]);
        if (has) {
          const int l = __ffsll((unsigned long long)has) - 1;
          p = q + 4 * l + k;
          base = __builtin_amdgcn_readlane(mine, l);
          sp.tok0 = __builtin_amdgcn_readlane(s.sp[k].tok0, l);
          sp.n_tok = __builtin_amdgcn_readlane(s.sp[k].n_tok, l);
          sp.len = __builtin_amdgcn_readlane(s.sp[k].len, l);
          sp.cap = s.sp[k].cap;
          found = true;
        }
        if (writes && q + 4 * lane + k < a.pc.n_prob) prefix[q + 4 * lane + k] = mine;
      }
      before += s.total;
      if (!writes && found) break;
    }
    if (writes && lane == 0) prefix[a.pc.n_prob] = T;
    if (at >= end) return;
    if (a.first && g == 0 && wave == 0 && lane == 0) a.first[(int64_t)cg * a.shares + share] = p;
  } else {
    sp = span_of(a, p);
  }

  for (;; sp = span_of(a, p)) {
    const int n_cols = min(sp.n_tok * G - col0, COLS);
    if (n_cols <= 0) {
      if (!SHARES || ++p >= a.pc.n_prob) return;
      continue;
    }
    const int vis_max = __builtin_amdgcn_readfirstlane(sp.visible(token_of(a, col0 + n_cols - 1)));
    const int vis_min = __builtin_amdgcn_readfirstlane(sp.visible(token_of(a, col0)));
    const int all = max(1, (int)((uint32_t)(vis_max + kRound4 - 1) / kRound4));  // the problem's rounds, and those of the share
    const int from = at - base, to = SHARES ? min(end - base, all) : all;
    const int r0 = from * kRound4, r1 = min(vis_max, to * kRound4);
    const bool whole = !SHARES || (from == 0 && to == all);
    at = base + to;
    base += all;

    // The codes and scales of a step's rows: row 16 t + 4 j + kg for V, and for K the row that holds the accumulator's row n;
    // their blocks, and where these lie.
    uint32_t xk[TS][KW], xv[TS][4], ksb[TS];
    u32x4_t vsb[TS];  // of 16 rows
    int blk[TS], next_blk[TS];
    int64_t codes_at[TS], scales_at[TS];
    const int k_row = 4 * (n & 3) + (n >> 2);
    // a wave-uniform address and a lane's 32-bit offset
    const uint32_t k_lane = k_row * RB + kg * (4 * KW), v_lane = kg * RB + n * (NI / 2);
    const uint32_t ks_lane = (kg * (8 * KW) / kGroup4) * R + k_row, vs_lane = (n * NI / kGroup4) * R;
    // the table entries of a step's rows are read a step before their codes
    int ahead[TS];
    const uniform_ints table = (uniform_ints)(uintptr_t)(a.pc.table + (int64_t)p * a.pc.table_stride);
    auto look = [&](int rb) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TS; ++t) ahead[t] = table[min(rb + 16 * t, (r1 - 1) & ~15) >> shift];
    };
    auto locate = [&](int rb) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TS; ++t) {
        const int r = min(rb + 16 * t, (r1 - 1) & ~15);
        next_blk[t] = (uint32_t)ahead[t] < (uint32_t)a.pc.n_blocks ? ahead[t] : -1;
        const int64_t unit = (int64_t)max(next_blk[t], 0) * a.pc.h_kv + g;
        codes_at[t] = (unit << shift) * RB + (r & (R - 1)) * RB;
        scales_at[t] = (unit << shift) * NG + (r & (R - 1));
      }
    };
    auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TS; ++t) {
        const uint8_t* ks = a.pc.k + codes_at[t];
        if constexpr (KW == 4) {
          const u32x4_t u = load_code<NT == 1>(reinterpret_cast<const u32x4_t*>(ks + k_lane));
#pragma unroll
          for (int i = 0; i < 4; ++i) xk[t][i] = u[i];
        } else {
          const u32x2_t u = load_code<NT == 1>(reinterpret_cast<const u32x2_t*>(ks + k_lane));
          xk[t][0] = u[0];
          xk[t][1] = u[1];
        }
        ksb[t] = (static_cast<const uint8_t*>(a.pc.k_scale) + scales_at[t])[ks_lane];
      }
    };
    auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TS; ++t) {
        const uint8_t* vs = a.pc.v + codes_at[t];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (NI == 8) xv[t][j] = load_code<NT == 1>(reinterpret_cast<const uint32_t*>(vs + (v_lane + 4 * j * RB)));
          else xv[t][j] = load_code<NT == 1>(reinterpret_cast<const uint16_t*>(vs + (v_lane + 4 * j * RB)));
        }
        vsb[t] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint8_t*>(a.pc.v_scale) + scales_at[t] + vs_lane);
      }
    };

    const int rb0 = r0 + wave * STEP;
    if (rb0 < r1) look(rb0);
    // a negative scale turns the queries' signs; a scale of 0 gives equal weights, as the least number does
    const float c = fmaxf(fabsf(a.c), 0x1p-126f);
    // the queries' operand: column n, elements D / 4 kg + 8 s .. + 7
    u32x4_t qf[NT][NS][QN];
    int vis[NT];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      const int col = col0 + 16 * ct + n;
      const bool live = 16 * ct + n < n_cols;
      const int j = live ? token_of(a, col) : 0, h = live ? col - j * G : 0;
      vis[ct] = live ? sp.visible(j) : 0;
      const int64_t at = (int64_t)(sp.tok0 + j) * a.q_stride + (int64_t)(g * G + h) * D;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int e = D / 4 * kg + 8 * s;
        if constexpr (DT == kDtBf16) {
          qf[ct][s][0] = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(a.q) + at + e);
          if (a.c < 0.f) qf[ct][s][0] ^= 0x80008000u;
        } else {
          const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at + e);
          const float4 x = src[0], y = src[1];
          float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
          if (a.c < 0.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = -f[i];
          }
          split_terms<QN>(f, qf[ct][s]);
        }
      }
    }

    if (rb0 < r1) {
      locate(rb0);
      load_k();
      load_v();
      if (rb0 + kRound4 < r1) look(rb0 + kRound4);
    }

    float m[NT], mu[NT];  // mu: m (0 before the first finite logit) and kSlack octaves
    f32x4v acc[NT][NI], sum[NT];
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      m[ct] = -INFINITY;
      mu[ct] = kSlack;
      sum[ct] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[ct][i] = f32x4v{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t v_turn = (8 * kg + 9) & 31;  // turns byte kg of a word to a float's exponent

    // A step's rows; the codes of the step at `next` (if any) load as this one's are used up.
    auto step = [&](int rb, int next) __attribute__((always_inline)) {
      int any = 0;
#pragma unroll
      for (int t = 0; t < TS; ++t) {
        blk[t] = next_blk[t];
        any |= blk[t];
      }
      // its rows are not all visible to every column, or a block is missing
      const bool masked = rb + STEP > vis_min || any < 0;
      f32x4v lg[NT][TS];
      // (codes are converted here, not where they were loaded a step before: registers)
#pragma unroll
      for (int t = 0; t < TS; ++t)
#pragma unroll
        for (int i = 0; i < KW; ++i) asm volatile("" : "+v"(xk[t][i]));
#pragma unroll
      for (int t = 0; t < TS; ++t) {
#pragma unroll
        for (int ct = 0; ct < NT; ++ct) lg[ct][t] = f32x4v{0.f, 0.f, 0.f, 0.f};
        const float ksc = __uint_as_float(ksb[t] << 23);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const u32x4_t kf = decode8_e2m1(xk[t][s], ksc);
#pragma unroll
          for (int q = QN - 1; q >= 0; --q)
#pragma unroll
            for (int ct = 0; ct < NT; ++ct) lg[ct][t] = mfma16(kf, qf[ct][s][q], lg[ct][t]);
        }
        if (masked) {
#pragma unroll
          for (int ct = 0; ct < NT; ++ct)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (blk[t] < 0 || rb + 16 * t + 4 * j + kg >= vis[ct]) lg[ct][t][j] = -INFINITY;
        }
      }
      if (next < r1) {
        locate(next);
        load_k();
        if (next + kRound4 < r1) look(next + kRound4);
      }
      float top[NT];
      bool over = false;
#pragma unroll
      for (int ct = 0; ct < NT; ++ct) {
        top[ct] = lg[ct][0][0];
#pragma unroll
        for (int e = 1; e < 4 * TS; ++e) top[ct] = fmaxf(top[ct], lg[ct][e >> 2][e & 3]);
        over = over || fmaf(top[ct], c, -m[ct]) > kSlack;
      }
      if (__ballot(over)) {
#pragma unroll
        for (int ct = 0; ct < NT; ++ct) {
          const float mn = fmaxf(m[ct], column_max(top[ct]) * c);
          const float f = m[ct] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[ct] - mn);
          m[ct] = mn;
          mu[ct] = mn == -INFINITY ? kSlack : mn + kSlack;
          sum[ct] *= f;
#pragma unroll
          for (int i = 0; i < NI; ++i) acc[ct][i] *= f;
        }
      }
#pragma unroll
      for (int u = 0; u < TS / 2; ++u) {  // two tiles at a time
        u32x4_t pf[NT][PN];
#pragma unroll
        for (int ct = 0; ct < NT; ++ct) {
          float w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(lg[ct][2 * u + (e >> 2)][e & 3], c, -mu[ct]));
          split_terms<PN>(w, pf[ct]);
          // their sum: as the products take them, with a row of ones
          const u32x4_t one = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
          for (int q = PN - 1; q >= 0; --q) sum[ct] = mfma16(one, pf[ct][q], sum[ct]);
        }
        float vsc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          asm volatile("" : "+v"(xv[2 * u + (e >> 2)][e & 3]));
          const uint32_t s = vsb[2 * u + (e >> 2)][e & 3];
          vsc[e] = __uint_as_float(__builtin_amdgcn_alignbit(s, s, v_turn));
        }
        if (masked) {
          // a row that a column does not see adds 0 times its values: these have to be finite
#pragma unroll
          for (int e = 0; e < 8; ++e) vsc[e] = fminf(fabsf(vsc[e]), 0x1p125f);
        }
        // V^T: pairs of elements of eight rows, put together as pairs of rows
        auto pair = [&](auto b) __attribute__((always_inline)) {
          constexpr int B = decltype(b)::value;
          uint32_t x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = decode2_e2m1<B>(xv[2 * u + (e >> 2)][e & 3], vsc[e]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            u32x4_t vf;
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], i ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int ct = 0; ct < NT; ++ct)
#pragma unroll
              for (int q = PN - 1; q >= 0; --q) acc[ct][2 * B + i] = mfma16(vf, pf[ct][q], acc[ct][2 * B + i]);
          }
        };
        pair(std::integral_constant<int, 0>{});
        pair(std::integral_constant<int, 1>{});
        if constexpr (NI == 8) {
          pair(std::integral_constant<int, 2>{});
          pair(std::integral_constant<int, 3>{});
        }
      }
      if (next < r1) load_v();
    };

    for (int rb = rb0; rb < r1; rb += kRound4) step(rb, rb + kRound4);  // the waves' steps in turn

    // merge of the waves, 16 columns at a time: element NI (4 kg + j) + i of column n
#pragma unroll
    for (int ct = 0; ct < NT; ++ct) {
      const int cols = min(n_cols - 16 * ct, 16);
      if (cols <= 0) break;
      if (kg == 0) {
        sh_m[wave][n] = m[ct];
        sh_s[wave][n] = sum[ct][0];
      }
      if (n < cols) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < NI; i += 4)
            *reinterpret_cast<float4*>(&sh_acc[(wave * cols + n) * kStride + (4 * kg + j) * NI + i]) =
                make_float4(acc[ct][i][j], acc[ct][i + 1][j], acc[ct][i + 2][j], acc[ct][i + 3][j]);
      }
      __syncthreads();
      for (int idx = tid; idx < cols * (D / 4); idx += kThreads) {
        const int cc = idx / (D / 4), e = idx % (D / 4) * 4;
        float M = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) M = fmaxf(M, sh_m[i][cc]);
        float S = 0.f;
        f32x4v A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          const float f = part_weight(sh_m[i][cc], M);
          S = fmaf(sh_s[i][cc], f, S);
          const f32x4v x = *reinterpret_cast<const f32x4v*>(&sh_acc[(i * cols + cc) * kStride + e]);
#pragma unroll
          for (int k = 0; k < 4; ++k) A[k] = fmaf(x[k], f, A[k]);
        }
        const int col = col0 + 16 * ct + cc;
        if (whole) {
          const int j = token_of(a, col);
          store_out4<DT>(a.out, ((int64_t)(sp.tok0 + j) * a.pc.h_q + g * G + (col - j * G)) * D + e, A, S);
        } else {
          float* pt = a.part + part4_at(cg * a.pc.h_kv + g, share, from > 0 ? 0 : 1, 16 * ct + cc, min(a.max_q * G, COLS), a.shares) * (D + 2);
          if (e == 0) *reinterpret_cast<float2*>(pt) = make_float2(M, S);
          *reinterpret_cast<float2*>(pt + 2 + e) = make_float2(A[0], A[1]);
          *reinterpret_cast<float2*>(pt + 4 + e) = make_float2(A[2], A[3]);
        }
      }
      if (ct + 1 < NT || SHARES) __syncthreads();
    }
    if (!SHARES || at >= end || ++p >= a.pc.n_prob) return;
  }
}

// One workgroup per (column, kv head, problem): the parts of the shares that the problem's rounds fall to, the waves' in
// turn, kJoin at a time in flight.  BY_SHARE: per (column, kv head, share but the first), for the problem that it begins in
// the middle of, where no earlier one does.
template <int DT, int D, bool BY_SHARE>
__global__ __launch_bounds__(kThreads) void paged_join4_kernel(PagedAttnArgs a, int COLS) {
  constexpr int E = D / 64, kJoin = 4;
  __shared__ float sh_a[kWaves][D], sh_m[kWaves], sh_s[kWaves];
  const int col = blockIdx.x, g = blockIdx.y, G = a.group, cg = (int)((uint32_t)col / (uint32_t)COLS);
  const int32_t* prefix = a.prefix + (int64_t)cg * (a.pc.n_prob + 1);
  const int T = prefix[a.pc.n_prob], share = (int)blockIdx.z + 1;
  int p = BY_SHARE ? a.first[(int64_t)cg * a.shares + share] : (int)blockIdx.z;
  const uint32_t S = share_of(T, a.shares);
  if (BY_SHARE && (uint32_t)share * S >= (uint32_t)T) return;  // no such share: its problem was not written
  const int lo = prefix[p], hi = prefix[p + 1];
  const Span sp = span_of(a, p);
  if (col >= sp.n_tok * G) return;
  if (BY_SHARE && ((uint32_t)share * S <= (uint32_t)lo || (uint32_t)(share - 1) * S > (uint32_t)lo)) return;
  const int s0 = (int)((uint32_t)lo / S), n = (int)((uint32_t)(hi - 1) / S) - s0 + 1;
  if (n == 1) return;  // one share had them all
  const int j = token_of(a, col);
  const int64_t row = (int64_t)(sp.tok0 + j) * a.pc.h_q + g * G + (col - j * G);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, cols = min(a.max_q * G, COLS);
  float m = -INFINITY, sum = 0.f, A[E];
#pragma unroll
  for (int e = 0; e < E; ++e) A[e] = 0.f;
  for (int i = wave; i < n; i += kJoin * kWaves) {
    float xm[kJoin], xs[kJoin], xa[kJoin][E];
#pragma unroll
    for (int j = 0; j < kJoin; ++j) {
      const bool in = i + j * kWaves < n;
      const int s = s0 + (in ? i + j * kWaves : i);
      const float* x = a.part + part4_at(cg * a.pc.h_kv + g, s, (uint32_t)s * S > (uint32_t)lo ? 0 : 1, col - cg * COLS, cols, a.shares) * (D + 2);
      xm[j] = in ? x[0] : -INFINITY;
      xs[j] = in ? x[1] : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) xa[j][e] = in ? x[2 + E * lane + e] : 0.f;
    }
    float mn = m;
#pragma unroll
    for (int j = 0; j < kJoin; ++j) mn = fmaxf(mn, xm[j]);
    const float f = part_weight(m, mn);
    sum *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) A[e] *= f;
#pragma unroll
    for (int j = 0; j < kJoin; ++j) {
      const float w = part_weight(xm[j], mn);
      sum = fmaf(xs[j], w, sum);
#pragma unroll
      for (int e = 0; e < E; ++e) A[e] = fmaf(xa[j][e], w, A[e]);
    }
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) sh_a[wave][E * lane + e] = A[e];
  if (lane == 0) {
    sh_m[wave] = m;
    sh_s[wave] = sum;
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

int tiles_of(int64_t cols) { return cols <= 16 ? 1 : 2; }

template <int DT, int D, int NT> hipError_t attend(PagedAttnArgs a, hipStream_t stream) {
  const int64_t cols = (int64_t)a.max_q * a.group;
  const unsigned h_kv = (unsigned)a.pc.h_kv, groups = (unsigned)((cols + 16 * NT - 1) / (16 * NT));
  const size_t lds = (size_t)kWaves * std::min<int64_t>(cols, 16) * (D + 4) * sizeof(float);
  if (a.shares == 0) {
    paged_attn4_kernel<DT, D, NT, false><<<dim3(h_kv, groups, (unsigned)a.pc.n_prob), kThreads, lds, stream>>>(a);
    return hipGetLastError();
  }
  // The join by the fewer of problems and shares, since most of its workgroups only end: one token over 2048 caches of 100 rows
  // (a bound of 4096) 126 us, by problems 169, four tokens 166 and 347; 100 caches of 1000 rows the same, four tokens over 64 39.8
  // by as many shares, by problems 36.9.
  const bool by_share = a.pc.n_prob > a.shares;
  a.first = by_share ? a.prefix + (int64_t)groups * (a.pc.n_prob + 1) : nullptr;
  paged_attn4_kernel<DT, D, NT, true><<<dim3(h_kv, groups, (unsigned)a.shares), kThreads, lds, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.shares == 1) return e;
  if (by_share)
    paged_join4_kernel<DT, D, true><<<dim3((unsigned)cols, h_kv, (unsigned)(a.shares - 1)), kThreads, 0, stream>>>(a, 16 * NT);
  else
    paged_join4_kernel<DT, D, false><<<dim3((unsigned)cols, h_kv, (unsigned)a.pc.n_prob), kThreads, 0, stream>>>(a, 16 * NT);
  return hipGetLastError();
}
template <int DT, int D> hipError_t attend(const PagedAttnArgs& a, hipStream_t stream) {
  return tiles_of((int64_t)a.max_q * a.pc.group()) == 1 ? attend<DT, D, 1>(a, stream) : attend<DT, D, 2>(a, stream);
}

}  // namespace

// Shares of a unit, a (kv head, group of columns): the fewest that take the least time in rounds of the workgroups that the
// chip holds at once.  The more columns the bound max_q admits, the fewer each group gets (fp32 turns: with 8 heads one from
// 32 groups on), though requests of a token all fall to the first: 60 of them over 32768 rows beside a turn of 64 (256) fp32
// tokens take 7.5 ms (29.7), by themselves 0.47; over 8 bits, where every problem has workgroups, 5.3 (6.3).
int paged4_shares(const Paged& pc, int max_q) {
  const int64_t cols = (int64_t)max_q * pc.group();
  const int nt = tiles_of(cols);
  const int64_t units = pc.h_kv * ((cols + 16 * nt - 1) / (16 * nt));
  const int64_t held = 256 * ((nt == 1 ? 3 : 2) - (pc.dtype == kDtF32 && pc.d == 128 ? 1 : 0));
  const int64_t most = std::max<int64_t>(1, held / units) + 8;
  int64_t best = 1;
  auto rounds = [&](int64_t n) { return (units * n + held - 1) / held; };
  for (int64_t n = 2; n <= most; ++n)
    if (rounds(n) * best < rounds(best) * n) best = n;
  return (int)best;
}

size_t paged4_prefix_bytes(const Paged& pc, int max_q, int shares) {
  const int64_t cols = (int64_t)max_q * pc.group(), nt = tiles_of(cols);
  return (size_t)(((cols + 16 * nt - 1) / (16 * nt) * (pc.n_prob + 1 + shares) * (int64_t)sizeof(int32_t) + 255) / 256 * 256);
}

size_t paged4_ws_bytes(const Paged& pc, int max_q, int shares) {
  const int64_t cols = (int64_t)max_q * pc.group(), nt = tiles_of(cols), groups = (cols + 16 * nt - 1) / (16 * nt);
  const int64_t parts = groups * pc.h_kv * shares * 2 * std::min<int64_t>(cols, 16 * nt);
  return paged4_prefix_bytes(pc, max_q, shares) + (size_t)(parts * (pc.d + 2)) * sizeof(float);
}

hipError_t launch_paged_attention4(PagedAttnArgs a, hipStream_t stream) {
  a.group = a.pc.group();
  a.group_inv = a.group > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group) : 0u;
  if (a.pc.dtype == kDtBf16) return a.pc.d == 64 ? attend<kDtBf16, 64>(a, stream) : attend<kDtBf16, 128>(a, stream);
  return a.pc.d == 64 ? attend<kDtF32, 64>(a, stream) : attend<kDtF32, 128>(a, stream);
}

}  // namespace kv
