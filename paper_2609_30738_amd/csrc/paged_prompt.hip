// Attention of many tokens of a problem over its 8-bit paged cache (kv_paged_attention with bf16 queries and
// more columns, (token, query head) pairs of a kv head, than paged_attention.hip's kernel takes at once).
//
// paged_prompt_kernel: one workgroup of W waves per (32 W columns, split of the rows, kv head, problem), each
//   wave 32 columns.  Tiles of 64 rows go through LDS in bf16, which holds code * scale exactly (a scale is a
//   power of two), both as they lie; the next tile's codes are in flight meanwhile, and the one after's blocks.
//   With v_mfma_f32_32x32x16_bf16,
//     S^T = K Q^T,  O^T = V^T P^T:
//   a lane of the accumulator holds one column and 16 of 32 rows, so the column's sum stays in the lane, and its
//   weights are, eight at a time, its own operand of the second product; V's operand is read with the transposing
//   LDS loads, in the order of those rows.
//   The weights are 2^(t - reference) without a running maximum: the reference moves only where they grow past 1.
//   They are rounded to bf16 for the second product (2^-9 of each, the step of the bf16 output); their sum is taken of
//   the unrounded ones.  The exponentials of a half of the tile run beside the matrix products of the other.
//   The grid's fastest axis is the kv head: workgroups go to the 8 XCDs in turn, so that with 8 heads one L2
//   holds one head's rows.  The last columns, which see the most rows, come first.
//
//   Bound by the matrix units, 43 % busy, by the weights that they do not hide, and by the LDS beside them, whose
//   operands a wave reads for itself.  Three prompts of up to 4096 tokens over caches of up to 16384 rows (32 heads
//   over 8, d = 128): 1838 us, 1.06 PFLOP/s of the 1.58 that a large product reaches; 1135 us at d = 64, 1926 from
//   int8.  At an earlier step (1900 us) the same without staging took 1612, without the operands' reads 1685, without
//   both 1303, the products alone 785.
//   Measured and left: V transposed as it is staged 2020 (then 1900), both halves' logits before the weights 1890
//   (then 1842), masked and unmasked tiles as two copies of the code 2905 (then 2372), raised wave priority around the
//   products 2005 (then 1900), the staging spread over the second product 1908, 64 columns a wave (half the operand
//   reads, but one wave a SIMD with its sums in the accumulation registers) 4612.
//   W: 4 waves for up to 128 columns, 8 beyond: 64 columns 54 us with 4 and 57 with 8, 1024 columns 415 and 299.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "paged.h"
#include "paged_codes.h"
#include "paged_span.h"

namespace kv {

namespace {

constexpr int kTile = 64;            // rows of a tile
constexpr float kOctaves = 24.f;     // of the weights below 1 when a reference is taken
constexpr float kLowest = 0x1p126f;  // minus it: below every logit

typedef float __attribute__((ext_vector_type(16))) f32x16v;

__device__ __forceinline__ f32x16v mfma32(const u32x4_t& a, const u32x4_t& b, const f32x16v& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), c,
                                                 0, 0, 0);
}

__device__ __forceinline__ float half_max(float v) {  // over the lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A tile in LDS, rows as in the cache: K rows are D + 8 elements apart, so that the 16-byte reads of eight rows
// fall on all banks, V rows D + 32, so that the transposing reads of 64 bytes of four rows do.
template <int D> struct Tile {
  static constexpr int KS = D + 8, VS = D + 32;
  uint16_t k[kTile * KS];
  uint16_t v[kTile * VS];
  int32_t has[kTile / 16];  // whether the 16 rows have a block
  int32_t nan[8];           // whether a wave found a NaN in V
};
// Behind the two tiles: the split's blocks and their scales.
template <int W> struct Blocks {
  static constexpr int N = prompt_split_blocks(W);
  int32_t id[N];  // -1: missing
  float k_scale[N], v_scale[N];
};

typedef short __attribute__((ext_vector_type(4))) s16x4_t;

// Of the 4 x 16 elements whose row j the lanes 4 j .. 4 j + 3 of a group of 16 point into, four each: column l % 16.
__device__ __forceinline__ u32x2_t read_transposed(const uint16_t* p) {
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4_t*)p));
}

}  // namespace

template <int QT, int D, int W>
__global__ __launch_bounds__(64 * W, 2) void paged_prompt_kernel(PagedAttnArgs a, int n_groups) {
  constexpr int NS = D / 16;  // matrix steps over the head dimension
  constexpr int ND = D / 32;  // 32-wide tiles of the output
  using T = Tile<D>;
  extern __shared__ __align__(16) char lds[];
  T* const tiles = reinterpret_cast<T*>(lds);
  Blocks<W>& blocks = *reinterpret_cast<Blocks<W>*>(lds + 2 * sizeof(T));

  const int g = blockIdx.x, split = blockIdx.y % a.n_split, cg = n_groups - 1 - blockIdx.y / a.n_split;
  const int p = blockIdx.z, G = a.pc.h_q / a.pc.h_kv;
  const Span sp = span_of(a, p);
  const int col0 = cg * 32 * W;
  const int n_cols = min(sp.n_tok * G - col0, 32 * W);
  if (n_cols <= 0) return;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int shift = a.pc.shift, R = 1 << shift;
  const int r0 = split * a.split_rows;
  const int vis_max = sp.visible((col0 + n_cols - 1) / G), vis_min = sp.visible(col0 / G);
  const int r1 = min(vis_max, r0 + a.split_rows);
  if (r0 >= r1 && a.n_split > 1) return;
  const int n_tiles = r1 > r0 ? (r1 - r0 + kTile - 1) / kTile : 0;

  // this lane's column, and its wave's
  const int wcol = col0 + 32 * wave;
  const int wcols = min(n_cols - 32 * wave, 32);  // may be 0 or less
  const bool live = n < wcols;
  const int col = live ? wcol + n : col0;
  const int vis = live ? sp.visible(col / G) : 0;
  const int wvis_max = wcols > 0 ? sp.visible((wcol + wcols - 1) / G) : 0;
  const int wvis_min = wcols > 0 ? sp.visible(wcol / G) : 0;
  const int64_t row = (int64_t)(sp.tok0 + col / G) * a.pc.h_q + g * G + col % G;
  // a negative scale turns the queries' signs; a scale of 0 gives equal weights, as the least number does
  const float c = fmaxf(fabsf(a.c), 0x1p-126f);
  u32x4_t qf[NS];
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)(sp.tok0 + col / G) * a.q_stride +
                        (int64_t)(g * G + col % G) * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = *reinterpret_cast<const u32x4_t*>(q + 16 * s + 8 * h);
      if (a.c < 0.f) qf[s] ^= 0x80008000u;
    }
  }

  // Staging: a wave takes the rows of 1 KB of K and of V, 16 bytes a lane.  They lie in one 16-row group, so
  // block, scale and address are the wave's.  Blocks and scales come from LDS: scalar loads return out of order
  // with the reads of the products' operands, which then have to be waited for all at once (177 us of 1900).
  constexpr int ROWS = 1024 / D, NTASK = kTile / (ROWS * W) > 0 ? kTile / (ROWS * W) : 1;
  static_assert(ROWS <= 16, "a task lies in one block");
  const int wv = __builtin_amdgcn_readfirstlane(wave), lane_row = lane / (D / 16), lane_e = lane % (D / 16) * 16;
  int32_t id[NTASK];  // the block of the tile after the codes', and its scales
  float next_ks[NTASK], next_vs[NTASK];
  u32x4_t kc[NTASK], vc[NTASK];
  float ksc[NTASK], vsc[NTASK];
  bool has[NTASK];
  for (int i = tid; i << shift < r1 - r0; i += 64 * W) {
    int block = a.pc.table[(int64_t)p * a.pc.table_stride + (r0 >> shift) + i];
    if ((uint32_t)block >= (uint32_t)a.pc.n_blocks) block = -1;
    const int64_t unit = (int64_t)max(block, 0) * a.pc.h_kv + g;
    // The conversion takes a scale's exponent alone, and an infinity in V would reach columns that do not see it (as
    // 0 times it): a block with another scale than block_scale's, or of values that leave bf16, gives NaN logits,
    // which reach the columns that see it.
    const float ks = a.pc.k_scale[unit], vs = a.pc.v_scale[unit];
    const bool ok = is_bf16_scale<QT>(ks) && is_bf16_scale<QT>(vs);
    blocks.id[i] = block;
    blocks.k_scale[i] = ok ? ks : NAN;
    blocks.v_scale[i] = ok && block >= 0 ? vs : 1.f;
  }
  __syncthreads();
  auto task_row = [&](int i) { return (wv + i * W) * ROWS; };
  auto ids = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NTASK; ++i) {
      if (task_row(i) >= kTile) break;
      const int r = t * kTile + task_row(i);
      const int at = min(r, r1 - r0 - 1) >> shift;
      id[i] = blocks.id[at];
      next_ks[i] = blocks.k_scale[at];
      next_vs[i] = blocks.v_scale[at];
      if (r0 + r >= r1) id[i] = -1;
    }
  };
  auto codes = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NTASK; ++i) {
      if (task_row(i) >= kTile) break;
      const int block = __builtin_amdgcn_readfirstlane(id[i]);
      has[i] = block >= 0;
      const int64_t unit = (int64_t)max(block, 0) * a.pc.h_kv + g;
      const int64_t at = ((unit << shift) + ((r0 + t * kTile + task_row(i)) & (R - 1))) * D;
      kc[i] = *reinterpret_cast<const u32x4_t*>(a.pc.k + at + 16 * (uint32_t)lane);
      vc[i] = *reinterpret_cast<const u32x4_t*>(a.pc.v + at + 16 * (uint32_t)lane);
      ksc[i] = next_ks[i];
      vsc[i] = next_vs[i];
    }
  };
  auto put = [&](uint16_t* to, const u32x4_t& c, float scale) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const u32x2_t y = decode4_bf16<QT>(c[2 * w], scale), z = decode4_bf16<QT>(c[2 * w + 1], scale);
      *reinterpret_cast<u32x4_t*>(to + 8 * w) = u32x4_t{y[0], y[1], z[0], z[1]};
    }
  };
  auto stage = [&](int t) __attribute__((always_inline)) {
    T& x = tiles[t & 1];
    const int rb = r0 + t * kTile;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < NTASK; ++i) {
      if (task_row(i) >= kTile) break;
      const int r = task_row(i) + lane_row;
      if constexpr (QT == kQtInt8) {
        // (an int8 code takes a register once converted: not where it was loaded, a tile before)
        asm volatile("" : "+v"(kc[i][0]), "+v"(kc[i][1]), "+v"(kc[i][2]), "+v"(kc[i][3]));
        asm volatile("" : "+v"(vc[i][0]), "+v"(vc[i][1]), "+v"(vc[i][2]), "+v"(vc[i][3]));
      }
      // (a missing block's or a later row's K may be anything: its logits are masked)
      put(&x.k[r * T::KS + lane_e], kc[i], ksc[i]);
      if (!has[i] || rb + task_row(i) + ROWS > r1) {
        // a row that no column sees holds anything: zero its values, so that 0 times them is 0
        if (!has[i] || rb + r >= r1) vc[i] = u32x4_t{0u, 0u, 0u, 0u};
      }
      if (QT == kQtE4m3 && rb + kTile > vis_min) {
#pragma unroll
        for (int j = 0; j < 4; ++j) nan = nan || (((vc[i][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
      }
      put(&x.v[r * T::VS + lane_e], vc[i], vsc[i]);
      if (lane == 0 && task_row(i) % 16 == 0) x.has[task_row(i) / 16] = has[i];
    }
    if (QT == kQtE4m3 && rb + kTile > vis_min) {
      const uint64_t any = __ballot(nan);
      if (lane == 0) x.nan[wave] = any != 0;
    }
  };

  // Weights are 2^(t - mu), mu = reference + kOctaves: at most 1 until a logit exceeds the reference by more.  A
  // tile whose weights sum to more than 1 in some lane raises the reference to its largest logit (the first
  // tile does: it starts below every logit); no maximum is taken otherwise.
  float mu = -kLowest, sum = 0.f;
  f32x16v acc[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) acc[i] = 0.f;

  auto compute = [&](int t) __attribute__((always_inline)) {
    const T& x = tiles[t & 1];
    const int rb = r0 + t * kTile;
    // Operands are read from LDS NS products ahead: the order below is kept as it stands.
    auto k_frag = [&](int kt, int d) __attribute__((always_inline)) {
      return *reinterpret_cast<const u32x4_t*>(&x.k[(32 * kt + n) * T::KS + 16 * d + 8 * h]);
    };
    auto v_frag = [&](int q) __attribute__((always_inline)) {  // of product q = ND u + i
      const int u = q / ND, i = q % ND;
      // rows 16 u + 4 h + {0..3, 8..11} of element 32 i + n
      const uint16_t* p = &x.v[(16 * u + 4 * h + (lane & 15) / 4) * T::VS + 32 * i + (lane & 16) + 4 * (lane & 3)];
      const u32x2_t y = read_transposed(p), z = read_transposed(p + 8 * T::VS);
      return u32x4_t{y[0], y[1], z[0], z[1]};
    };
    f32x16v s[2];
    u32x4_t f[NS], pf[4];  // pf: weights of rows 16 u + 4 h + {0..3, 8..11}
    float part[4];
    // weights of the logits j, j + 1 of half kt
    auto weigh = [&](int kt, int j) __attribute__((always_inline)) {
      const int u = 2 * kt + (j >> 3);
      const float w0 = __builtin_amdgcn_exp2f(fmaf(s[kt][j], c, -mu)), w1 = __builtin_amdgcn_exp2f(fmaf(s[kt][j + 1], c, -mu));
      part[u] = j & 7 ? part[u] + w0 : w0;
      part[u] += w1;
      pf[u][(j & 7) >> 1] = pack_bf16(w0, w1);
    };
    // the half's weights join the sum; where they are too large they are taken again from a higher reference
    auto settle = [&](int kt) __attribute__((always_inline)) {
      if (__ballot(part[2 * kt] + part[2 * kt + 1] > 1.f)) {
        float tm = s[kt][0];
#pragma unroll
        for (int j = 1; j < 16; ++j) tm = fmaxf(tm, s[kt][j]);
        // a column whose logits are all -inf so far keeps the lowest reference
        const float top = fmaxf(half_max(tm) * c, -kLowest), mn = fmaxf(mu, top + kOctaves);
        const float r = __builtin_amdgcn_exp2f(mu - mn);
        mu = mn;
        sum *= r;
#pragma unroll
        for (int i = 0; i < ND; ++i) acc[i] *= r;
#pragma unroll
        for (int j = 0; j < 16; j += 2) weigh(kt, j);
      }
      sum += part[2 * kt] + part[2 * kt + 1];
    };
    const int has = __builtin_amdgcn_readfirstlane(x.has[0] & x.has[1] & x.has[2] & x.has[3]);
    const bool masked = rb + kTile > wvis_min || !has;
    auto mask = [&](int kt) __attribute__((always_inline)) {
      if (!masked) return;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int r = 32 * kt + 8 * (j >> 2) + 4 * h + (j & 3);
        if (rb + r >= vis || !x.has[2 * kt + (j >> 3)]) s[kt][j] = -INFINITY;
      }
    };
    bool nan_rows = false;
    if (QT == kQtE4m3 && rb + kTile > wvis_min) {
      int any = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) any |= x.nan[w];
      nan_rows = __builtin_amdgcn_readfirstlane(any) != 0;
    }
#pragma unroll
    for (int d = 0; d < NS; ++d) f[d] = k_frag(0, d);
    __builtin_amdgcn_sched_barrier(0);
    s[0] = 0.f;
#pragma unroll
    for (int d = 0; d < NS; ++d) {
      s[0] = mfma32(f[d], qf[d], s[0]);
      f[d] = k_frag(1, d);
      __builtin_amdgcn_sched_barrier(0);
    }
    mask(0);
    // the second half's products beside the first one's weights
    s[1] = 0.f;
#pragma unroll
    for (int d = 0; d < NS; ++d) {
      s[1] = mfma32(f[d], qf[d], s[1]);
      f[d] = v_frag(d);
#pragma unroll
      for (int j = 16 * d / NS; j < 16 * (d + 1) / NS; j += 2) weigh(0, j);
      __builtin_amdgcn_sched_barrier(0);
    }
    settle(0);
    mask(1);
    if (QT == kQtE4m3 && nan_rows) {
      // a NaN counts for the columns that see its row alone: it leaves the products, and the columns that
      // see one are marked by a product of indicators
#pragma unroll
      for (int j = 0; j < 16; j += 2) weigh(1, j);
      settle(1);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          u32x4_t vf = v_frag(ND * u + i), nf, seen;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            nf[w] = ((vf[w] & 0x7FFFu) > 0x7F80u ? 0x3F80u : 0u) | ((vf[w] & 0x7FFF0000u) > 0x7F800000u ? 0x3F800000u : 0u);
            vf[w] &= ((nf[w] & 0xFFFFu) ? 0u : 0xFFFFu) | ((nf[w] >> 16) ? 0u : 0xFFFF0000u);
            const int r = rb + 16 * u + 8 * (w >> 1) + 4 * h + 2 * (w & 1);
            seen[w] = (r < vis ? 0x3F80u : 0u) | (r + 1 < vis ? 0x3F800000u : 0u);
          }
          f32x16v hit;
          hit = 0.f;
          hit = mfma32(nf, seen, hit);
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (hit[j] > 0.f) acc[i][j] = NAN;
          acc[i] = mfma32(vf, pf[u], acc[i]);
        }
    } else {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < 4 * ND; ++q) {
        if (q == 2 * ND) settle(1);
        acc[q % ND] = mfma32(f[q % NS], pf[q / ND], acc[q % ND]);
        if (q + NS < 4 * ND) f[q % NS] = v_frag(q + NS);
        if (q < 2 * ND) {
#pragma unroll
          for (int j = 8 * q / ND; j < 8 * (q + 1) / ND; j += 2) weigh(1, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  if (n_tiles > 0) {
    ids(0);
    codes(0);
    if (n_tiles > 1) ids(1);
    stage(0);
    if (n_tiles > 1) codes(1);
    if (n_tiles > 2) ids(2);
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
      if (r0 + t * kTile < wvis_max) compute(t);
      if (t + 1 < n_tiles) {
        stage(t + 1);
        if (t + 2 < n_tiles) codes(t + 2);
        if (t + 3 < n_tiles) ids(t + 3);
      }
      __syncthreads();
    }
  }

  if (!live) return;
  sum = half_sum(sum);
  if (a.n_split == 1) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* out = static_cast<uint16_t*>(a.out) + row * D;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        u32x2_t y;
        y[0] = pack_bf16(acc[i][j] * inv, acc[i][j + 1] * inv);
        y[1] = pack_bf16(acc[i][j + 2] * inv, acc[i][j + 3] * inv);
        *reinterpret_cast<u32x2_t*>(out + 32 * i + 2 * j + 4 * h) = y;
      }
  } else {
    float* pt = a.part + (row * a.n_split + split) * (D + 2);
    if (h == 0) {
      pt[0] = mu > -kLowest ? mu : -INFINITY;
      pt[1] = sum;
    }
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int j = 0; j < 16; j += 2)
        *reinterpret_cast<float2*>(pt + 2 + 32 * i + 8 * (j >> 2) + 4 * h + (j & 3)) = make_float2(acc[i][j], acc[i][j + 1]);
  }
}

namespace {

template <int QT, int D, int W> hipError_t attend(const PagedAttnArgs& a, hipStream_t stream) {
  const int groups = (a.max_q * a.pc.group() + 32 * W - 1) / (32 * W);
  const dim3 grid((unsigned)a.pc.h_kv, (unsigned)(groups * a.n_split), (unsigned)a.pc.n_prob);
  constexpr int lds = 2 * (int)sizeof(Tile<D>) + (int)sizeof(Blocks<W>);
  auto kernel = paged_prompt_kernel<QT, D, W>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  kernel<<<grid, 64 * W, lds, stream>>>(a, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_prompt(const PagedAttnArgs& a, int waves, hipStream_t stream) {
  auto w = [&](auto qt, auto d) {
    return waves == 4 ? attend<qt.value, d.value, 4>(a, stream) : attend<qt.value, d.value, 8>(a, stream);
  };
  auto d = [&](auto qt) {
    return a.pc.d == 64 ? w(qt, std::integral_constant<int, 64>{}) : w(qt, std::integral_constant<int, 128>{});
  };
  return a.pc.qtype == kQtE4m3 ? d(std::integral_constant<int, kQtE4m3>{}) : d(std::integral_constant<int, kQtInt8>{});
}

}  // namespace kv
