// C ABI of the eviction path: host-side validation, workspace sizing and dispatch to the gfx950
// kernels.  Nothing here allocates device memory, keeps state between calls or launches anything
// before every argument has been checked.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "kernels.h"
#include "kvevict.h"
#include "paged.h"

namespace {

constexpr int kMaxLen = 1 << 24;
constexpr int kMaxGrid = 65535;
constexpr int kMaxCompactBudget = 8192;
constexpr float kLog2eF = 1.4426950408889634f;  // log2(e): kernels take logits in base 2
constexpr int kMaxPool = 63;  // widest max-pool window of kv_mmr_select_ex
constexpr size_t kWsAlign = 256;
constexpr int64_t kMaxTokenStride = (int64_t)1 << 26;
constexpr int kMaxRotated = 1 << 25;  // tokens of a rotation: its launch stays below 2^32 threads

size_t align_up(size_t x) { return (x + kWsAlign - 1) & ~(kWsAlign - 1); }

int elem_bytes(int dtype) { return dtype == KV_BF16 ? 2 : 4; }

bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

// Checks shared by every entry point; fills the launch shape.
int check_problem(const kv_problem* pr, kv::Shape* s) {
  if (!pr) return KV_ERR_NULL;
  if (pr->dtype != KV_F32 && pr->dtype != KV_BF16) return KV_ERR_DTYPE;
  if (pr->n_prob < 1 || pr->n_prob > kMaxGrid) return KV_ERR_ARG;
  if (!pr->len_host || !pr->tok_off_host || !pr->len_dev || !pr->tok_off_dev) return KV_ERR_NULL;
  if (pr->h_kv < 1 || pr->h_q < pr->h_kv || pr->h_q % pr->h_kv != 0 || pr->h_kv > kMaxGrid)
    return KV_ERR_SHAPE;
  if (pr->d != 64 && pr->d != 128) return KV_ERR_SHAPE;
  if (pr->w < 2) return KV_ERR_SHAPE;
  const int64_t rows = (int64_t)(pr->h_q / pr->h_kv) * pr->w;
  if (rows > 128) return KV_ERR_SHAPE;
  if (pr->w != 32 && rows > 64) return KV_ERR_SHAPE;
  int max_len = 0;
  for (int p = 0; p < pr->n_prob; ++p) {
    const int L = pr->len_host[p];
    if (L < pr->w + 1 || L > kMaxLen) return KV_ERR_SHAPE;
    if (pr->tok_off_host[p] < 0) return KV_ERR_SHAPE;
    if (L > max_len) max_len = L;
  }
  s->dtype = pr->dtype == KV_BF16 ? kv::kDtBf16 : kv::kDtF32;
  s->n_prob = pr->n_prob;
  s->h_q = pr->h_q;
  s->h_kv = pr->h_kv;
  s->d = pr->d;
  s->w = pr->w;
  s->max_len = max_len;
  s->lens = pr->len_dev;
  s->tok_off = pr->tok_off_dev;
  if (s->max_chunks() > kMaxGrid) return KV_ERR_SHAPE;
  return KV_OK;
}

// The uniform budget (per_problem = false), or the row stride of per-problem budgets, which may
// exceed a short problem's candidates (its own B_p is checked by check_budgets).
int check_budget(const kv_problem* pr, int32_t budget, int32_t keep_tail, bool per_problem = false) {
  if (budget < 1) return KV_ERR_BUDGET;
  for (int p = 0; p < pr->n_prob; ++p) {
    const int L = pr->len_host[p];
    if (keep_tail < 0 || keep_tail > L - 1) return KV_ERR_ARG;
    if (!per_problem && budget > L - keep_tail) return KV_ERR_BUDGET;
  }
  return KV_OK;
}

// Per-problem budgets (both arrays or neither): every B_p in [1, budget] and <= L_p - keep_tail.
int check_budgets(const kv_problem* pr, int32_t budget, int32_t keep_tail, const int32_t* b_host,
                  const int32_t* b_dev) {
  if (!b_host && !b_dev) return KV_OK;
  if (!b_host || !b_dev) return KV_ERR_NULL;
  for (int p = 0; p < pr->n_prob; ++p) {
    const int32_t b = b_host[p];
    if (b < 1 || b > budget || b > pr->len_host[p] - keep_tail) return KV_ERR_BUDGET;
  }
  return KV_OK;
}

// Largest candidate count of the batch (budget of problem p: b_host[p], or `budget`).
int max_candidates(const kv_problem* pr, int32_t budget, int32_t cand_mult, int32_t keep_tail,
                   const int32_t* b_host = nullptr) {
  int m = 0;
  for (int p = 0; p < pr->n_prob; ++p) {
    const int n_cand = pr->len_host[p] - keep_tail;
    const int64_t b = b_host ? b_host[p] : budget;
    const int64_t c = cand_mult > 0 ? std::min<int64_t>((int64_t)cand_mult * b, n_cand) : n_cand;
    if (c > m) m = (int)c;
  }
  return m;
}

int launch_status(hipError_t e) { return e == hipSuccess ? KV_OK : KV_ERR_LAUNCH; }

// Polls a workgroup of the one-launch window path makes for its unit's other segments before it
// computes their partials itself: the default, or KVEVICT_SPIN_LIMIT (0 takes that path at once).
uint32_t spin_limit() {
  const char* e = std::getenv("KVEVICT_SPIN_LIMIT");
  if (e && *e) {
    char* end = nullptr;
    const unsigned long v = std::strtoul(e, &end, 10);
    if (end && *end == '\0') return (uint32_t)std::min<unsigned long>(v, 1ul << 30);
  }
  return kv::kDefaultSpinLimit;
}

// Segment plan of the streaming window kernels for this batch.
kv::StreamPlan stream_plan_of(const kv_problem* pr, const kv::Shape& s) {
  return kv::stream_plan(s, pr->len_host);
}

// The plan of the candidate kernel (max_cand: the largest C_p).  Its second pass revisits the tiles
// that can hold a candidate, few where tiles far outnumber candidates: then a unit is read little
// more than once, and whole units pay even where they leave CUs idle (128 units of 30000 keys with
// salient ones: 414 us as two workgroups each through base scores, 305 whole).  Where every second tile
// can hold a candidate they do not (112 units of 8000 keys, C = 256: 190 and 226 us), nor where no key
// stands out at all (128 units of 30000 keys of noise alone: 437 and 700 us), which the sizes
// do not tell.
kv::StreamPlan cand_plan_of(const kv_problem* pr, const kv::Shape& s, int max_cand) {
  return kv::stream_plan(s, pr->len_host,
                         s.max_len / 32 >= 2 * max_cand ? kv::WgRule::kWhole : kv::WgRule::kEven);
}

// Workspace of the window entry points: the larger of the chunked and the streaming layouts.  Units of
// one segment use no partials; at w = 32 they have always been counted.
size_t window_ws_bytes(const kv_problem* pr, const kv::Shape& s) {
  size_t b = kv::window_stats_ws_bytes(s);
  if (kv::stream_shape_ok(s, 1.f)) {
    const kv::StreamPlan plan = stream_plan_of(pr, s);
    if (s.w == 32 || plan.max_segs > 1) b = std::max(b, kv::stream_ws_bytes(s, plan));
  }
  return align_up(b);
}

// Token rows that per-token arrays of the batch span (mu, sigma and the scores per kv head):
// max_p tok_off[p] + L_p, which is sum_p L_p for packed offsets.  Arrays in the workspace are
// sized by it, so offsets with gaps cannot reach past them.
int64_t token_extent(const kv_problem* pr) {
  int64_t t = 0;
  for (int p = 0; p < pr->n_prob; ++p) t = std::max<int64_t>(t, pr->tok_off_host[p] + pr->len_host[p]);
  return t;
}

// Whether kv_window_base_scores forms the scores inside the window kernel's second pass (bf16
// streaming shapes with every unit in one workgroup), or from mu / sigma in the workspace.
bool scores_in_window_pass(const kv_problem* pr, const kv::Shape& s, float scale) {
  return kv::stream_shape_ok(s, scale) && stream_plan_of(pr, s).one_wg();
}

// Workspace of kv_window_base_scores with this scale: none where the window kernel's second pass forms
// the scores of whole units; the chunked kernels (every shape with scale <= 0 among them) form them in
// their second pass too and need the window paths' part; else that part and rows of mu and sigma.
size_t base_scores_ws_bytes(const kv_problem* pr, const kv::Shape& s, float scale) {
  if (!kv::stream_shape_ok(s, scale)) return window_ws_bytes(pr, s);
  if (stream_plan_of(pr, s).one_wg()) return 0;
  const size_t keys = (size_t)token_extent(pr) * pr->h_kv;
  return window_ws_bytes(pr, s) + 2 * align_up(keys * sizeof(float));
}

// Batches of w = 32 whose units are one segment each: their queries answer for scale > 0 only, the
// others for every scale.
bool one_segment_units(const kv_problem* pr, const kv::Shape& s) {
  return s.w == 32 && kv::stream_shape_ok(s, 1.f) && stream_plan_of(pr, s).max_segs == 1;
}

// Candidate lists of kv_window_candidates: one list of `stride` 8-byte entries per (problem, kv
// head).
size_t cand_lists_bytes(const kv_problem* pr, int stride) {
  return align_up((size_t)pr->n_prob * pr->h_kv * stride * sizeof(uint64_t));
}

// Whether kv_window_candidates forms the candidate lists inside the window kernel: w = 32, every
// unit of a streaming shape in one workgroup, units of at most kCandMaxLen keys, cand_mult > 0 (the caller has
// checked the candidate count against the selection's limit).
bool cands_in_window_pass(const kv_problem* pr, const kv::Shape& s, float scale, int32_t cand_mult,
                          int max_cand) {
  return s.w == 32 && kv::stream_shape_ok(s, scale) && cand_plan_of(pr, s, max_cand).one_wg() &&
         cand_mult > 0 && s.max_len <= kv::kCandMaxLen;
}

// Workspace of kv_window_candidates: the lists and the units' normalisers, then with the fused
// path the tile codes of its first pass, without it the scores and what kv_window_base_scores needs
// after them.
size_t cand_ws_bytes(const kv_problem* pr, const kv::Shape& s, int stride, float scale, bool fused) {
  const size_t head = cand_lists_bytes(pr, stride) + align_up((size_t)pr->n_prob * pr->h_kv * sizeof(float));
  if (fused)
    return head + align_up((size_t)pr->n_prob * pr->h_kv * kv::cand_code_stride(s) * sizeof(uint32_t));
  return head + align_up((size_t)token_extent(pr) * pr->h_kv * sizeof(float)) +
         base_scores_ws_bytes(pr, s, scale);
}

// Selection, and with k_out / v_out the compaction of the selected rows, in one launch; base
// scores from mu / sigma, or given (score).
// Where the selection's base scores come from: mu / sigma (with lambda1), given scores, or the
// candidate lists of kv_window_candidates; with cut_out the lists are written (and without sel_idx
// only the candidate cut runs).
struct ScoreSource {
  const float* mu = nullptr;
  const float* sigma = nullptr;
  const float* lambda1 = nullptr;
  const float* score = nullptr;
  const uint64_t* cand_in = nullptr;
  const float* cand_in_max = nullptr;
  uint64_t* cut_out = nullptr;
  float* cut_max = nullptr;
  int list_stride = 0;
};

int mmr_select_impl(const kv_problem* pr, const ScoreSource& src, const void* k, const void* v,
                    const float* lambda2, int32_t budget,
                    int32_t cand_mult, int32_t keep_tail, const kv_select_opts* opts,
                    int32_t* sel_idx, float* sel_score, int32_t* cand_idx, float* cand_corr,
                    void* k_out, void* v_out, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!src.score && !src.cand_in && (!src.mu || !src.sigma || !src.lambda1)) return KV_ERR_NULL;
  if (!k || (!src.cut_out && (!lambda2 || !sel_idx))) return KV_ERR_NULL;
  if (!aligned16(k)) return KV_ERR_ARG;
  if (k_out && (!aligned16(v) || !aligned16(k_out) || !aligned16(v_out))) return KV_ERR_ARG;
  // the kernels form cand_mult * B_p in 32-bit arithmetic (B_p <= budget)
  if (cand_mult < 0 || (int64_t)cand_mult * budget > INT32_MAX) return KV_ERR_ARG;
  const int32_t pool = opts ? opts->pool : 1;
  const float w_mu = opts ? opts->w_mu : 1.f;
  const int32_t* b_host = opts ? opts->budget_host : nullptr;
  const int32_t* b_dev = opts ? opts->budget_dev : nullptr;
  if (pool < 1 || pool > kMaxPool || pool % 2 == 0 || !std::isfinite(w_mu)) return KV_ERR_ARG;
  st = check_budget(pr, budget, keep_tail, b_host != nullptr || b_dev != nullptr);
  if (st != KV_OK) return st;
  st = check_budgets(pr, budget, keep_tail, b_host, b_dev);
  if (st != KV_OK) return st;
  if (k_out && budget > kMaxCompactBudget) return KV_ERR_BUDGET;
  const int max_cand = max_candidates(pr, budget, cand_mult, keep_tail, b_host);
  if (max_cand > kv::select_max_candidates(pr->d, elem_bytes(pr->dtype))) return KV_ERR_SHAPE;
  if ((src.cand_in || src.cut_out) && pool != 1) return KV_ERR_ARG;  // lists hold unpooled scores
  kv::SelectArgs a;
  a.mu = src.mu;
  a.sigma = src.sigma;
  a.score = src.score;
  a.cand_in = src.cand_in;
  a.cand_in_max = src.cand_in_max;
  a.cut_out = src.cut_out;
  a.cut_max = src.cut_max;
  a.list_stride = src.list_stride;
  a.k = k;
  a.lambda1 = src.lambda1;
  a.lambda2 = lambda2;
  a.pool = pool;
  a.w_mu = w_mu;
  a.budget = budget;
  a.budgets = b_dev;
  a.cand_mult = cand_mult;
  a.keep_tail = keep_tail;
  a.cand_stride = kv_candidate_stride(pr, budget, cand_mult, keep_tail);
  a.max_cand = max_cand;
  a.max_cand_all = max_candidates(pr, budget, 0, keep_tail);
  a.sel_idx = sel_idx;
  a.sel_score = sel_score;
  a.cand_idx = cand_idx;
  a.cand_corr = cand_corr;
  a.v = v;
  a.k_out = k_out;
  a.v_out = v_out;
  a.out_rows = budget + keep_tail;
  if ((cand_idx || cand_corr) && a.cand_stride < 1) return KV_ERR_ARG;
  return launch_status(kv::launch_mmr_select(s, a, static_cast<hipStream_t>(stream)));
}

// kv_window_candidates; with sel (the caller has checked the selection's arguments and, where the
// window kernel cuts the candidates, that every C_p <= kCandSelectMax) the selection of each unit
// follows its cut in the same launch.
int window_candidates_impl(const kv_problem* pr, const void* q_win, const void* k, float scale,
                           const float* lambda1, int32_t sigma_rows, int32_t budget,
                           int32_t cand_mult, int32_t keep_tail, const kv_select_opts* opts,
                           float* row_max, float* row_sum, void* ws, size_t ws_bytes,
                           const kv::CandSelect* sel, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!q_win || !k || !lambda1 || !row_max || !row_sum) return KV_ERR_NULL;
  if (!aligned16(q_win) || !aligned16(k)) return KV_ERR_ARG;
  if (!std::isfinite(scale)) return KV_ERR_ARG;
  if (sigma_rows != KV_SIGMA_GROUP_MEAN && sigma_rows != KV_SIGMA_ALL_ROWS) return KV_ERR_ARG;
  if (cand_mult < 0 || (int64_t)cand_mult * budget > INT32_MAX) return KV_ERR_ARG;
  const int32_t pool = opts ? opts->pool : 1;
  const float w_mu = opts ? opts->w_mu : 1.f;
  const int32_t* b_host = opts ? opts->budget_host : nullptr;
  const int32_t* b_dev = opts ? opts->budget_dev : nullptr;
  if (pool != 1 || !std::isfinite(w_mu)) return KV_ERR_ARG;
  st = check_budget(pr, budget, keep_tail, b_host != nullptr || b_dev != nullptr);
  if (st != KV_OK) return st;
  st = check_budgets(pr, budget, keep_tail, b_host, b_dev);
  if (st != KV_OK) return st;
  const int stride = max_candidates(pr, budget, cand_mult, keep_tail, b_host);
  if (stride > kv::select_max_candidates(pr->d, elem_bytes(pr->dtype))) return KV_ERR_SHAPE;
  const bool fused = cands_in_window_pass(pr, s, scale, cand_mult, stride);
  const size_t need = cand_ws_bytes(pr, s, stride, scale, fused);
  if (ws_bytes < need || !ws || (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)))
    return KV_ERR_WORKSPACE;
  const bool all = sigma_rows == KV_SIGMA_ALL_ROWS;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  char* base = static_cast<char*>(ws);
  const size_t n_units = (size_t)pr->n_prob * pr->h_kv;
  uint64_t* lists = reinterpret_cast<uint64_t*>(base);
  float* cmax = reinterpret_cast<float*>(base + cand_lists_bytes(pr, stride));
  const size_t head = cand_lists_bytes(pr, stride) + align_up(n_units * sizeof(float));
  if (fused)
    return launch_status(kv::launch_stream_window_cands(
        s, cand_plan_of(pr, s, stride), q_win, k, scale, lambda1, w_mu, budget, b_dev, cand_mult,
        keep_tail, row_max, row_sum, lists, cmax, stride, reinterpret_cast<uint32_t*>(base + head),
        all, sel, hs));
  // the scores into the workspace, then the candidate cut of the selection kernel, with sel followed
  // by the greedy and the compaction in the same workgroup (one launch less, and the candidates
  // need not come back from memory)
  float* score = reinterpret_cast<float*>(base + head);
  const size_t score_bytes = align_up((size_t)token_extent(pr) * pr->h_kv * sizeof(float));
  char* rest = base + head + score_bytes;  // kv_window_base_scores' workspace: window part, mu, sigma
  const kv::StreamPlan plan =
      kv::stream_shape_ok(s, scale) ? kv::stream_plan(s, pr->len_host, kv::WgRule::kAny) : kv::StreamPlan{};
  const size_t win = window_ws_bytes(pr, s);
  if (kv::stream_shape_ok(s, scale) && s.w == 32 && cand_mult > 0 && kv::prune_segs_ok(plan, stride) &&
      win + kv::prune_segs_bytes(s) <= base_scores_ws_bytes(pr, s, scale)) {
    // only the scores that can reach the cut (the codes take the place of mu and sigma)
    st = launch_status(kv::launch_prune_segs(s, plan, q_win, k, scale, lambda1, w_mu, budget, b_dev, cand_mult,
                                             keep_tail, rest, rest + win, row_max, row_sum, score, all, hs));
  } else {
    st = kv_window_base_scores(pr, q_win, k, scale, lambda1, w_mu, sigma_rows, row_max, row_sum, score, rest,
                               ws_bytes - head - score_bytes, stream);
  }
  if (st != KV_OK) return st;
  ScoreSource src;
  src.score = score;
  src.cut_out = lists;
  src.cut_max = cmax;
  src.list_stride = stride;
  if (sel)
    return mmr_select_impl(pr, src, k, sel->v, sel->lambda2, budget, cand_mult, keep_tail, opts,
                           sel->sel_idx, sel->sel_score, nullptr, nullptr, sel->k_out, sel->v_out,
                           stream);
  return mmr_select_impl(pr, src, k, nullptr, nullptr, budget, cand_mult, keep_tail, opts, nullptr,
                         nullptr, nullptr, nullptr, nullptr, nullptr, stream);
}

}  // namespace

extern "C" {

const char* kv_strerror(int status) {
  switch (status) {
    case KV_OK: return "success";
    case KV_ERR_NULL: return "a required pointer is NULL";
    case KV_ERR_SHAPE: return "unsupported head layout, window, length or candidate count";
    case KV_ERR_DTYPE: return "unsupported dtype";
    case KV_ERR_BUDGET: return "budget outside [1, L - keep_tail]";
    case KV_ERR_WORKSPACE: return "workspace too small or misaligned";
    case KV_ERR_LAUNCH: return "HIP launch failed";
    case KV_ERR_ARG: return "invalid argument";
    case KV_ERR_SCRATCH: return "batch needs more scratch than KV_NOALLOC_SCRATCH_BYTES";
    default: return "unknown status";
  }
}

int kv_version(void) { return 1; }

size_t kv_workspace_bytes(const kv_problem* pr, int32_t budget, int32_t cand_mult,
                          int32_t keep_tail) {
  kv::Shape s;
  if (check_problem(pr, &s) != KV_OK) return 0;
  (void)budget;
  (void)cand_mult;
  (void)keep_tail;
  return window_ws_bytes(pr, s);
}

int32_t kv_candidate_stride(const kv_problem* pr, int32_t budget, int32_t cand_mult,
                            int32_t keep_tail) {
  kv::Shape s;
  if (check_problem(pr, &s) != KV_OK || cand_mult < 0 || budget < 1) return 0;
  // `budget` may be the row stride of per-problem budgets: no bound by the candidates here
  if (check_budget(pr, budget, keep_tail, true) != KV_OK) return 0;
  if (cand_mult > 0) {
    const int64_t c = (int64_t)cand_mult * budget;
    return c > INT32_MAX ? 0 : (int32_t)c;
  }
  return max_candidates(pr, budget, 0, keep_tail);
}

int kv_window_scores(const kv_problem* pr, const void* q_win, const void* k, float scale,
                     float* row_max, float* row_sum, void* ws, size_t ws_bytes, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!q_win || !k || !row_max || !row_sum) return KV_ERR_NULL;
  if (!aligned16(q_win) || !aligned16(k)) return KV_ERR_ARG;
  if (!std::isfinite(scale)) return KV_ERR_ARG;
  if (ws_bytes < window_ws_bytes(pr, s) || !ws ||
      (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)))
    return KV_ERR_WORKSPACE;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (kv::stream_shape_ok(s, scale)) {
    const kv::StreamPlan plan = stream_plan_of(pr, s);
    if (plan.max_segs == 1)  // one segment per unit: pass 1 writes the row statistics itself
      return launch_status(kv::launch_stream_stats(s, plan, q_win, k, scale, nullptr, row_max,
                                                   row_sum, hs));
    st = launch_status(kv::launch_stream_stats(s, plan, q_win, k, scale, ws, nullptr, nullptr, hs));
    if (st != KV_OK) return st;
    return launch_status(kv::launch_combine_partials(s, ws, plan.seg_keys, plan.max_segs,
                                                     s.row_blocks() * 32, row_max, row_sum, hs));
  }
  return launch_status(kv::launch_window_stats(s, q_win, k, scale, ws, row_max, row_sum, hs));
}

int kv_mu_sigma(const kv_problem* pr, const void* q_win, const void* k, float scale,
                const float* row_max, const float* row_sum, float* mu, float* sigma, float* attn,
                void* stream) {
  return kv_mu_sigma_ex(pr, q_win, k, scale, row_max, row_sum, KV_SIGMA_GROUP_MEAN, mu, sigma,
                        attn, stream);
}

int kv_mu_sigma_ex(const kv_problem* pr, const void* q_win, const void* k, float scale,
                   const float* row_max, const float* row_sum, int32_t sigma_rows, float* mu,
                   float* sigma, float* attn, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!q_win || !k || !row_max || !row_sum || !mu || !sigma) return KV_ERR_NULL;
  if (!aligned16(q_win) || !aligned16(k)) return KV_ERR_ARG;
  if (!std::isfinite(scale)) return KV_ERR_ARG;
  if (sigma_rows != KV_SIGMA_GROUP_MEAN && sigma_rows != KV_SIGMA_ALL_ROWS) return KV_ERR_ARG;
  const bool all = sigma_rows == KV_SIGMA_ALL_ROWS;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (kv::stream_shape_ok(s, scale) && !attn)
    return launch_status(kv::launch_stream_mu_sigma(s, stream_plan_of(pr, s), q_win, k, scale,
                                                    nullptr, row_max, row_sum, nullptr, nullptr,
                                                    mu, sigma, all, hs));
  return launch_status(kv::launch_mu_sigma(s, q_win, k, scale, row_max, row_sum, mu, sigma, attn,
                                           all, hs));
}

int kv_window_mu_sigma(const kv_problem* pr, const void* q_win, const void* k, float scale,
                       float* row_max, float* row_sum, float* mu, float* sigma, void* ws,
                       size_t ws_bytes, void* stream) {
  return kv_window_mu_sigma_ex(pr, q_win, k, scale, KV_SIGMA_GROUP_MEAN, row_max, row_sum, mu,
                               sigma, ws, ws_bytes, stream);
}

int kv_window_mu_sigma_ex(const kv_problem* pr, const void* q_win, const void* k, float scale,
                          int32_t sigma_rows, float* row_max, float* row_sum, float* mu,
                          float* sigma, void* ws, size_t ws_bytes, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!q_win || !k || !row_max || !row_sum || !mu || !sigma) return KV_ERR_NULL;
  if (!aligned16(q_win) || !aligned16(k)) return KV_ERR_ARG;
  if (!std::isfinite(scale)) return KV_ERR_ARG;
  if (sigma_rows != KV_SIGMA_GROUP_MEAN && sigma_rows != KV_SIGMA_ALL_ROWS) return KV_ERR_ARG;
  const bool all = sigma_rows == KV_SIGMA_ALL_ROWS;
  if (ws_bytes < window_ws_bytes(pr, s) || !ws ||
      (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)))
    return KV_ERR_WORKSPACE;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (kv::stream_shape_ok(s, scale)) {
    const kv::StreamPlan plan = stream_plan_of(pr, s);
    if (plan.one_wg())  // both passes of a unit in one workgroup
      return launch_status(kv::launch_stream_window(s, plan, q_win, k, scale, row_max, row_sum, mu,
                                                    sigma, all, hs));
    // several workgroups per unit: one cooperative launch if the grid fits the chip at once
    bool launched = false;
    st = launch_status(kv::launch_stream_window_coop(s, plan, q_win, k, scale, ws, row_max, row_sum,
                                                     mu, sigma, all, spin_limit(), hs, &launched));
    if (st != KV_OK || launched) return st;
    // segment partials, then normalisers, row statistics and mu / sigma in one more pass
    st = launch_status(kv::launch_stream_stats(s, plan, q_win, k, scale, ws, nullptr, nullptr, hs));
    if (st != KV_OK) return st;
    return launch_status(kv::launch_stream_mu_sigma(s, plan, q_win, k, scale, ws, nullptr,
                                                    nullptr, row_max, row_sum, mu, sigma, all, hs));
  }
  // other shapes: chunked row statistics, then a second pass over K
  return launch_status(kv::launch_window_passes(s, q_win, k, scale, ws, row_max, row_sum, mu, sigma,
                                                all, nullptr, hs));
}

int kv_window_mu_sigma_noalloc(const kv_problem* pr, const void* q_win, const void* k, float scale,
                               int32_t sigma_rows, float* row_max, float* row_sum, float* mu,
                               float* sigma, void* stream) {
  static_assert(KV_NOALLOC_SCRATCH_BYTES == kv::kNoAllocScratchBytes, "scratch size");
  kv::Shape s;
  const int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (window_ws_bytes(pr, s) > kv::kNoAllocScratchBytes) return KV_ERR_SCRATCH;
  void* ws = nullptr;
  if (!q_win || !k || !row_max || !row_sum || !mu || !sigma) return KV_ERR_NULL;
  if (kv::noalloc_scratch(&ws) != hipSuccess) return KV_ERR_LAUNCH;
  return kv_window_mu_sigma_ex(pr, q_win, k, scale, sigma_rows, row_max, row_sum, mu, sigma, ws,
                               kv::kNoAllocScratchBytes, stream);
}

size_t kv_base_scores_workspace_bytes(const kv_problem* pr) {
  kv::Shape s;
  if (check_problem(pr, &s) != KV_OK) return 0;
  const size_t need = base_scores_ws_bytes(pr, s, 1.f);
  return one_segment_units(pr, s) ? need : std::max(need, base_scores_ws_bytes(pr, s, -1.f));
}

int kv_window_base_scores(const kv_problem* pr, const void* q_win, const void* k, float scale,
                          const float* lambda1, float w_mu, int32_t sigma_rows, float* row_max,
                          float* row_sum, float* score, void* ws, size_t ws_bytes, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!q_win || !k || !lambda1 || !row_max || !row_sum || !score) return KV_ERR_NULL;
  if (!aligned16(q_win) || !aligned16(k) || !aligned16(score)) return KV_ERR_ARG;
  if (!std::isfinite(scale) || !std::isfinite(w_mu)) return KV_ERR_ARG;
  if (sigma_rows != KV_SIGMA_GROUP_MEAN && sigma_rows != KV_SIGMA_ALL_ROWS) return KV_ERR_ARG;
  const bool fused = scores_in_window_pass(pr, s, scale);
  const size_t need = base_scores_ws_bytes(pr, s, scale);
  if (need > 0 && (ws_bytes < need || !ws || (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1))))
    return KV_ERR_WORKSPACE;
  const bool all = sigma_rows == KV_SIGMA_ALL_ROWS;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (fused)
    return launch_status(kv::launch_stream_window_scores(s, stream_plan_of(pr, s), q_win, k, scale,
                                                         lambda1, w_mu, row_max, row_sum, score,
                                                         all, hs));
  const size_t win = window_ws_bytes(pr, s);
  const kv::ScoreMode sm{score, lambda1, w_mu};
  if (!kv::stream_shape_ok(s, scale))  // the chunked kernels form them in their second pass
    return launch_status(kv::launch_window_passes(s, q_win, k, scale, ws, row_max, row_sum, nullptr,
                                                  nullptr, all, &sm, hs));
  {
    // several workgroups per unit: the one-launch path in base-score mode when the grid fits
    bool launched = false;
    st = launch_status(kv::launch_stream_window_coop(s, stream_plan_of(pr, s), q_win, k, scale, ws,
                                                     row_max, row_sum, nullptr, nullptr, all,
                                                     spin_limit(), hs, &launched, &sm));
    if (st != KV_OK || launched) return st;
  }
  // mu / sigma into the workspace after the window paths' own part, then the scores from them
  const size_t keys = (size_t)token_extent(pr) * pr->h_kv;
  float* mu = reinterpret_cast<float*>(static_cast<char*>(ws) + win);
  float* sigma = reinterpret_cast<float*>(static_cast<char*>(ws) + win + align_up(keys * sizeof(float)));
  st = kv_window_mu_sigma_ex(pr, q_win, k, scale, sigma_rows, row_max, row_sum, mu, sigma, ws, win,
                             stream);
  if (st != KV_OK) return st;
  return launch_status(kv::launch_base_scores(s, mu, sigma, lambda1, w_mu, score, hs));
}

int kv_mmr_select(const kv_problem* pr, const float* mu, const float* sigma, const void* k,
                  const float* lambda1, const float* lambda2, int32_t budget, int32_t cand_mult,
                  int32_t keep_tail, int32_t* sel_idx, float* sel_score, int32_t* cand_idx,
                  float* cand_corr, void* ws, size_t ws_bytes, void* stream) {
  return kv_mmr_select_ex(pr, mu, sigma, k, lambda1, lambda2, budget, cand_mult, keep_tail, nullptr,
                          sel_idx, sel_score, cand_idx, cand_corr, ws, ws_bytes, stream);
}

int kv_mmr_select_ex(const kv_problem* pr, const float* mu, const float* sigma, const void* k,
                     const float* lambda1, const float* lambda2, int32_t budget, int32_t cand_mult,
                     int32_t keep_tail, const kv_select_opts* opts, int32_t* sel_idx,
                     float* sel_score, int32_t* cand_idx, float* cand_corr, void* ws,
                     size_t ws_bytes, void* stream) {
  (void)ws;
  (void)ws_bytes;
  ScoreSource src;
  src.mu = mu;
  src.sigma = sigma;
  src.lambda1 = lambda1;
  return mmr_select_impl(pr, src, k, nullptr, lambda2, budget, cand_mult, keep_tail, opts, sel_idx,
                         sel_score, cand_idx, cand_corr, nullptr, nullptr, stream);
}

int kv_mmr_select_compact(const kv_problem* pr, const float* mu, const float* sigma, const void* k,
                          const void* v, const float* lambda1, const float* lambda2,
                          int32_t budget, int32_t cand_mult, int32_t keep_tail, int32_t* sel_idx,
                          void* k_out, void* v_out, void* ws, size_t ws_bytes, void* stream) {
  (void)ws;
  (void)ws_bytes;
  if (!v || !k_out || !v_out) return KV_ERR_NULL;
  ScoreSource src;
  src.mu = mu;
  src.sigma = sigma;
  src.lambda1 = lambda1;
  return mmr_select_impl(pr, src, k, v, lambda2, budget, cand_mult, keep_tail, nullptr, sel_idx,
                         nullptr, nullptr, nullptr, k_out, v_out, stream);
}

int kv_mmr_select_scored(const kv_problem* pr, const float* score, const void* k, const void* v,
                         const float* lambda2, int32_t budget,
                         int32_t cand_mult, int32_t keep_tail, const kv_select_opts* opts,
                         int32_t* sel_idx, float* sel_score, int32_t* cand_idx, float* cand_corr,
                         void* k_out, void* v_out, void* stream) {
  if (!score) return KV_ERR_NULL;
  if (!aligned16(score)) return KV_ERR_ARG;
  if ((k_out != nullptr) != (v_out != nullptr)) return KV_ERR_NULL;
  if (k_out && !v) return KV_ERR_NULL;
  ScoreSource src;
  src.score = score;
  return mmr_select_impl(pr, src, k, v, lambda2, budget, cand_mult, keep_tail, opts, sel_idx,
                         sel_score, cand_idx, cand_corr, k_out, v_out, stream);
}

size_t kv_candidates_workspace_bytes(const kv_problem* pr, int32_t budget, int32_t cand_mult,
                                     int32_t keep_tail, const kv_select_opts* opts) {
  kv::Shape s;
  if (check_problem(pr, &s) != KV_OK) return 0;
  const int32_t* b_host = opts ? opts->budget_host : nullptr;
  if (cand_mult < 0 || budget < 1 || check_budget(pr, budget, keep_tail, b_host != nullptr) != KV_OK)
    return 0;
  if (opts && opts->pool != 1) return 0;
  const int stride = max_candidates(pr, budget, cand_mult, keep_tail, b_host);
  if (stride > kv::select_max_candidates(pr->d, elem_bytes(pr->dtype))) return 0;
  const bool fused = cands_in_window_pass(pr, s, 1.f, cand_mult, stride);
  const size_t need = cand_ws_bytes(pr, s, stride, 1.f, fused);
  return fused && one_segment_units(pr, s) ? need : std::max(need, cand_ws_bytes(pr, s, stride, -1.f, false));
}

int kv_window_candidates(const kv_problem* pr, const void* q_win, const void* k, float scale,
                         const float* lambda1, int32_t sigma_rows, int32_t budget,
                         int32_t cand_mult, int32_t keep_tail, const kv_select_opts* opts,
                         float* row_max, float* row_sum, void* ws, size_t ws_bytes, void* stream) {
  return window_candidates_impl(pr, q_win, k, scale, lambda1, sigma_rows, budget, cand_mult,
                                keep_tail, opts, row_max, row_sum, ws, ws_bytes, nullptr, stream);
}

int kv_mmr_select_candidates(const kv_problem* pr, const void* ws, size_t ws_bytes, const void* k,
                             const void* v, const float* lambda2, int32_t budget,
                             int32_t cand_mult, int32_t keep_tail, const kv_select_opts* opts,
                             int32_t* sel_idx, float* sel_score, int32_t* cand_idx,
                             float* cand_corr, void* k_out, void* v_out, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if ((k_out != nullptr) != (v_out != nullptr)) return KV_ERR_NULL;
  if (k_out && !v) return KV_ERR_NULL;
  if (cand_mult < 0) return KV_ERR_ARG;
  const int32_t* b_host = opts ? opts->budget_host : nullptr;
  st = check_budget(pr, budget, keep_tail, b_host != nullptr);
  if (st != KV_OK) return st;
  const int stride = max_candidates(pr, budget, cand_mult, keep_tail, b_host);
  const size_t lists = cand_lists_bytes(pr, stride);
  if (ws_bytes < lists + align_up((size_t)pr->n_prob * pr->h_kv * sizeof(float)) || !ws ||
      (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)))
    return KV_ERR_WORKSPACE;
  ScoreSource src;
  src.cand_in = static_cast<const uint64_t*>(ws);
  src.cand_in_max = reinterpret_cast<const float*>(static_cast<const char*>(ws) + lists);
  src.list_stride = stride;
  return mmr_select_impl(pr, src, k, v, lambda2, budget, cand_mult, keep_tail, opts, sel_idx,
                         sel_score, cand_idx, cand_corr, k_out, v_out, stream);
}

int kv_evict_pass(const kv_problem* pr, const void* q_win, const void* k, const void* v,
                  float scale, const float* lambda1, const float* lambda2, int32_t sigma_rows,
                  int32_t budget, int32_t cand_mult, int32_t keep_tail, const kv_select_opts* opts,
                  float* row_max, float* row_sum, int32_t* sel_idx, float* sel_score, void* k_out,
                  void* v_out, void* ws, size_t ws_bytes, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  // the selection's own checks first: nothing runs unless both calls would
  if (!lambda2 || !sel_idx) return KV_ERR_NULL;
  if ((k_out != nullptr) != (v_out != nullptr)) return KV_ERR_NULL;
  if (k_out && !v) return KV_ERR_NULL;
  if (k_out && (!aligned16(v) || !aligned16(k_out) || !aligned16(v_out))) return KV_ERR_ARG;
  if (k_out && budget > kMaxCompactBudget) return KV_ERR_BUDGET;
  if (cand_mult < 0 || (int64_t)cand_mult * budget > INT32_MAX) return KV_ERR_ARG;
  const int32_t* b_host = opts ? opts->budget_host : nullptr;
  const int32_t* b_dev = opts ? opts->budget_dev : nullptr;
  st = check_budget(pr, budget, keep_tail, b_host != nullptr || b_dev != nullptr);
  if (st != KV_OK) return st;
  const int stride = max_candidates(pr, budget, cand_mult, keep_tail, b_host);
  // one launch for the cut and the selection: in the window kernel up to kCandSelectMax candidates,
  // in the selection kernel where that cuts them from the scores
  if (!cands_in_window_pass(pr, s, scale, cand_mult, stride) || stride <= kv::kCandSelectMax) {
    kv::CandSelect sel{lambda2, sel_idx, sel_score, v, k_out, v_out, budget + keep_tail};
    return window_candidates_impl(pr, q_win, k, scale, lambda1, sigma_rows, budget, cand_mult,
                                  keep_tail, opts, row_max, row_sum, ws, ws_bytes, &sel, stream);
  }
  st = kv_window_candidates(pr, q_win, k, scale, lambda1, sigma_rows, budget, cand_mult,
                            keep_tail, opts, row_max, row_sum, ws, ws_bytes, stream);
  if (st != KV_OK) return st;
  return kv_mmr_select_candidates(pr, ws, ws_bytes, k, v, lambda2, budget, cand_mult, keep_tail,
                                  opts, sel_idx, sel_score, nullptr, nullptr, k_out, v_out, stream);
}

int kv_compact_cache(const kv_problem* pr, const void* k, const void* v, const int32_t* sel_idx,
                     int32_t budget, int32_t keep_tail, void* k_out, void* v_out, void* stream) {
  return kv_compact_cache_ex(pr, k, v, sel_idx, budget, keep_tail, nullptr, nullptr, 0, k_out,
                             v_out, stream);
}

int kv_compact_cache_ex(const kv_problem* pr, const void* k, const void* v,
                        const int32_t* sel_idx, int32_t budget, int32_t keep_tail,
                        const int32_t* budget_host, const int32_t* budget_dev, int32_t out_rows,
                        void* k_out, void* v_out, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  if (!k || !v || !sel_idx || !k_out || !v_out) return KV_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_out) || !aligned16(v_out)) return KV_ERR_ARG;
  st = check_budget(pr, budget, keep_tail, budget_host != nullptr || budget_dev != nullptr);
  if (st != KV_OK) return st;
  st = check_budgets(pr, budget, keep_tail, budget_host, budget_dev);
  if (st != KV_OK) return st;
  if (budget > kMaxCompactBudget) return KV_ERR_BUDGET;
  if (out_rows == 0) out_rows = budget + keep_tail;
  if (out_rows < budget + keep_tail) return KV_ERR_ARG;
  return launch_status(kv::launch_compact(s, k, v, sel_idx, budget, budget_dev, keep_tail,
                                          out_rows, k_out, v_out,
                                          static_cast<hipStream_t>(stream)));
}

namespace {

int check_cache_batch(const kv_cache_batch* cb) {
  if (!cb) return KV_ERR_NULL;
  if (cb->dtype != KV_F32 && cb->dtype != KV_BF16) return KV_ERR_DTYPE;
  if (cb->n_prob < 1 || cb->n_prob > kMaxGrid) return KV_ERR_ARG;
  if (!cb->len_host || !cb->len_dev) return KV_ERR_NULL;
  if (cb->h_kv < 1 || cb->h_kv > kMaxGrid || cb->h_q < cb->h_kv || cb->h_q % cb->h_kv != 0 ||
      cb->h_q / cb->h_kv > 8)
    return KV_ERR_SHAPE;
  if (cb->d != 64 && cb->d != 128) return KV_ERR_SHAPE;
  if (cb->row_stride < 1 || cb->row_stride > kMaxLen) return KV_ERR_SHAPE;
  for (int p = 0; p < cb->n_prob; ++p)
    if (cb->len_host[p] < 0 || cb->len_host[p] > cb->row_stride) return KV_ERR_SHAPE;
  return KV_OK;
}

kv::DecodePlan decode_plan_of(const kv_cache_batch* cb) {
  int max_len = 0;
  for (int p = 0; p < cb->n_prob; ++p) max_len = std::max(max_len, (int)cb->len_host[p]);
  return kv::decode_plan(cb->n_prob, cb->h_kv, max_len, cb->h_q / cb->h_kv, cb->d * elem_bytes(cb->dtype));
}

}  // namespace

size_t kv_decode_workspace_bytes(const kv_cache_batch* cb) {
  if (check_cache_batch(cb) != KV_OK) return 0;
  return align_up(kv::decode_ws_bytes(cb->n_prob, cb->h_q, cb->d, decode_plan_of(cb)));
}

int kv_decode_attention(const kv_cache_batch* cb, const void* q, void* k_cache, void* v_cache,
                        const void* k_new, const void* v_new, float scale, float* out, void* ws,
                        size_t ws_bytes, void* stream) {
  int st = check_cache_batch(cb);
  if (st != KV_OK) return st;
  if (!q || !k_cache || !v_cache || !out) return KV_ERR_NULL;
  if ((k_new == nullptr) != (v_new == nullptr)) return KV_ERR_NULL;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) ||
      (k_new && (!aligned16(k_new) || !aligned16(v_new))))
    return KV_ERR_ARG;
  if (!std::isfinite(scale)) return KV_ERR_ARG;
  for (int p = 0; p < cb->n_prob; ++p) {
    const int len = cb->len_host[p];
    if (k_new ? len >= cb->row_stride : len < 1) return KV_ERR_SHAPE;
  }
  const kv::DecodePlan plan = decode_plan_of(cb);
  if (plan.n_split > kMaxGrid) return KV_ERR_SHAPE;
  const size_t need = align_up(kv::decode_ws_bytes(cb->n_prob, cb->h_q, cb->d, plan));
  if (need > 0 && (ws_bytes < need || !ws || (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1))))
    return KV_ERR_WORKSPACE;
  kv::DecodeArgs a;
  a.q = q;
  a.k = k_cache;
  a.v = v_cache;
  a.k_new = k_new;
  a.v_new = v_new;
  a.lens = cb->len_dev;
  a.h_q = cb->h_q;
  a.h_kv = cb->h_kv;
  a.row_stride = cb->row_stride;
  a.c = scale * kLog2eF;
  a.split_rows = plan.split_rows;
  a.n_split = plan.n_split;
  a.out = out;
  a.part = static_cast<float*>(ws);
  return launch_status(kv::launch_decode(cb->dtype == KV_BF16 ? kv::kDtBf16 : kv::kDtF32, cb->d,
                                         cb->n_prob, a, static_cast<hipStream_t>(stream)));
}

namespace {

// Checks shared by the paged entry points; fills the kernels' description.  tables: only what the block
// tables need (the pools and the head layout may be unset).
int check_paged(const kv_paged_cache* c, kv::Paged* pc, bool tables = false) {
  if (!c) return KV_ERR_NULL;
  if (c->n_prob < 1 || c->n_prob > kMaxGrid) return KV_ERR_ARG;
  if (!c->table || !c->len) return KV_ERR_NULL;
  if (c->block_rows != 16 && c->block_rows != 32 && c->block_rows != 64 && c->block_rows != 128)
    return KV_ERR_SHAPE;
  // slots are 32-bit numbers, and so are a problem's rows
  if (c->n_blocks < 1 || (int64_t)c->n_blocks * c->block_rows > INT32_MAX) return KV_ERR_SHAPE;
  if (c->table_stride < 1 || (int64_t)c->table_stride * c->block_rows > INT32_MAX) return KV_ERR_SHAPE;
  if (!tables) {
    if (c->dtype != KV_F32 && c->dtype != KV_BF16) return KV_ERR_DTYPE;
    if (c->qtype != KV_E4M3 && c->qtype != KV_INT8 && c->qtype != KV_E2M1) return KV_ERR_DTYPE;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return KV_ERR_NULL;
    if (!aligned16(c->k) || !aligned16(c->v)) return KV_ERR_ARG;
    if (c->qtype == KV_E2M1 && (!aligned16(c->k_scale) || !aligned16(c->v_scale))) return KV_ERR_ARG;
    if (c->h_kv < 1 || c->h_kv > 4096 || c->h_q < c->h_kv || c->h_q % c->h_kv != 0 || c->h_q / c->h_kv > 16)
      return KV_ERR_SHAPE;
    if (c->d != 64 && c->d != 128) return KV_ERR_SHAPE;
    if (c->max_len < 0 || c->max_len > kMaxLen) return KV_ERR_SHAPE;
  }
  pc->dtype = c->dtype == KV_BF16 ? kv::kDtBf16 : kv::kDtF32;
  pc->qtype = c->qtype == KV_E4M3 ? kv::kQtE4m3 : c->qtype == KV_INT8 ? kv::kQtInt8 : kv::kQtE2m1;
  pc->n_prob = c->n_prob;
  pc->h_q = c->h_q;
  pc->h_kv = c->h_kv;
  pc->d = c->d;
  pc->shift = c->block_rows == 16 ? 4 : (c->block_rows == 32 ? 5 : (c->block_rows == 64 ? 6 : 7));
  pc->n_blocks = c->n_blocks;
  pc->table_stride = c->table_stride;
  pc->max_len = c->max_len;
  pc->k = static_cast<uint8_t*>(c->k);
  pc->v = static_cast<uint8_t*>(c->v);
  pc->k_scale = c->k_scale;
  pc->v_scale = c->v_scale;
  pc->table = c->table;
  pc->len = c->len;
  return KV_OK;
}

// Elements between two tokens' rows of `heads` heads: 0 is packed; whole 16-byte chunks, and at most kMaxTokenStride
// (the kernels' offsets within a few tokens are 32-bit).
int check_stride(const kv::Paged& pc, int heads, int64_t* stride) {
  const int64_t packed = (int64_t)heads * pc.d;
  if (*stride == 0) *stride = packed;
  if (*stride < packed || *stride > kMaxTokenStride || *stride % (pc.dtype == kv::kDtBf16 ? 8 : 4) != 0) return KV_ERR_ARG;
  return KV_OK;
}

// A rotation of heads of d elements; fills the kernels' description.
int check_rotary(const kv_rotary* r, int d, kv::Rotary* rot) {
  if (!r || !r->freq) return KV_ERR_NULL;
  if (r->layout != KV_ROTARY_HALF && r->layout != KV_ROTARY_INTERLEAVED) return KV_ERR_ARG;
  if (!std::isfinite(r->factor) || (reinterpret_cast<uintptr_t>(r->freq) & 7)) return KV_ERR_ARG;
  if (r->rot_dim < 16 || r->rot_dim > d || r->rot_dim % 16 != 0) return KV_ERR_SHAPE;
  *rot = {r->layout == KV_ROTARY_INTERLEAVED, r->rot_dim, r->inverse ? -1.f : 1.f, r->factor, r->freq};
  return KV_OK;
}

// Whether n rows of x_bytes bytes, x_step apart, meet n of out_bytes, out_step apart.
bool rows_overlap(const void* x, int64_t x_step, int64_t x_bytes, const void* out, int64_t out_step, int64_t out_bytes, int64_t n) {
  const intptr_t p = reinterpret_cast<intptr_t>(x), q = reinterpret_cast<intptr_t>(out);
  if (p >= q + (n - 1) * out_step + out_bytes || q >= p + (n - 1) * x_step + x_bytes) return false;
  if (x_step != out_step || n == 1) return true;
  // slices of the same wide rows
  const int64_t apart = ((q - p) % x_step + x_step) % x_step;
  return apart < x_bytes || x_step - apart < out_bytes;
}

// The rows of a rotation from x to out.
int check_rotate(const kv::Rotary& rot, int dtype, int heads, int d, const void* x, int64_t x_stride, const int32_t* pos, int n_tok,
                 void* out, int64_t out_stride, kv::RotateArgs* a) {
  if (!x || !out || !pos) return KV_ERR_NULL;
  if (!aligned16(x) || !aligned16(out) || n_tok < 1) return KV_ERR_ARG;
  if (n_tok > kMaxRotated) return KV_ERR_SHAPE;
  kv::Paged pc{};
  pc.dtype = dtype;
  pc.d = d;
  int st = check_stride(pc, heads, &x_stride);
  if (st == KV_OK) st = check_stride(pc, heads, &out_stride);
  if (st != KV_OK) return st;
  const int64_t e = dtype == kv::kDtBf16 ? 2 : 4;
  const int64_t bytes = (int64_t)heads * d * e;
  const bool in_place = x == out && (x_stride == out_stride || n_tok == 1);
  if (!in_place && rows_overlap(x, x_stride * e, bytes, out, out_stride * e, bytes, n_tok)) return KV_ERR_ARG;
  *a = {rot, x, out, x_stride, out_stride, pos, n_tok, heads, 1};
  return KV_OK;
}

// Tokens of an attention call, and the launch they take.
int check_tokens(const kv::Paged& pc, int32_t n_tok, int32_t max_q, kv::PagedPlan* plan) {
  if (n_tok < 1 || max_q < 1 || max_q > n_tok) return KV_ERR_ARG;
  if (max_q > kMaxLen) return KV_ERR_SHAPE;
  *plan = kv::paged_plan(pc, max_q);
  // the rounds of all problems are counted in 32 bits
  if (plan->shares && ((int64_t)pc.max_len / 128 + 1) * pc.n_prob > INT32_MAX) return KV_ERR_SHAPE;
  return kv::paged_grid_groups(pc, max_q, *plan) > kMaxGrid ? KV_ERR_SHAPE : KV_OK;
}

// kv_paged_tables' arrays.  in_place: whether an input is written as an output, in one of the ways that the header
// allows; KV_ERR_ARG where arrays overlap in any other.
int check_overlaps(const kv::Paged& pc, const kv::TablesArgs& a, bool* in_place) {
  struct Words {
    const int32_t* at;
    int64_t n;
  };
  const int64_t n = pc.n_prob;
  enum { kLen = 1, kTable = 2, kTok = 4, kBlk = 8, kSlots = 16, kTaken = 32 };
  const Words outs[] = {{pc.len, n},         {pc.table, n * pc.table_stride}, {a.tok_off, n + 1},
                        {a.blk_off, n + 1}, {a.slots, a.n_slots},             {a.taken_out, 1}};
  constexpr int kOuts = sizeof(outs) / sizeof(outs[0]);
  auto met = [&](const Words& x) {  // the outputs that x overlaps
    int m = 0;
    for (int i = 0; i < kOuts; ++i) {
      const uintptr_t p = reinterpret_cast<uintptr_t>(x.at), q = reinterpret_cast<uintptr_t>(outs[i].at);
      if (p && q && x.n > 0 && outs[i].n > 0 && p < q + outs[i].n * sizeof(int32_t) && q < p + x.n * sizeof(int32_t)) m |= 1 << i;
    }
    return m;
  };
  // (the count and the last offset are one value)
  const int total = a.taken_out == a.blk_off + n ? kBlk | kTaken : 0;
  for (int i = 0; i < kOuts; ++i) {
    const int others = met(outs[i]) & ~(1 << i);
    if (others && (others | 1 << i) != total) return KV_ERR_ARG;
  }
  const int len_in = a.len_in == pc.len ? 0 : met({a.len_in, n}), add = a.add == pc.len ? 0 : met({a.add, n});
  const int taken = met({a.taken_in, 1});
  if (len_in || add || (taken & ~(kBlk | kTaken)) || met({a.free_blocks, a.n_free})) return KV_ERR_ARG;
  *in_place = a.len_in == pc.len || a.add == pc.len || taken;
  return KV_OK;
}

}  // namespace

int kv_paged_tables(const kv_paged_cache* c, const int32_t* len_in, const int32_t* add,
                    const int32_t* free_blocks, int32_t n_free, const int32_t* taken_in,
                    int32_t* taken_out, int32_t* tok_off, int32_t* blk_off, int32_t* slots,
                    int32_t n_slots, void* stream) {
  kv::Paged pc{};
  const int st = check_paged(c, &pc, true);
  if (st != KV_OK) return st;
  if (!tok_off || !blk_off || (!slots && n_slots > 0)) return KV_ERR_NULL;
  if (n_free < 0 || n_slots < 0) return KV_ERR_ARG;
  kv::TablesArgs a{len_in, add, free_blocks, n_free, taken_in, taken_out, tok_off, blk_off, slots, n_slots,
                   aligned16(slots), false};
  const int overlaps = check_overlaps(pc, a, &a.in_place);
  if (overlaps != KV_OK) return overlaps;
  return launch_status(kv::launch_paged_tables(pc, a, static_cast<hipStream_t>(stream)));
}

int kv_paged_append(const kv_paged_cache* c, const void* k_new, const void* v_new, int64_t tok_stride,
                    const int32_t* slots, int32_t n_tok, void* stream) {
  kv::Paged pc{};
  int st = check_paged(c, &pc);
  if (st != KV_OK) return st;
  if (!k_new || !v_new || !slots) return KV_ERR_NULL;
  if (!aligned16(k_new) || !aligned16(v_new) || n_tok < 1) return KV_ERR_ARG;
  st = check_stride(pc, pc.h_kv, &tok_stride);
  if (st != KV_OK) return st;
  return launch_status(kv::launch_paged_append(pc, k_new, v_new, tok_stride, slots, n_tok,
                                               static_cast<hipStream_t>(stream)));
}

int kv_rotate(const kv_rotary* r, int32_t dtype, int32_t heads, int32_t d, const void* x, int64_t x_stride,
              const int32_t* pos, int32_t n_tok, void* out, int64_t out_stride, void* stream) {
  if (dtype != KV_F32 && dtype != KV_BF16) return KV_ERR_DTYPE;
  if ((d != 64 && d != 128) || heads < 1 || heads > kMaxTokenStride / d) return KV_ERR_SHAPE;
  kv::Rotary rot;
  int st = check_rotary(r, d, &rot);
  if (st != KV_OK) return st;
  kv::RotateArgs a;
  const int dt = dtype == KV_BF16 ? kv::kDtBf16 : kv::kDtF32;
  st = check_rotate(rot, dt, heads, d, x, x_stride, pos, n_tok, out, out_stride, &a);
  if (st != KV_OK) return st;
  return launch_status(kv::launch_rotate(dt, d, a, static_cast<hipStream_t>(stream)));
}

int kv_paged_append_rotated(const kv_paged_cache* c, const kv_rotary* r, const int32_t* pos, const void* q, int64_t q_stride,
                            void* q_out, int64_t q_out_stride, const void* k_new, const void* v_new, int64_t tok_stride,
                            const int32_t* slots, int32_t n_tok, void* stream) {
  kv::Paged pc{};
  int st = check_paged(c, &pc);
  if (st != KV_OK) return st;
  kv::Rotary rot;
  st = check_rotary(r, pc.d, &rot);
  if (st != KV_OK) return st;
  if (!pos || !k_new || !v_new || !slots || (q != nullptr) != (q_out != nullptr)) return KV_ERR_NULL;
  if (!aligned16(k_new) || !aligned16(v_new) || n_tok < 1) return KV_ERR_ARG;
  if (n_tok > kMaxRotated) return KV_ERR_SHAPE;
  st = check_stride(pc, pc.h_kv, &tok_stride);
  if (st != KV_OK) return st;
  kv::RotateArgs rq{rot, nullptr, nullptr, 0, 0, pos, n_tok, 0, 1};
  if (q) {
    st = check_rotate(rot, pc.dtype, pc.h_q, pc.d, q, q_stride, pos, n_tok, q_out, q_out_stride, &rq);
    if (st != KV_OK) return st;
    const int64_t e = pc.dtype == kv::kDtBf16 ? 2 : 4, q_bytes = (int64_t)pc.h_q * pc.d * e, bytes = (int64_t)pc.h_kv * pc.d * e;
    for (const void* rows : {k_new, v_new})
      if (rows_overlap(rows, tok_stride * e, bytes, q_out, rq.out_stride * e, q_bytes, n_tok)) return KV_ERR_ARG;
  }
  return launch_status(kv::launch_paged_append_rotated(pc, rq, k_new, v_new, tok_stride, slots, static_cast<hipStream_t>(stream)));
}

int kv_paged_rows(const kv_paged_cache* c, const int64_t* row_off, int64_t n_rows, void* k_out, void* v_out, void* stream) {
  kv::Paged pc{};
  const int st = check_paged(c, &pc);
  if (st != KV_OK) return st;
  if (!row_off || (!k_out && !v_out)) return KV_ERR_NULL;
  if (!aligned16(k_out) || !aligned16(v_out) || n_rows < 1) return KV_ERR_ARG;
  const uintptr_t kp = reinterpret_cast<uintptr_t>(k_out), vp = reinterpret_cast<uintptr_t>(v_out);
  const uintptr_t row_bytes = (uintptr_t)pc.h_kv * pc.d * (pc.dtype == kv::kDtBf16 ? 2 : 4), apart = kp > vp ? kp - vp : vp - kp;
  if (k_out && v_out && apart / row_bytes < (uintptr_t)n_rows) return KV_ERR_ARG;
  return launch_status(kv::launch_paged_rows(pc, row_off, n_rows, k_out, v_out, static_cast<hipStream_t>(stream)));
}

int kv_rotary_frequencies(int32_t family, double base, const double* params_host, int32_t n_params, int32_t rot_dim,
                          double* freq_host, float* factor_host) {
  if (!freq_host || !factor_host) return KV_ERR_NULL;
  const int wanted[] = {0, 1, 1, 4, 4};
  if (family < KV_ROTARY_PLAIN || family > KV_ROTARY_BANDS || n_params != wanted[family]) return KV_ERR_ARG;
  if (n_params > 0 && !params_host) return KV_ERR_NULL;
  if (rot_dim < (family == KV_ROTARY_NTK ? 4 : 2) || rot_dim % 2 != 0 || !(base > 1) || !std::isfinite(base)) return KV_ERR_ARG;
  for (int i = 0; i < n_params; ++i)
    if (!(params_host[i] > 0) || !std::isfinite(params_host[i])) return KV_ERR_ARG;
  const double F = n_params > 0 ? params_host[0] : 1.0, r = rot_dim, kTwoPi = 6.283185307179586;
  if (F < 1) return KV_ERR_ARG;
  if (family == KV_ROTARY_YARN && !(params_host[2] > params_host[3])) return KV_ERR_ARG;
  if (family == KV_ROTARY_BANDS && !(params_host[3] > params_host[2])) return KV_ERR_ARG;
  if (family == KV_ROTARY_NTK) base *= std::pow(F, r / (r - 2));
  double lo = 0, hi = 0;
  if (family == KV_ROTARY_YARN) {
    auto at = [&](double turns) { return r * std::log(params_host[1] / (kTwoPi * turns)) / (2 * std::log(base)); };
    lo = std::max(std::floor(at(params_host[2])), 0.0);
    hi = std::min(std::ceil(at(params_host[3])), r - 1);
  }
  *factor_host = family == KV_ROTARY_YARN ? (float)(0.1 * std::log(F) + 1) : 1.f;
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / r);
    double keep = 1;  // the share of the unscaled frequency
    if (family == KV_ROTARY_LINEAR) keep = 0;
    else if (family == KV_ROTARY_YARN) keep = 1 - std::min(std::max((i - lo) / std::max(hi - lo, 1e-3), 0.0), 1.0);
    else if (family == KV_ROTARY_BANDS)
      keep = std::min(std::max((params_host[1] * f / kTwoPi - params_host[2]) / (params_host[3] - params_host[2]), 0.0), 1.0);
    freq_host[i] = keep == 1 ? f : f * ((1 - keep) / F + keep);
  }
  return KV_OK;
}

int kv_paged_compact(const kv_problem* pr, const void* k, const void* v, const int32_t* sel_idx,
                     int32_t budget, int32_t keep_tail, const int32_t* budget_host,
                     const int32_t* budget_dev, const kv_paged_cache* c, void* stream) {
  kv::Shape s;
  int st = check_problem(pr, &s);
  if (st != KV_OK) return st;
  kv::Paged pc{};
  st = check_paged(c, &pc);
  if (st != KV_OK) return st;
  if (!k || !v || !sel_idx) return KV_ERR_NULL;
  if (!aligned16(k) || !aligned16(v)) return KV_ERR_ARG;
  if (c->dtype != pr->dtype) return KV_ERR_DTYPE;
  if (pc.n_prob != s.n_prob || pc.h_kv != s.h_kv || pc.d != s.d) return KV_ERR_SHAPE;
  st = check_budget(pr, budget, keep_tail, budget_host != nullptr || budget_dev != nullptr);
  if (st != KV_OK) return st;
  st = check_budgets(pr, budget, keep_tail, budget_host, budget_dev);
  if (st != KV_OK) return st;
  if (budget > kMaxCompactBudget) return KV_ERR_BUDGET;
  // every problem's kept rows fit its row of the table
  for (int p = 0; p < pr->n_prob; ++p) {
    const int64_t rows = (int64_t)(budget_host ? budget_host[p] : budget) + keep_tail;
    if (rows > (int64_t)pc.table_stride << pc.shift) return KV_ERR_SHAPE;
  }
  return launch_status(kv::launch_paged_compact(pc, s.lens, s.max_len, s.tok_off, k, v, sel_idx, budget, budget_dev,
                                                keep_tail, static_cast<hipStream_t>(stream)));
}

size_t kv_paged_attention_workspace_bytes(const kv_paged_cache* c, int32_t n_tok, int32_t max_q) {
  kv::Paged pc{};
  kv::PagedPlan plan;
  if (check_paged(c, &pc) != KV_OK || check_tokens(pc, n_tok, max_q, &plan) != KV_OK) return 0;
  return align_up(kv::paged_ws_bytes(pc, n_tok, max_q, plan));
}

int kv_paged_attention(const kv_paged_cache* c, const void* q, int64_t q_stride, const int32_t* tok_off,
                       int32_t n_tok, int32_t max_q, float scale, void* out, void* ws, size_t ws_bytes,
                       void* stream) {
  kv::PagedAttnArgs a{};
  int st = check_paged(c, &a.pc);
  if (st != KV_OK) return st;
  if (!q || !out) return KV_ERR_NULL;
  // (the kernels take powers of two: the scale times log2(e))
  if (!aligned16(q) || !aligned16(out) || !std::isfinite(scale * kLog2eF)) return KV_ERR_ARG;
  kv::PagedPlan plan;
  st = check_tokens(a.pc, n_tok, max_q, &plan);
  if (st != KV_OK) return st;
  if (!tok_off && (n_tok != a.pc.n_prob || max_q != 1)) return KV_ERR_ARG;
  st = check_stride(a.pc, a.pc.h_q, &q_stride);
  if (st != KV_OK) return st;
  const size_t need = align_up(kv::paged_ws_bytes(a.pc, n_tok, max_q, plan));
  if (need > 0 && (ws_bytes < need || !ws || (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1))))
    return KV_ERR_WORKSPACE;
  a.q = q;
  a.q_stride = q_stride;
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  a.max_q = max_q;
  a.c = scale * kLog2eF;
  a.out = out;
  a.split_rows = plan.split_rows;
  a.n_split = plan.n_split;
  a.part = static_cast<float*>(ws);
  a.shares = plan.shares;
  if (plan.shares) {
    a.prefix = static_cast<int32_t*>(ws);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + kv::paged4_prefix_bytes(a.pc, max_q, plan.shares));
  }
  return launch_status(kv::launch_paged_attention(a, plan, static_cast<hipStream_t>(stream)));
}

int kv_pyramid_budgets(int32_t budget, int32_t n_layers, double beta, int32_t* budgets_host) {
  if (!budgets_host) return KV_ERR_NULL;
  if (budget < 1 || n_layers < 1 || !(beta >= 1.0) || !std::isfinite(beta)) return KV_ERR_ARG;
  if (n_layers == 1) {
    budgets_host[0] = budget;
    return KV_OK;
  }
  const int64_t b_min = std::max<int64_t>(1, (int64_t)std::floor((double)budget / beta));
  const int64_t b_max = 2 * (int64_t)budget - b_min, span = b_max - b_min, n1 = n_layers - 1;
  for (int64_t l = 0; l < n_layers; ++l) {
    // the linear budget of layer l rounded away from `budget`; layers l and n-1-l sum to 2 budget
    int64_t b;
    if (2 * l < n1) b = b_max - (l * span) / n1;
    else if (2 * l == n1) b = budget;
    else b = b_min + ((n1 - l) * span) / n1;
    budgets_host[l] = (int32_t)b;
  }
  return KV_OK;
}

int kv_depth_profile(int32_t family, const double* params_host, int32_t n_params,
                     int32_t n_layers, float* lambda_out_host) {
  if (!params_host || !lambda_out_host) return KV_ERR_NULL;
  if (n_layers < 1) return KV_ERR_ARG;
  switch (family) {
    case KV_PROFILE_GLOBAL:
      if (n_params != 1) return KV_ERR_ARG;
      break;
    case KV_PROFILE_SEGMENTS:
      if (n_params < 1 || n_params > n_layers) return KV_ERR_ARG;
      break;
    case KV_PROFILE_CURVE:
      if (n_params != 3) return KV_ERR_ARG;
      break;
    default:
      return KV_ERR_ARG;
  }
  for (int l = 0; l < n_layers; ++l) {
    double a;
    if (family == KV_PROFILE_GLOBAL) {
      a = params_host[0];
    } else if (family == KV_PROFILE_SEGMENTS) {
      a = params_host[((int64_t)n_params * l) / n_layers];
    } else {
      const double t = n_layers == 1 ? 0.0 : (double)l / (double)(n_layers - 1);
      a = params_host[0] + params_host[1] * t + params_host[2] * t * t;
    }
    lambda_out_host[l] = (float)std::sinh(a);
  }
  return KV_OK;
}

}  // extern "C"
