"""ctypes binding of libkvevict.so, with the same names as the C ABI (include/kvevict.h).

Argument marshalling only: every function checks that tensors are contiguous device tensors,
passes their addresses and the current HIP stream, and raises KvError on a negative status.  All
computation happens in the library's gfx950 kernels.  Loading fails loudly if the library has not
been built; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

KV_OK = 0
KV_ERR_NULL = -1
KV_ERR_SHAPE = -2
KV_ERR_DTYPE = -3
KV_ERR_BUDGET = -4
KV_ERR_WORKSPACE = -5
KV_ERR_LAUNCH = -6
KV_ERR_ARG = -7
KV_ERR_SCRATCH = -8
KV_NOALLOC_SCRATCH_BYTES = 16 << 20

KV_SIGMA_GROUP_MEAN = 0
KV_SIGMA_ALL_ROWS = 1
SIGMA_ROWS = {"group_mean": KV_SIGMA_GROUP_MEAN, "all_rows": KV_SIGMA_ALL_ROWS}

KV_F32 = 0
KV_BF16 = 1

KV_E4M3 = 0
KV_INT8 = 1
KV_E2M1 = 4

KV_ROTARY_HALF = 0
KV_ROTARY_INTERLEAVED = 1
ROTARY_LAYOUTS = {"half": KV_ROTARY_HALF, "interleaved": KV_ROTARY_INTERLEAVED}
ROTARY_FAMILIES = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}

KV_PROFILE_GLOBAL = 0
KV_PROFILE_SEGMENTS = 1
KV_PROFILE_CURVE = 2
PROFILE_FAMILIES = {"global": KV_PROFILE_GLOBAL, "segments": KV_PROFILE_SEGMENTS,
                    "curve": KV_PROFILE_CURVE}

# KVEVICT_LIB selects another build of the same library (the host-sanitized one of the CPU tests)
LIB_PATH = os.environ.get("KVEVICT_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                         "libkvevict.so")

SYMBOLS = ("kv_strerror", "kv_version", "kv_workspace_bytes", "kv_candidate_stride",
           "kv_window_scores", "kv_mu_sigma", "kv_mu_sigma_ex", "kv_window_mu_sigma",
           "kv_window_mu_sigma_ex", "kv_window_mu_sigma_noalloc", "kv_window_base_scores",
           "kv_base_scores_workspace_bytes", "kv_mmr_select", "kv_mmr_select_ex",
           "kv_mmr_select_compact", "kv_mmr_select_scored", "kv_window_candidates",
           "kv_candidates_workspace_bytes", "kv_mmr_select_candidates", "kv_evict_pass",
           "kv_compact_cache", "kv_compact_cache_ex", "kv_decode_workspace_bytes",
           "kv_decode_attention", "kv_paged_tables", "kv_paged_append", "kv_paged_compact",
           "kv_paged_attention", "kv_paged_attention_workspace_bytes", "kv_paged_append_rotated",
           "kv_paged_rows", "kv_rotate", "kv_rotary_frequencies", "kv_pyramid_budgets",
           "kv_depth_profile")


class KvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


class KvProblem(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_prob", ctypes.c_int32), ("h_q", ctypes.c_int32),
                ("h_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("w", ctypes.c_int32),
                ("len_host", ctypes.c_void_p), ("tok_off_host", ctypes.c_void_p),
                ("len_dev", ctypes.c_void_p), ("tok_off_dev", ctypes.c_void_p)]


class KvCacheBatch(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_prob", ctypes.c_int32), ("h_q", ctypes.c_int32),
                ("h_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("row_stride", ctypes.c_int32),
                ("len_host", ctypes.c_void_p), ("len_dev", ctypes.c_void_p)]


class KvPagedCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "qtype", "n_prob", "h_q", "h_kv", "d", "block_rows",
                                              "n_blocks", "table_stride", "max_len")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "table", "len")]


class KvRotary(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("inverse", ctypes.c_int32),
                ("factor", ctypes.c_float), ("freq", ctypes.c_void_p)]


class KvSelectOpts(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_int32), ("w_mu", ctypes.c_float),
                ("budget_host", ctypes.c_void_p), ("budget_dev", ctypes.c_void_p)]


_LIB = None


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        h = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        pr = ctypes.POINTER(KvProblem)
        h.kv_strerror.argtypes = [ctypes.c_int]
        h.kv_strerror.restype = ctypes.c_char_p
        h.kv_version.argtypes = []
        h.kv_version.restype = ctypes.c_int
        h.kv_workspace_bytes.argtypes = [pr, i32, i32, i32]
        h.kv_workspace_bytes.restype = sz
        h.kv_candidate_stride.argtypes = [pr, i32, i32, i32]
        h.kv_candidate_stride.restype = i32
        h.kv_window_scores.argtypes = [pr, vp, vp, ctypes.c_float, vp, vp, vp, sz, vp]
        h.kv_mu_sigma.argtypes = [pr, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp, vp]
        h.kv_window_mu_sigma.argtypes = [pr, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp, sz, vp]
        h.kv_mu_sigma_ex.argtypes = [pr, vp, vp, ctypes.c_float, vp, vp, i32, vp, vp, vp, vp]
        h.kv_window_mu_sigma_ex.argtypes = [pr, vp, vp, ctypes.c_float, i32, vp, vp, vp, vp, vp,
                                            sz, vp]
        h.kv_window_mu_sigma_noalloc.argtypes = [pr, vp, vp, ctypes.c_float, i32, vp, vp, vp, vp,
                                                 vp]
        h.kv_window_base_scores.argtypes = [pr, vp, vp, ctypes.c_float, vp, ctypes.c_float, i32,
                                            vp, vp, vp, vp, sz, vp]
        h.kv_base_scores_workspace_bytes.argtypes = [pr]
        h.kv_base_scores_workspace_bytes.restype = sz
        h.kv_mmr_select_scored.argtypes = [pr, vp, vp, vp, vp, i32, i32, i32,
                                           ctypes.POINTER(KvSelectOpts), vp, vp, vp, vp, vp, vp, vp]
        h.kv_window_candidates.argtypes = [pr, vp, vp, ctypes.c_float, vp, i32, i32, i32, i32,
                                           ctypes.POINTER(KvSelectOpts), vp, vp, vp, sz, vp]
        h.kv_candidates_workspace_bytes.argtypes = [pr, i32, i32, i32,
                                                    ctypes.POINTER(KvSelectOpts)]
        h.kv_candidates_workspace_bytes.restype = sz
        h.kv_mmr_select_candidates.argtypes = [pr, vp, sz, vp, vp, vp, i32, i32, i32,
                                               ctypes.POINTER(KvSelectOpts), vp, vp, vp, vp, vp,
                                               vp, vp]
        h.kv_evict_pass.argtypes = [pr, vp, vp, vp, ctypes.c_float, vp, vp, i32, i32, i32, i32,
                                    ctypes.POINTER(KvSelectOpts), vp, vp, vp, vp, vp, vp, vp, sz,
                                    vp]
        h.kv_mmr_select.argtypes = [pr, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz,
                                    vp]
        h.kv_mmr_select_compact.argtypes = [pr, vp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp,
                                            vp, sz, vp]
        h.kv_mmr_select_ex.argtypes = [pr, vp, vp, vp, vp, vp, i32, i32, i32,
                                       ctypes.POINTER(KvSelectOpts), vp, vp, vp, vp, vp, sz, vp]
        h.kv_compact_cache.argtypes = [pr, vp, vp, vp, i32, i32, vp, vp, vp]
        h.kv_compact_cache_ex.argtypes = [pr, vp, vp, vp, i32, i32, vp, vp, i32, vp, vp, vp]
        cb = ctypes.POINTER(KvCacheBatch)
        h.kv_decode_workspace_bytes.argtypes = [cb]
        h.kv_decode_workspace_bytes.restype = sz
        h.kv_decode_attention.argtypes = [cb, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
        pc, i64 = ctypes.POINTER(KvPagedCache), ctypes.c_int64
        h.kv_paged_tables.argtypes = [pc, vp, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp]
        h.kv_paged_append.argtypes = [pc, vp, vp, i64, vp, i32, vp]
        h.kv_paged_compact.argtypes = [pr, vp, vp, vp, i32, i32, vp, vp, pc, vp]
        h.kv_paged_attention_workspace_bytes.argtypes = [pc, i32, i32]
        h.kv_paged_attention_workspace_bytes.restype = sz
        h.kv_paged_attention.argtypes = [pc, vp, i64, vp, i32, i32, ctypes.c_float, vp, vp, sz, vp]
        ro = ctypes.POINTER(KvRotary)
        h.kv_rotate.argtypes = [ro, i32, i32, i32, vp, i64, vp, i32, vp, i64, vp]
        h.kv_paged_append_rotated.argtypes = [pc, ro, vp, vp, i64, vp, i64, vp, vp, i64, vp, i32, vp]
        h.kv_paged_rows.argtypes = [pc, vp, i64, vp, vp, vp]
        h.kv_rotary_frequencies.argtypes = [i32, ctypes.c_double, ctypes.POINTER(ctypes.c_double), i32, i32,
                                            ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_float)]
        h.kv_pyramid_budgets.argtypes = [i32, i32, ctypes.c_double, ctypes.POINTER(ctypes.c_int32)]
        h.kv_depth_profile.argtypes = [i32, ctypes.POINTER(ctypes.c_double), i32, i32,
                                       ctypes.POINTER(ctypes.c_float)]
        for name in ("kv_window_scores", "kv_mu_sigma", "kv_mu_sigma_ex", "kv_window_mu_sigma",
                     "kv_window_mu_sigma_ex", "kv_window_mu_sigma_noalloc",
                     "kv_window_base_scores", "kv_mmr_select", "kv_mmr_select_ex",
                     "kv_mmr_select_scored", "kv_window_candidates", "kv_mmr_select_candidates",
                     "kv_evict_pass", "kv_compact_cache", "kv_compact_cache_ex", "kv_decode_attention",
                     "kv_paged_tables", "kv_paged_append", "kv_paged_compact", "kv_paged_attention",
                     "kv_rotate", "kv_paged_append_rotated", "kv_paged_rows", "kv_rotary_frequencies",
                     "kv_pyramid_budgets", "kv_depth_profile"):
            getattr(h, name).restype = ctypes.c_int
        _LIB = h
    return _LIB


def strerror(status: int) -> str:
    return lib().kv_strerror(int(status)).decode()


def version() -> int:
    return int(lib().kv_version())


def _check(status: int, where: str) -> None:
    if status != KV_OK:
        raise KvError(status, where)


class Batch:
    """Shape of a batch of problems (one problem = one layer of one sequence).

    Holds the host lengths/offsets and their device copies and exposes the kv_problem struct.
    """

    def __init__(self, dtype: str, h_q: int, h_kv: int, d: int, w: int, lens: Sequence[int],
                 tok_off: Optional[Sequence[int]] = None, device=None):
        import torch
        self.dtype_name = dtype
        self.h_q, self.h_kv, self.d, self.w = int(h_q), int(h_kv), int(d), int(w)
        self.lens_host = np.ascontiguousarray(np.asarray(lens, dtype=np.int32))
        if tok_off is None:
            off = np.zeros(len(self.lens_host), dtype=np.int64)
            if len(off) > 1:
                off[1:] = np.cumsum(self.lens_host.astype(np.int64))[:-1]
        else:
            off = np.asarray(tok_off, dtype=np.int64)
        self.tok_off_host = np.ascontiguousarray(off)
        dev = torch.device("cuda") if device is None else torch.device(device)
        self.lens_dev = torch.from_numpy(self.lens_host).to(dev)
        self.tok_off_dev = torch.from_numpy(self.tok_off_host).to(dev)
        self.struct = KvProblem(KV_BF16 if dtype == "bf16" else KV_F32, len(self.lens_host),
                                self.h_q, self.h_kv, self.d, self.w,
                                self.lens_host.ctypes.data, self.tok_off_host.ctypes.data,
                                self.lens_dev.data_ptr(), self.tok_off_dev.data_ptr())

    @property
    def n_prob(self) -> int:
        return len(self.lens_host)

    @property
    def total_tokens(self) -> int:
        return int(self.lens_host.astype(np.int64).sum())

    def ref(self):
        return ctypes.byref(self.struct)


class Budgets:
    """Per-problem budgets B_p: the host values and their device copy (budget_host / budget_dev of
    kv_select_opts and kv_compact_cache_ex)."""

    def __init__(self, values: Sequence[int], device=None):
        import torch
        self.host = np.ascontiguousarray(np.asarray(values, dtype=np.int32))
        dev = torch.device("cuda") if device is None else torch.device(device)
        self.dev = torch.from_numpy(self.host).to(dev)

    @property
    def max(self) -> int:
        return int(self.host.max())

    def pointers(self):
        return ctypes.c_void_p(self.host.ctypes.data), ctypes.c_void_p(self.dev.data_ptr())


def _ptr(t) -> ctypes.c_void_p:
    if t is None:
        return ctypes.c_void_p(0)
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous device tensors")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def workspace_bytes(batch: Batch, budget: int, cand_mult: int = 4,
                    keep_tail: Optional[int] = None) -> int:
    tail = batch.w if keep_tail is None else keep_tail
    return int(lib().kv_workspace_bytes(batch.ref(), budget, cand_mult, tail))


def candidate_stride(batch: Batch, budget: int, cand_mult: int = 4,
                     keep_tail: Optional[int] = None) -> int:
    tail = batch.w if keep_tail is None else keep_tail
    return int(lib().kv_candidate_stride(batch.ref(), budget, cand_mult, tail))


def window_scores(batch: Batch, q_win, k, scale: float, row_max, row_sum, ws,
                  stream=None) -> None:
    _check(lib().kv_window_scores(batch.ref(), _ptr(q_win), _ptr(k), float(scale), _ptr(row_max),
                                  _ptr(row_sum), _ptr(ws), 0 if ws is None else ws.numel() *
                                  ws.element_size(), _stream(stream)), "kv_window_scores")


def mu_sigma(batch: Batch, q_win, k, scale: float, row_max, row_sum, mu, sigma, attn=None,
             stream=None) -> None:
    _check(lib().kv_mu_sigma(batch.ref(), _ptr(q_win), _ptr(k), float(scale), _ptr(row_max),
                             _ptr(row_sum), _ptr(mu), _ptr(sigma), _ptr(attn), _stream(stream)),
           "kv_mu_sigma")


def window_mu_sigma(batch: Batch, q_win, k, scale: float, row_max, row_sum, mu, sigma, ws,
                    stream=None) -> None:
    _check(lib().kv_window_mu_sigma(batch.ref(), _ptr(q_win), _ptr(k), float(scale),
                                    _ptr(row_max), _ptr(row_sum), _ptr(mu), _ptr(sigma), _ptr(ws),
                                    0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream(stream)), "kv_window_mu_sigma")


def _sigma_rows(sigma_rows) -> int:
    return SIGMA_ROWS[sigma_rows] if isinstance(sigma_rows, str) else int(sigma_rows)


def mu_sigma_ex(batch: Batch, q_win, k, scale: float, row_max, row_sum, sigma_rows, mu, sigma,
                attn=None, stream=None) -> None:
    """kv_mu_sigma_ex; sigma_rows is "group_mean", "all_rows" or a KV_SIGMA_* value."""
    _check(lib().kv_mu_sigma_ex(batch.ref(), _ptr(q_win), _ptr(k), float(scale), _ptr(row_max),
                                _ptr(row_sum), _sigma_rows(sigma_rows), _ptr(mu), _ptr(sigma),
                                _ptr(attn), _stream(stream)), "kv_mu_sigma_ex")


def window_mu_sigma_ex(batch: Batch, q_win, k, scale: float, sigma_rows, row_max, row_sum, mu,
                       sigma, ws, stream=None) -> None:
    """kv_window_mu_sigma_ex; sigma_rows is "group_mean", "all_rows" or a KV_SIGMA_* value."""
    _check(lib().kv_window_mu_sigma_ex(batch.ref(), _ptr(q_win), _ptr(k), float(scale),
                                       _sigma_rows(sigma_rows), _ptr(row_max), _ptr(row_sum),
                                       _ptr(mu), _ptr(sigma), _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(),
                                       _stream(stream)), "kv_window_mu_sigma_ex")


def window_mu_sigma_noalloc(batch: Batch, q_win, k, scale: float, row_max, row_sum, mu, sigma,
                            sigma_rows="group_mean", stream=None) -> None:
    """kv_window_mu_sigma_noalloc (no workspace: the library's static scratch)."""
    _check(lib().kv_window_mu_sigma_noalloc(batch.ref(), _ptr(q_win), _ptr(k), float(scale),
                                            _sigma_rows(sigma_rows), _ptr(row_max),
                                            _ptr(row_sum), _ptr(mu), _ptr(sigma),
                                            _stream(stream)), "kv_window_mu_sigma_noalloc")


def base_scores_workspace_bytes(batch: Batch) -> int:
    return int(lib().kv_base_scores_workspace_bytes(batch.ref()))


def window_base_scores(batch: Batch, q_win, k, scale: float, lambda1, row_max, row_sum, score,
                       w_mu: float = 1.0, sigma_rows="group_mean", ws=None, stream=None) -> None:
    """kv_window_base_scores."""
    _check(lib().kv_window_base_scores(batch.ref(), _ptr(q_win), _ptr(k), float(scale),
                                       _ptr(lambda1), float(w_mu), _sigma_rows(sigma_rows),
                                       _ptr(row_max), _ptr(row_sum), _ptr(score), _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(),
                                       _stream(stream)), "kv_window_base_scores")


def _select_opts(pool, w_mu, budgets):
    if pool is None and w_mu is None and budgets is None:
        return None
    bh, bd = budgets.pointers() if budgets is not None else (None, None)
    return ctypes.byref(KvSelectOpts(1 if pool is None else int(pool),
                                     1.0 if w_mu is None else float(w_mu), bh, bd))


def mmr_select_scored(batch: Batch, score, k, v, lambda2, budget: int, cand_mult: int,
                      keep_tail: int, sel_idx, sel_score=None, cand_idx=None, cand_corr=None,
                      k_out=None, v_out=None, pool: Optional[int] = None,
                      budgets: Optional[Budgets] = None, stream=None) -> None:
    """kv_mmr_select_scored; with k_out / v_out the compaction runs in the same launch."""
    _check(lib().kv_mmr_select_scored(batch.ref(), _ptr(score), _ptr(k), _ptr(v), _ptr(lambda2),
                                      int(budget), int(cand_mult),
                                      int(keep_tail), _select_opts(pool, None, budgets),
                                      _ptr(sel_idx), _ptr(sel_score), _ptr(cand_idx),
                                      _ptr(cand_corr), _ptr(k_out), _ptr(v_out),
                                      _stream(stream)), "kv_mmr_select_scored")


def candidates_workspace_bytes(batch: Batch, budget: int, cand_mult: int, keep_tail: int,
                               w_mu: Optional[float] = None,
                               budgets: Optional[Budgets] = None) -> int:
    return int(lib().kv_candidates_workspace_bytes(batch.ref(), int(budget), int(cand_mult),
                                                   int(keep_tail),
                                                   _select_opts(None, w_mu, budgets)))


def window_candidates(batch: Batch, q_win, k, scale: float, lambda1, budget: int, cand_mult: int,
                      keep_tail: int, row_max, row_sum, ws, w_mu: Optional[float] = None,
                      budgets: Optional[Budgets] = None, sigma_rows="group_mean",
                      stream=None) -> None:
    """kv_window_candidates: row statistics out, the candidates into ws (see
    candidates_workspace_bytes) for mmr_select_candidates with the same selection arguments."""
    _check(lib().kv_window_candidates(batch.ref(), _ptr(q_win), _ptr(k), float(scale),
                                      _ptr(lambda1), _sigma_rows(sigma_rows), int(budget),
                                      int(cand_mult), int(keep_tail),
                                      _select_opts(None, w_mu, budgets), _ptr(row_max),
                                      _ptr(row_sum), _ptr(ws),
                                      0 if ws is None else ws.numel() * ws.element_size(),
                                      _stream(stream)), "kv_window_candidates")


def mmr_select_candidates(batch: Batch, ws, k, v, lambda2, budget: int, cand_mult: int,
                          keep_tail: int, sel_idx, sel_score=None, cand_idx=None, cand_corr=None,
                          k_out=None, v_out=None, w_mu: Optional[float] = None,
                          budgets: Optional[Budgets] = None, stream=None) -> None:
    """kv_mmr_select_candidates; with k_out / v_out the compaction runs in the same launch."""
    _check(lib().kv_mmr_select_candidates(batch.ref(), _ptr(ws),
                                          0 if ws is None else ws.numel() * ws.element_size(),
                                          _ptr(k), _ptr(v), _ptr(lambda2), int(budget),
                                          int(cand_mult), int(keep_tail),
                                          _select_opts(None, w_mu, budgets), _ptr(sel_idx),
                                          _ptr(sel_score), _ptr(cand_idx), _ptr(cand_corr),
                                          _ptr(k_out), _ptr(v_out), _stream(stream)),
           "kv_mmr_select_candidates")


def evict_pass(batch: Batch, q_win, k, v, scale: float, lambda1, lambda2, budget: int,
               cand_mult: int, keep_tail: int, row_max, row_sum, sel_idx, ws, sel_score=None,
               k_out=None, v_out=None, w_mu: Optional[float] = None,
               budgets: Optional[Budgets] = None, sigma_rows="group_mean", stream=None) -> None:
    """kv_evict_pass: window_candidates then mmr_select_candidates (with k_out / v_out the
    compaction), in one launch where the window kernel cuts the candidates and C <= 256."""
    _check(lib().kv_evict_pass(batch.ref(), _ptr(q_win), _ptr(k), _ptr(v), float(scale),
                               _ptr(lambda1), _ptr(lambda2), _sigma_rows(sigma_rows), int(budget),
                               int(cand_mult), int(keep_tail), _select_opts(None, w_mu, budgets),
                               _ptr(row_max), _ptr(row_sum), _ptr(sel_idx), _ptr(sel_score),
                               _ptr(k_out), _ptr(v_out), _ptr(ws),
                               0 if ws is None else ws.numel() * ws.element_size(),
                               _stream(stream)), "kv_evict_pass")


def mmr_select(batch: Batch, mu, sigma, k, lambda1, lambda2, budget: int, cand_mult: int,
               keep_tail: int, sel_idx, sel_score=None, cand_idx=None, cand_corr=None, ws=None,
               stream=None) -> None:
    _check(lib().kv_mmr_select(batch.ref(), _ptr(mu), _ptr(sigma), _ptr(k), _ptr(lambda1),
                               _ptr(lambda2), int(budget), int(cand_mult), int(keep_tail),
                               _ptr(sel_idx), _ptr(sel_score), _ptr(cand_idx), _ptr(cand_corr),
                               _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                               _stream(stream)), "kv_mmr_select")


def mmr_select_compact(batch: Batch, mu, sigma, k, v, lambda1, lambda2, budget: int,
                       cand_mult: int, keep_tail: int, sel_idx, k_out, v_out, ws=None,
                       stream=None) -> None:
    _check(lib().kv_mmr_select_compact(batch.ref(), _ptr(mu), _ptr(sigma), _ptr(k), _ptr(v),
                                       _ptr(lambda1), _ptr(lambda2), int(budget), int(cand_mult),
                                       int(keep_tail), _ptr(sel_idx), _ptr(k_out), _ptr(v_out),
                                       _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                       _stream(stream)), "kv_mmr_select_compact")


def mmr_select_ex(batch: Batch, mu, sigma, k, lambda1, lambda2, budget: int, cand_mult: int,
                  keep_tail: int, sel_idx, sel_score=None, cand_idx=None, cand_corr=None, ws=None,
                  pool: Optional[int] = None, w_mu: Optional[float] = None,
                  budgets: Optional[Budgets] = None, stream=None) -> None:
    """kv_mmr_select_ex; options are passed as NULL when pool, w_mu and budgets are all None.
    With `budgets`, `budget` is the row stride of sel_idx / sel_score."""
    opts = _select_opts(pool, w_mu, budgets)
    _check(lib().kv_mmr_select_ex(batch.ref(), _ptr(mu), _ptr(sigma), _ptr(k), _ptr(lambda1),
                                  _ptr(lambda2), int(budget), int(cand_mult), int(keep_tail), opts,
                                  _ptr(sel_idx), _ptr(sel_score), _ptr(cand_idx),
                                  _ptr(cand_corr), _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(),
                                  _stream(stream)), "kv_mmr_select_ex")


def compact_cache(batch: Batch, k, v, sel_idx, budget: int, keep_tail: int, k_out, v_out,
                  stream=None) -> None:
    _check(lib().kv_compact_cache(batch.ref(), _ptr(k), _ptr(v), _ptr(sel_idx), int(budget),
                                  int(keep_tail), _ptr(k_out), _ptr(v_out), _stream(stream)),
           "kv_compact_cache")


def compact_cache_ex(batch: Batch, k, v, sel_idx, budget: int, keep_tail: int,
                     budgets: Optional[Budgets], k_out, v_out, out_rows: int = 0,
                     stream=None) -> None:
    bh, bd = budgets.pointers() if budgets is not None else (None, None)
    _check(lib().kv_compact_cache_ex(batch.ref(), _ptr(k), _ptr(v), _ptr(sel_idx), int(budget),
                                     int(keep_tail), bh, bd, int(out_rows), _ptr(k_out),
                                     _ptr(v_out), _stream(stream)), "kv_compact_cache_ex")


class CacheBatch:
    """Shape of a batch of caches for decoding (kv_cache_batch): per-problem lengths on the host
    and the device.  `advance()` adds one row to every length (after a call that appended)."""

    def __init__(self, dtype: str, h_q: int, h_kv: int, d: int, row_stride: int,
                 lens: Sequence[int], device=None):
        import torch
        self.dtype_name = dtype
        self.h_q, self.h_kv, self.d, self.row_stride = int(h_q), int(h_kv), int(d), int(row_stride)
        self.lens_host = np.ascontiguousarray(np.asarray(lens, dtype=np.int32))
        self._dev = torch.device("cuda") if device is None else torch.device(device)
        self._sync()

    def _sync(self):
        import torch
        self.lens_dev = torch.from_numpy(self.lens_host).to(self._dev)
        self.struct = KvCacheBatch(KV_BF16 if self.dtype_name == "bf16" else KV_F32,
                                   len(self.lens_host), self.h_q, self.h_kv, self.d,
                                   self.row_stride, self.lens_host.ctypes.data,
                                   self.lens_dev.data_ptr())

    def advance(self):
        self.lens_host = self.lens_host + 1
        self._sync()

    @property
    def n_prob(self) -> int:
        return len(self.lens_host)

    def ref(self):
        return ctypes.byref(self.struct)


def decode_workspace_bytes(cb: CacheBatch) -> int:
    return int(lib().kv_decode_workspace_bytes(cb.ref()))


def decode_attention(cb: CacheBatch, q, k_cache, v_cache, k_new, v_new, scale: float, out,
                     ws=None, stream=None) -> None:
    _check(lib().kv_decode_attention(cb.ref(), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_new),
                                     _ptr(v_new), float(scale), _ptr(out), _ptr(ws),
                                     0 if ws is None else ws.numel() * ws.element_size(),
                                     _stream(stream)), "kv_decode_attention")


def _place(index: int) -> str:
    """A device by its index, for what is said to the caller (below 0: that of an object on the host)."""
    return f"cuda:{index}" if index >= 0 else "a GPU"


def _token_rows(t, dtype, index: int, heads: int, d: int, name: str):
    """Address and token stride of [tokens, heads, d] rows on device `index`; tokens may lie apart (slices of a
    projection)."""
    n, h, e = t.shape if t.dim() == 3 else (0, -1, -1)
    if h != heads or e != d or t.dtype is not dtype or t.get_device() != index:
        raise ValueError(f"{name} must be a {dtype} tensor [tokens, {heads}, {d}] on {_place(index)}")
    apart, between, one = t.stride()
    if one != 1 or (between != d and heads > 1):
        raise ValueError(f"the heads of a token must be contiguous in {name}")
    if n <= 1:
        return t.data_ptr(), heads * d
    if apart < heads * d:
        raise ValueError(f"the tokens overlap in {name}")
    return t.data_ptr(), apart


def _flat(t, dtype, index: int, n: int, name: str):
    """Address of a contiguous tensor of at least n elements on device `index`."""
    if t.dtype is not dtype or t.get_device() != index or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of at least {n} elements on {_place(index)}")
    return t.data_ptr()


class _OnDevice:
    """What launches on a device of its own."""

    def _on(self, device):
        import torch
        self.device = device
        self._index = device.index if device.type == "cuda" else -2  # (no tensor is on it)
        self._int32, self._int64 = torch.int32, torch.int64
        # the queries under torch.cuda's where this torch has them (torch.cuda.current_stream() makes an object of
        # the stream: 3 us of a call of 9)
        self._current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                                   lambda index: torch.cuda.current_stream(index).cuda_stream)

    def _stream(self, stream):
        """The stream to launch on: kernels go to the current device, which has to be the tensors'."""
        index = self._index
        if index != self._current_device():
            raise ValueError(f"the {self._what} is on {self.device}, which is not the current device")
        return self._raw_stream(index) if stream is None else stream.cuda_stream


_FOUR_BITS = "float4_e2m1fn_x2"


def _code_types():
    """The types of a paged cache's codes, those of 4 bits where this torch has them."""
    import torch
    types = {torch.float8_e4m3fn: KV_E4M3, torch.int8: KV_INT8}
    if hasattr(torch, _FOUR_BITS):
        types[getattr(torch, _FOUR_BITS)] = KV_E2M1
    return types


class PagedCache(_OnDevice):
    """A batch of 8- or 4-bit caches in shared blocks (kv_paged_cache), around the caller's device tensors:
    k, v [n_blocks, h_kv, block_rows, d] (torch.float8_e4m3fn or int8), k_scale, v_scale
    [n_blocks, h_kv] fp32, table [n_prob, table_stride] int32 and lens [n_prob] int32.  4 bits: k, v
    [n_blocks, h_kv, block_rows, d / 2] torch.float4_e2m1fn_x2, scales [n_blocks, h_kv, d / 32, block_rows]
    torch.float8_e8m0fnu.  dtype ("bf16" or "f32") is that of queries, new rows and outputs; max_len bounds the
    lengths (default: what the table holds)."""

    _what = "cache"

    def __init__(self, dtype: str, h_q: int, k, v, k_scale, v_scale, table, lens,
                 max_len: Optional[int] = None):
        import torch
        n_blocks, h_kv, block_rows, d = k.shape
        qtype = _code_types().get(k.dtype)
        if qtype is None or v.dtype != k.dtype or v.shape != k.shape:
            raise ValueError("k and v must be float8_e4m3fn, int8 or float4_e2m1fn_x2 tensors of one shape")
        n_scales, scales = n_blocks * h_kv, torch.float32
        if qtype == KV_E2M1:
            d *= 2
            n_scales, scales = n_scales * (d // 32) * block_rows, torch.float8_e8m0fnu
        if dtype not in ("bf16", "f32"):
            raise ValueError("dtype must be bf16 or f32")
        self._tables(table, lens, n_blocks, block_rows)
        self.dtype_name = dtype
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.rows_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        s = self.struct
        s.dtype = KV_BF16 if dtype == "bf16" else KV_F32
        s.qtype = qtype
        s.h_q, s.h_kv, s.d = self.h_q, self.h_kv, self.d = int(h_q), h_kv, d
        s.max_len = min(table.shape[1] * block_rows, 1 << 24) if max_len is None else int(max_len)
        s.k, s.v = self._arg(k, k.dtype, 0, "k"), self._arg(v, k.dtype, 0, "v")
        s.k_scale = self._arg(k_scale, scales, n_scales, "k_scale")
        s.v_scale = self._arg(v_scale, scales, n_scales, "v_scale")

    def _tables(self, table, lens, n_blocks, block_rows):
        import torch
        if table.dim() != 2 or lens.numel() != table.shape[0]:
            raise ValueError("table must be [n_prob, table_stride] and lens [n_prob]")
        self.table, self.lens = table, lens
        self._on(table.device)
        self.n_prob = table.shape[0]
        self.struct = KvPagedCache(n_prob=self.n_prob, block_rows=int(block_rows), n_blocks=int(n_blocks),
                                   table_stride=table.shape[1], table=self._arg(table, torch.int32, 0, "table"),
                                   len=self._arg(lens, torch.int32, 0, "lens"))
        self._ref = ctypes.byref(self.struct)

    @classmethod
    def for_tables(cls, block_rows: int, n_blocks: int, table, lens) -> "PagedCache":
        """A cache without pools: what paged_tables needs."""
        self = cls.__new__(cls)
        self._tables(table, lens, n_blocks, block_rows)
        return self

    @classmethod
    def allocate(cls, dtype: str, qtype: str, h_q: int, h_kv: int, d: int, block_rows: int, n_blocks: int,
                 n_prob: int, table_stride: int, max_len: Optional[int] = None, device=None) -> "PagedCache":
        """Empty pools (their contents are undefined) of qtype "e4m3", "int8" or "e2m1", a table of missing blocks and
        lengths of 0."""
        import torch
        dev = torch.device("cuda") if device is None else torch.device(device)
        four = qtype == "e2m1"
        if four and not hasattr(torch, _FOUR_BITS):
            raise ValueError(f"4-bit caches need a torch that has {_FOUR_BITS}")
        qt = getattr(torch, {"e4m3": "float8_e4m3fn", "int8": "int8", "e2m1": _FOUR_BITS}[qtype])
        pool = lambda: torch.empty(n_blocks, h_kv, block_rows, d // 2 if four else d, dtype=torch.uint8, device=dev).view(qt)
        scales = lambda: (torch.empty(n_blocks, h_kv, d // 32, block_rows, dtype=torch.uint8, device=dev)
                          .view(torch.float8_e8m0fnu) if four else
                          torch.empty(n_blocks, h_kv, dtype=torch.float32, device=dev))
        return cls(dtype, h_q, pool(), pool(), scales(), scales(),
                   torch.full((n_prob, table_stride), -1, dtype=torch.int32, device=dev),
                   torch.zeros(n_prob, dtype=torch.int32, device=dev), max_len)

    def ref(self):
        return self._ref

    def _arg(self, t, dtype, n: int, name: str):
        """Address of a contiguous tensor of at least n elements on the cache's device (None: NULL)."""
        return None if t is None else _flat(t, dtype, self._index, n, name)

    def _rows(self, t, heads: int, name: str):
        return _token_rows(t, self.rows_dtype, self._index, heads, self.d, name)


def paged_tables(pc: PagedCache, len_in, add, free_blocks, taken_in, taken_out, tok_off, blk_off, slots,
                 n_free: Optional[int] = None, stream=None) -> None:
    """kv_paged_tables: writes pc.table, pc.lens, tok_off, blk_off [n_prob + 1], slots and taken_out.
    len_in None: empty caches; add None: one row each; free_blocks None: n_free blocks 0, 1, 2, ..
    (default: the pool's)."""
    n, i32, arg = pc.n_prob, pc._int32, pc._arg
    if free_blocks is not None:
        n_free = free_blocks.numel() if n_free is None else min(int(n_free), free_blocks.numel())
    elif n_free is None:
        n_free = pc.struct.n_blocks
    _check(lib().kv_paged_tables(pc._ref, arg(len_in, i32, n, "len_in"), arg(add, i32, n, "add"),
                                 arg(free_blocks, i32, 0, "free_blocks"), int(n_free),
                                 arg(taken_in, i32, 1, "taken_in"), arg(taken_out, i32, 1, "taken_out"),
                                 arg(tok_off, i32, n + 1, "tok_off"), arg(blk_off, i32, n + 1, "blk_off"),
                                 arg(slots, i32, 0, "slots"), 0 if slots is None else slots.numel(),
                                 pc._stream(stream)), "kv_paged_tables")


def paged_append(pc: PagedCache, k_new, v_new, slots, stream=None) -> None:
    """kv_paged_append: k_new, v_new [tokens, h_kv, d], tokens of one stride (slices of a projection's
    output, for instance); slots [tokens] int32.  No tokens: nothing to do."""
    kp, ks = pc._rows(k_new, pc.h_kv, "k_new")
    vp, vs = pc._rows(v_new, pc.h_kv, "v_new")
    n = k_new.shape[0]
    if v_new.shape[0] != n or ks != vs:
        raise ValueError("k_new and v_new must have one shape and token stride")
    sp, st = pc._arg(slots, pc._int32, n, "slots"), pc._stream(stream)
    if n:
        _check(lib().kv_paged_append(pc._ref, kp, vp, ks, sp, n, st), "kv_paged_append")


class Rotary(_OnDevice):
    """A rotation by positions (kv_rotary): layout "half" or "interleaved", freq [rot_dim / 2] float64 on the device (radians a
    position; rotary_frequencies gives them), the factor of the rotated elements, and whether it turns back."""

    _what = "rotation"

    def __init__(self, layout: str, freq, factor: float = 1.0, inverse: bool = False):
        import torch
        if layout not in ROTARY_LAYOUTS:
            raise ValueError("layout must be half or interleaved")
        if freq.dtype is not torch.float64 or not freq.is_cuda or not freq.is_contiguous() or freq.dim() != 1:
            raise ValueError("freq must be a contiguous float64 device tensor [rot_dim / 2]")
        self.freq = freq
        self._on(freq.device)
        self._codes = {torch.bfloat16: KV_BF16, torch.float32: KV_F32}
        self.struct = KvRotary(ROTARY_LAYOUTS[layout], 2 * freq.numel(), int(bool(inverse)), float(factor), freq.data_ptr())
        self._ref = ctypes.byref(self.struct)

    def ref(self):
        return self._ref


def rotary_frequencies(family: str, rot_dim: int, base: float = 10000.0, params: Sequence[float] = ()):
    """-> (frequencies [rot_dim / 2] float64, factor) of a family "plain", "linear" (F), "ntk" (F), "yarn" (F, L0,
    beta_fast, beta_slow) or "bands" (F, L0, low, high)."""
    fam = ROTARY_FAMILIES[family] if isinstance(family, str) else int(family)
    p = (ctypes.c_double * len(params))(*[float(x) for x in params])
    out, factor = (ctypes.c_double * max(1, int(rot_dim) // 2))(), ctypes.c_float()
    _check(lib().kv_rotary_frequencies(fam, float(base), p, len(params), int(rot_dim), out, ctypes.byref(factor)),
           "kv_rotary_frequencies")
    return np.frombuffer(out, dtype=np.float64).copy(), float(factor.value)


def rotate(rot: Rotary, x, pos, out, stream=None) -> None:
    """kv_rotate: x [tokens, heads, d] bf16 or fp32 (tokens of one stride) at positions pos [tokens] int32, to out of the
    same shape and type, which may be x.  No tokens: nothing to do."""
    dtype, index = x.dtype, rot._index
    code = rot._codes.get(dtype)
    if code is None or x.dim() != 3:
        raise ValueError("x must be a bfloat16 or float32 tensor [tokens, heads, d]")
    n, heads, d = x.shape
    xp, xs = _token_rows(x, dtype, index, heads, d, "x")
    op, os_ = _token_rows(out, dtype, index, heads, d, "out")
    if out.shape[0] != n:
        raise ValueError("out must have the shape of x")
    pp, st = _flat(pos, rot._int32, index, n, "pos"), rot._stream(stream)
    if n:
        _check(lib().kv_rotate(rot._ref, code, heads, d, xp, xs, pp, n, op, os_, st), "kv_rotate")


def paged_append_rotated(pc: PagedCache, rot: Rotary, pos, k_new, v_new, slots, q=None, q_out=None, stream=None) -> None:
    """kv_paged_append_rotated: paged_append with k_new rotated to positions pos [tokens] int32 on the way, and with q
    [tokens, h_q, d] its rotation in q_out (which may be q).  No tokens: nothing to do."""
    kp, ks = pc._rows(k_new, pc.h_kv, "k_new")
    vp, vs = pc._rows(v_new, pc.h_kv, "v_new")
    n = k_new.shape[0]
    if v_new.shape[0] != n or ks != vs:
        raise ValueError("k_new and v_new must have one shape and token stride")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    qp, qs, op, os_ = None, 0, None, 0
    if q is not None:
        qp, qs = pc._rows(q, pc.h_q, "q")
        op, os_ = pc._rows(q_out, pc.h_q, "q_out")
        if q.shape[0] != n or q_out.shape[0] != n:
            raise ValueError("q and q_out must have as many tokens as k_new")
    if rot._index != pc._index:
        raise ValueError(f"the rotation is on {rot.device}, the cache on {pc.device}")
    pp, sp, st = pc._arg(pos, pc._int32, n, "pos"), pc._arg(slots, pc._int32, n, "slots"), pc._stream(stream)
    if n:
        _check(lib().kv_paged_append_rotated(pc._ref, rot._ref, pp, qp, qs, op, os_, kp, vp, ks, sp, n, st),
               "kv_paged_append_rotated")


def paged_rows(pc: PagedCache, row_off, k_out, v_out, n_rows: Optional[int] = None, stream=None) -> None:
    """kv_paged_rows: the rows of every problem p into k_out and v_out (either may be None) at row_off[p] h_kv d elements,
    [h_kv][row_off[p + 1] - row_off[p]][d]; row_off [n_prob + 1] int64.  n_rows: the rows that the outputs hold (default:
    all)."""
    unit = pc.h_kv * pc.d
    held = [t.numel() // unit for t in (k_out, v_out) if t is not None]
    if not held:
        raise ValueError("one of k_out and v_out is needed")
    n_rows = min(held) if n_rows is None else int(n_rows)
    kp = pc._arg(k_out, pc.rows_dtype, n_rows * unit, "k_out")
    vp = pc._arg(v_out, pc.rows_dtype, n_rows * unit, "v_out")
    op, st = pc._arg(row_off, pc._int64, pc.n_prob + 1, "row_off"), pc._stream(stream)
    if n_rows:
        _check(lib().kv_paged_rows(pc._ref, op, n_rows, kp, vp, st), "kv_paged_rows")


def paged_compact(batch: Batch, k, v, sel_idx, budget: int, keep_tail: int, pc: PagedCache,
                  budgets: Optional[Budgets] = None, stream=None) -> None:
    """kv_paged_compact: the selected rows of k and v and the tail into pc's blocks."""
    bh, bd = budgets.pointers() if budgets is not None else (None, None)
    n = batch.total_tokens * batch.h_kv * batch.d
    _check(lib().kv_paged_compact(batch.ref(), pc._arg(k, pc.rows_dtype, n, "k"), pc._arg(v, pc.rows_dtype, n, "v"),
                                  pc._arg(sel_idx, pc._int32, batch.n_prob * batch.h_kv * int(budget), "sel_idx"),
                                  int(budget), int(keep_tail), bh, bd, pc._ref, pc._stream(stream)),
           "kv_paged_compact")


def paged_attention_workspace_bytes(pc: PagedCache, n_tok: Optional[int] = None, max_q: int = 1) -> int:
    n_tok = pc.n_prob if n_tok is None else n_tok
    return int(lib().kv_paged_attention_workspace_bytes(pc._ref, int(n_tok), int(max_q)))


def paged_attention(pc: PagedCache, q, scale: float, out, tok_off=None, max_q: int = 1, ws=None,
                    stream=None) -> None:
    """kv_paged_attention: q [tokens, h_q, d] (tokens of one stride), out the same shape, contiguous;
    tok_off [n_prob + 1] int32 for several tokens to a problem, at most max_q each.  With tok_off no tokens
    at all are nothing to do."""
    qp, qs = pc._rows(q, pc.h_q, "q")
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    n, off, op = q.shape[0], pc._arg(tok_off, pc._int32, pc.n_prob + 1, "tok_off"), pc._arg(out, pc.rows_dtype, 0, "out")
    wp, st = None if ws is None else pc._arg(ws, ws.dtype, 0, "ws"), pc._stream(stream)
    if n or off is None:
        _check(lib().kv_paged_attention(pc._ref, qp, qs, off, n, max_q, scale, op, wp,
                                        0 if ws is None else ws.numel() * ws.element_size(), st), "kv_paged_attention")


def pyramid_budgets(budget: int, n_layers: int, beta: float) -> np.ndarray:
    """Depth-decreasing per-layer budgets at the total of a uniform `budget` (int32)."""
    out = (ctypes.c_int32 * n_layers)()
    _check(lib().kv_pyramid_budgets(int(budget), int(n_layers), float(beta), out),
           "kv_pyramid_budgets")
    return np.frombuffer(out, dtype=np.int32).copy()


def depth_profile(family: str, params: Sequence[float], n_layers: int) -> np.ndarray:
    """lambda per layer (float32) from a Global / Segments / Curve latent profile."""
    fam = PROFILE_FAMILIES[family] if isinstance(family, str) else int(family)
    p = (ctypes.c_double * len(params))(*[float(x) for x in params])
    out = (ctypes.c_float * n_layers)()
    _check(lib().kv_depth_profile(fam, p, len(params), int(n_layers), out), "kv_depth_profile")
    return np.frombuffer(out, dtype=np.float32).copy()
