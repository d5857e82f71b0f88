"""Appending with the rotation on the way into 8-bit blocks (kv_paged_append_rotated), by the runs of tokens that fall to a
block: bit for bit what kv_rotate of fp32 rows gives, appended by the definition in float64 (oracle/paged.py).

Which kernel takes a call goes by its tokens to a request (up to four: runs taken by waves; more: by workgroups), so
every case has as many requests as its form needs.
"""
import numpy as np
import pytest

from oracle import paged
from paper_2609_30738_amd import _lib
from tests.test_gpu_paged import _dev, _dt, _host, _image, _pool, _rng, _rows, _same_image, _say

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "e4m3"), ("bf16", "int8"), ("f32", "e4m3"), ("f32", "int8")]


def _turned(r, x, pos):
    """x rotated by kv_rotate, as fp32 rows."""
    import torch
    out = torch.empty(x.shape, dtype=torch.float32, device="cuda")
    _lib.rotate(r, x.float().contiguous(), pos, out)
    return out


def _holding(rng, pc, scales):
    """Random codes that are numbers in every block, and its scale of every head one of `scales`."""
    import torch
    for pool, scale in ((pc.k, pc.k_scale), (pc.v, pc.v_scale)):
        pool.view(torch.uint8).copy_(_dev((rng.integers(0, 0x70, tuple(pool.shape)) + 128 * rng.integers(0, 2, tuple(pool.shape))).astype(np.uint8)))
        scale.copy_(_dev(rng.choice(np.asarray(scales, np.float32), tuple(scale.shape))))
    return pc


@pytest.mark.parametrize("dtype,qtype", TYPES)
@pytest.mark.parametrize("d,layout", [(128, "half"), (64, "interleaved")])
@pytest.mark.parametrize("n_prob,tokens", [(9, 1), (9, 3), (2, 20)])
def test_held_scales_at_the_ends(dtype, qtype, d, layout, n_prob, tokens):
    """Blocks whose rows in use have the largest power of two, 2^127, the smallest, 2^-126, ones between them or 0: new rows
    near fp32's largest number (whose rotation may be infinite), ordinary ones, zeros, an infinity and a NaN."""
    rng = _rng(n_prob, tokens, d, len(dtype))
    R, h_kv, held = 32, 3, 7
    n_blocks = n_prob + 2
    pc = _holding(rng, _lib.PagedCache.allocate(dtype, qtype, h_kv, h_kv, d, R, n_blocks, n_prob, 1),
                  [2.0 ** 127, 2.0 ** 126, 2.0 ** -126, 1.0, 0.0])
    f, factor = _lib.rotary_frequencies("plain", d // 2)
    r = _lib.Rotary(layout, _dev(f), factor)
    blocks, T = rng.permutation(n_blocks)[:n_prob], n_prob * tokens
    slots = (blocks[:, None] * R + held + np.arange(tokens)).reshape(-1).astype(np.int32)
    size = 2.0 ** rng.choice([126, 100, 0, -126], (T, h_kv, 1))
    k, v = (_dev((np.clip(rng.standard_normal((T, h_kv, d)), -3.9, 3.9) * size).astype(np.float32), _dt(dtype)) for _ in range(2))
    k[0, 0, 3], k[1, 1, 5], v[0, 1, 0], v[1, 0, 9], v[2, 2] = float("nan"), float("inf"), float("-inf"), float("nan"), 0
    pos = _dev(rng.integers(0, 9999, T).astype(np.int32))
    codes, scales = _image(pc)
    codes = [x.copy() for x in codes]
    _say("held scales", dtype, qtype, d, layout, n_prob, tokens)
    k32 = _turned(r, k, pos)
    _lib.paged_append_rotated(pc, r, pos, k, v, _dev(slots))
    for c, s, x in zip(codes, scales, (k32, v)):
        paged.append(c, s, _host(x), slots, qtype)
    _same_image(pc, codes, scales, "held scales")


def _few(rng, n):
    """Up to four rows a request."""
    return rng.integers(0, 5, n)


def _one_long(rng, n):
    """One request of many rows among single and empty ones."""
    adds = rng.integers(0, 2, n)
    adds[n // 3] = 2 * n
    return adds


def _one_each(rng, n):
    return np.ones(n, int)


def _appended(rng, dtype, qtype, d, R, layout, rot, counts, n_prob, h_kv, odd=False):
    """Three calls of up to four tokens a request on average, behind what the last ones left: codes and scales as defined,
    the queries of two of them as kv_rotate's."""
    import torch
    steps = [counts(rng, n_prob) for _ in range(3)]
    rows = np.sum(steps, 0)
    stride = int(rows.max()) // R + 1
    n_blocks = int((rows // R + 1).sum()) + 3
    pc = _pool(_lib.PagedCache.allocate(dtype, qtype, 2 * h_kv, h_kv, d, R, n_blocks, n_prob, stride))
    ids, table, at = rng.permutation(n_blocks), [], 0
    for n in rows // R + 1:
        table.append(ids[at:at + n])
        at += n
    f, factor = _lib.rotary_frequencies("bands", rot, 1e4, (8.0, 8192.0, 1.0, 4.0))
    r = _lib.Rotary(layout, _dev(f), factor)
    codes, scales = _image(pc)
    codes, held = [x.copy() for x in codes], np.zeros(n_prob, int)
    for step, adds in enumerate(steps):
        slots = [table[p][i // R] * R + i % R for p in range(n_prob) for i in range(held[p], held[p] + adds[p])]
        slots += [-1, n_blocks * R] if step == 1 and len(slots) + 2 <= 4 * n_prob else []
        T = len(slots)
        assert T <= 4 * n_prob
        qkv = _rows(rng, T, 4 * h_kv, d, dtype) * 2.0 ** (3 * step)  # (scales that grow)
        if odd:
            for _ in range(6):
                qkv[rng.integers(T), rng.integers(2 * h_kv, 4 * h_kv), rng.integers(d)] = float(rng.choice([np.nan, np.inf, -np.inf]))
        q, k, v = qkv[:, :2 * h_kv], qkv[:, 2 * h_kv:3 * h_kv], qkv[:, 3 * h_kv:]
        pos = _dev(rng.integers(0, 1 << 20, T).astype(np.int32))
        want, k32 = torch.empty(q.shape, dtype=q.dtype, device="cuda"), _turned(r, k, pos)
        _lib.rotate(r, q, pos, want)
        q_out = torch.empty_like(want) if step != 1 else None
        _say("rotated runs", dtype, qtype, d, R, layout, rot, counts.__name__, n_prob, step, T)
        _lib.paged_append_rotated(pc, r, pos, k, v, _dev(np.asarray(slots, np.int32)), q=None if q_out is None else q, q_out=q_out)
        for c, s, x in zip(codes, scales, (k32, v)):
            paged.append(c, s, _host(x), np.asarray(slots), qtype)
        _same_image(pc, codes, scales, f"step {step}")
        assert q_out is None or torch.equal(q_out, want), step
        held += adds


@pytest.mark.parametrize("dtype,qtype", TYPES)
@pytest.mark.parametrize("d,layout,rot", [(128, "half", 128), (64, "interleaved", 64), (128, "interleaved", 48), (64, "half", 16)])
@pytest.mark.parametrize("R", [16, 32, 64, 128])
@pytest.mark.parametrize("counts,n_prob", [(_few, 5), (_few, 90), (_one_long, 40), (_one_long, 130)])
def test_runs_of_few_rows(dtype, qtype, d, layout, rot, R, counts, n_prob):
    """Runs of a few rows, and one of up to a block's among single ones: past a wave's tile (4 to 16 rows), over ends of
    blocks, behind rows whose scale grows, over several windows of 64 tokens."""
    _appended(_rng(R, d, rot, n_prob, len(dtype), 1), dtype, qtype, d, R, layout, rot, counts, n_prob, 2)


@pytest.mark.parametrize("dtype,qtype", TYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("counts,n_prob", [(_few, 60), (_one_long, 50)])
def test_runs_of_numbers_that_are_none(dtype, qtype, layout, counts, n_prob):
    """NaN and infinite elements in runs of all sizes."""
    _appended(_rng(n_prob, len(dtype), 2), dtype, qtype, 64, 64, layout, 32, counts, n_prob, 2, odd=True)


@pytest.mark.parametrize("dtype,qtype", TYPES)
@pytest.mark.parametrize("R,h_kv", [(16, 1), (128, 3)])
def test_one_row_of_many_requests(dtype, qtype, R, h_kv):
    """More requests than a workgroup each: every workgroup takes several, the last window is not full."""
    _appended(_rng(R, h_kv, len(dtype), 3), dtype, qtype, 64, R, "half", 64, _one_each, 1300, h_kv)


def test_single_rows_and_few_of_them_with_many_heads():
    """More heads than one round of a workgroup's waves takes, beside parts of the heads."""
    rng = _rng(4)
    for n_prob in (1, 3, 200):
        _appended(rng, "bf16", "e4m3", 128, 64, "half", 128, _one_each, n_prob, 13)
