"""Appending with the rotation on the way into 8-bit blocks (kv_paged_append_rotated), by the runs of tokens that fall to a
block: bit for bit what kv_rotate of fp32 rows gives, appended by the definition in float64 (oracle/paged.py).

Which kernel takes a call goes by its tokens to a request (up to four: runs taken by waves; more: by workgroups), so
every case has as many requests as its form needs.
"""
import numpy as np
import pytest

from oracle import paged
from paper_2609_30738_amd import _lib
from tests.test_gpu_paged import _dev, _dt, _host, _image, _rng, _same_image, _say

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
