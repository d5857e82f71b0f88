"""The 4-bit paged cache, rotary positions and reading a cache back on the host: the oracle's pins, the families of
frequencies, and the refusals of the entry points (nothing here launches a kernel: host addresses stand in for device
pointers)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged, rotary
from paper_2609_30738_amd import _lib
from tests.test_abi_cpu import BUF, NULL, P, HostProblem
from tests.test_paged_cpu import BAD_CACHES, ODD, _append, _attend, _cache, _compact

E2M1 = dict(qtype=_lib.KV_E2M1)


# ------------------------------------------------------------------------------------------------
# the oracle
# ------------------------------------------------------------------------------------------------

def test_oracle_values_and_order_of_halves():
    assert paged.values4(np.array([0x10, 0x32, 0x54, 0x76, 0x98, 0xFE], np.uint8)).tolist() == \
        [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -4, -6]


def test_oracle_rounds_to_nearest_and_ties_to_even():
    """Every midpoint, its fp32 neighbours and the numbers themselves, by a search over all codes."""
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float32)
    mid = (grid[1:] + grid[:-1]) / 2
    pts = np.concatenate([grid, mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(9))]).astype(np.float64)
    pts = np.concatenate([pts, -pts])
    for y in pts:
        x = np.zeros(32)
        x[0], x[1] = y, 6.0  # the largest pins the scale
        codes, b = paged.encode4(x)
        assert b.tolist() == [127]
        got = int(codes[0] & 15)
        dist = np.abs(grid.astype(np.float64) - abs(y))
        best = np.flatnonzero(dist == dist.min())
        want = best[0] if len(best) == 1 else [c for c in best if c % 2 == 0][0]
        assert got & 7 == want and bool(got & 8) == bool(np.signbit(y)), y


def test_oracle_scale_is_the_least():
    for e in (-120, -3, 0, 7, 120):
        s = 6 * 2.0 ** e
        assert paged.scale_byte4(s) == 127 + e and paged.scale_byte4(np.nextafter(s, np.inf)) == 128 + e
    assert paged.scale_byte4(0.0) == 2 and paged.scale_byte4(3.4e38) == 252


def test_oracle_numbers_that_are_none():
    x = np.zeros(32)
    x[:5] = np.nan, np.inf, -np.inf, 3.0, -0.0
    codes, b = paged.encode4(x)
    assert b.tolist() == [126]  # 3 = 6 / 2
    assert paged.values4(codes)[:5].tolist() == [0, 6, -6, 6, 0]


def test_oracle_rotation_keeps_lengths_and_turns_back():
    rng = np.random.default_rng(5)
    x, pos = rng.standard_normal((7, 3, 64)), np.array([0, 1, -5, 100, 1 << 20, 31744, 7])
    f, _ = rotary.frequencies("plain", 32, 1e4)
    for layout in ("half", "interleaved"):
        y, _ = rotary.rotate(x, pos, f, layout)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
        np.testing.assert_array_equal(y[0], x[0])
        np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
        z, _ = rotary.rotate(y, pos, f, layout, inverse=True)
        np.testing.assert_allclose(z, x, atol=1e-12)
        # logits depend on the distance alone
        q, k = x[:1], x[1:2]
        for a, b in ((9, 4), (1009, 1004)):
            dot = (rotary.rotate(q, [a], f, layout)[0] * rotary.rotate(k, [b], f, layout)[0]).sum()
            assert abs(dot - (rotary.rotate(q, [5], f, layout)[0] * k).sum()) < 1e-9


def test_oracle_rotation_is_a_product_of_complex_numbers():
    x = np.random.default_rng(6).standard_normal((4, 1, 16))
    pos, f = np.array([3, 0, 17, -2]), np.array([1.0, 0.3, 0.01, 2.5, 0.7, 0.2, 0.1, 1e-5])
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * 1.25 * np.exp(1j * pos[:, None] * f)[:, None]
    got, _ = rotary.rotate(x, pos, f, "interleaved", 1.25)
    np.testing.assert_allclose(got[..., 0::2], z.real, atol=1e-14)
    np.testing.assert_allclose(got[..., 1::2], z.imag, atol=1e-14)
    order = np.concatenate([np.arange(0, 16, 2), np.arange(1, 16, 2)])
    np.testing.assert_array_equal(rotary.rotate(x[..., order], pos, f, "half", 1.25)[0], got[..., order])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradient_is_the_inverse_rotation(layout):
    """Of L = <w, rotate(x)>: the inverse rotation of w, against central differences (the rotation is linear: what
    they leave is rounding, 2^-52 of the terms of L over the step)."""
    rng = np.random.default_rng(7)
    x, w, pos = rng.standard_normal((3, 2, 64)), rng.standard_normal((3, 2, 64)), np.array([5, 900, -3])
    f, _ = rotary.frequencies("yarn", 48, 1e4, (4.0, 100.0, 32.0, 1.0))
    g, _ = rotary.rotate(w, pos, f, layout, 1.14, inverse=True)
    h = 2.0 ** -10
    loss = lambda y: float((w * rotary.rotate(y, pos, f, layout, 1.14)[0]).sum())  # noqa: E731
    for at in [(0, 0, 0), (1, 1, 24), (2, 0, 47), (0, 1, 48), (1, 0, 63), (2, 1, 1)]:
        up, down = x.copy(), x.copy()
        up[at] += h
        down[at] -= h
        assert abs((loss(up) - loss(down)) / (2 * h) - (g[at] if at[2] < 48 else w[at])) < 400 * 2.0 ** -52 * 16 / h


# ------------------------------------------------------------------------------------------------
# frequencies
# ------------------------------------------------------------------------------------------------

FAMILIES = [("plain", ()), ("linear", (4.0,)), ("ntk", (8.0,)), ("yarn", (4.0, 8192.0, 32.0, 1.0)),
            ("yarn", (32.0, 512.0, 16.0, 2.0)), ("yarn", (1.0, 8192.0, 32.0, 1.0)), ("bands", (8.0, 8192.0, 1.0, 4.0)),
            ("bands", (2.0, 100.0, 0.5, 40.0))]


@pytest.mark.parametrize("family,params", FAMILIES)
@pytest.mark.parametrize("rot_dim", [16, 64, 80, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(family, params, rot_dim, base):
    got, factor = _lib.rotary_frequencies(family, rot_dim, base, params)
    want, want_factor = rotary.frequencies(family, rot_dim, base, params)
    np.testing.assert_allclose(got, want, rtol=1e-13)  # a few roundings of pow, log and the mixture
    assert factor == np.float32(want_factor)
    if family != "plain" and params[0] > 1:
        plain = rotary.frequencies("plain", rot_dim, base)[0]
        assert got[-1] < plain[-1] and np.all(got <= plain * (1 + 1e-15))


def test_frequencies_refusals():
    f = lambda *a, **k: _lib.rotary_frequencies(*a, **k)  # noqa: E731
    for args in (("plain", 15), ("plain", 0), ("plain", -2), ("ntk", 2, 1e4, (2.0,)), ("plain", 16, 1.0), ("plain", 16, math.inf),
                 ("plain", 16, math.nan), ("plain", 16, 1e4, (1.0,)), ("linear", 16), ("linear", 16, 1e4, (0.5,)),
                 ("linear", 16, 1e4, (math.nan,)), ("yarn", 16, 1e4, (4.0, 8192.0, 1.0, 32.0)),
                 ("yarn", 16, 1e4, (4.0, 0.0, 32.0, 1.0)), ("bands", 16, 1e4, (4.0, 8192.0, 4.0, 1.0)),
                 ("bands", 16, 1e4, (4.0, 8192.0, 1.0)), (5, 16), (-1, 16)):
        with pytest.raises(_lib.KvError) as e:
            f(*args)
        assert e.value.status == _lib.KV_ERR_ARG, args
    out = (ctypes.c_double * 8)()
    one = ctypes.c_float()
    assert _lib.lib().kv_rotary_frequencies(0, 1e4, None, 0, 16, None, ctypes.byref(one)) == _lib.KV_ERR_NULL
    assert _lib.lib().kv_rotary_frequencies(0, 1e4, None, 0, 16, out, None) == _lib.KV_ERR_NULL
    assert _lib.lib().kv_rotary_frequencies(1, 1e4, None, 1, 16, out, ctypes.byref(one)) == _lib.KV_ERR_NULL


# ------------------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------------------

def _rot(**kw):
    a = dict(layout=0, rot_dim=64, inverse=0, factor=1.0, freq=P.value)
    a.update(kw)
    return ctypes.byref(_lib.KvRotary(**a))


def _rotate(rot, dtype=_lib.KV_BF16, heads=8, d=128, x=P, xs=0, pos=P, n=4, out=ctypes.c_void_p(P.value + (1 << 20)), os_=0):
    return _lib.lib().kv_rotate(rot, dtype, heads, d, x, xs, pos, n, out, os_, NULL)


def _append_rotated(c, rot, pos=P, q=P, qs=0, qo=ctypes.c_void_p(P.value + (1 << 20)), qos=0, k=P, v=P, stride=0, slots=P, n=4):
    return _lib.lib().kv_paged_append_rotated(c, rot, pos, q, qs, qo, qos, k, v, stride, slots, n, NULL)


def _rows(c, off=P, n=100, k=P, v=P):
    return _lib.lib().kv_paged_rows(c, off, n, k, v, NULL)


BAD_ROTATIONS = [(dict(layout=2), _lib.KV_ERR_ARG), (dict(layout=-1), _lib.KV_ERR_ARG), (dict(rot_dim=0), _lib.KV_ERR_SHAPE),
                 (dict(rot_dim=8), _lib.KV_ERR_SHAPE), (dict(rot_dim=40), _lib.KV_ERR_SHAPE),
                 (dict(rot_dim=144), _lib.KV_ERR_SHAPE), (dict(factor=math.nan), _lib.KV_ERR_ARG),
                 (dict(factor=math.inf), _lib.KV_ERR_ARG), (dict(freq=None), _lib.KV_ERR_NULL),
                 (dict(freq=P.value + 4), _lib.KV_ERR_ARG)]


@pytest.mark.parametrize("kw,code", BAD_ROTATIONS)
def test_rotation_checks(kw, code):
    assert _rotate(_rot(**kw)) == code and _append_rotated(ctypes.byref(_cache(**E2M1)), _rot(**kw)) == code


def test_rotate_checks():
    r = _rot()
    assert _rotate(None) == _rotate(r, x=NULL) == _rotate(r, out=NULL) == _rotate(r, pos=NULL) == _lib.KV_ERR_NULL
    assert _rotate(r, x=ODD) == _rotate(r, out=ODD) == _rotate(r, n=0) == _lib.KV_ERR_ARG
    assert _rotate(r, dtype=2) == _lib.KV_ERR_DTYPE
    assert _rotate(r, d=96) == _rotate(r, heads=0) == _rotate(r, heads=1 << 20) == _rotate(r, n=(1 << 25) + 1) == _lib.KV_ERR_SHAPE
    assert _rotate(_rot(rot_dim=80), d=64) == _lib.KV_ERR_SHAPE
    for s in (1016, 1028, -8, (1 << 26) + 8):
        assert _rotate(r, xs=s) == _rotate(r, os_=s) == _lib.KV_ERR_ARG


def test_rotate_overlaps():
    """Rows that meet other rows than their own: out shifted within a row, a row further, in place with another stride, a
    slice that reaches into the next one."""
    r, e = _rot(), 2
    at = lambda n: ctypes.c_void_p(P.value + e * n)  # noqa: E731
    packed = 8 * 128
    for kw in (dict(out=at(8)), dict(out=at(packed)), dict(out=at(3 * packed + packed - 8)), dict(out=P, os_=2 * packed),
               dict(xs=2 * packed, out=at(packed - 8), os_=2 * packed), dict(xs=2 * packed, out=at(packed + 8), os_=2 * packed),
               dict(xs=4 * packed, out=at(4 * packed), os_=packed), dict(x=at(2 * packed), out=P),
               dict(n=1, out=at(8)), dict(n=1, out=at(packed - 8))):
        assert _rotate(r, **kw) == _lib.KV_ERR_ARG, kw
    c = ctypes.byref(_cache(**E2M1))
    assert _append_rotated(c, r, qo=at(8)) == _append_rotated(c, r, qo=at(4096)) == _lib.KV_ERR_ARG
    # the rotated queries over the keys or values: the same rows, a slice that reaches into theirs
    far = ctypes.c_void_p(P.value + (1 << 20))
    for kw in (dict(k=far), dict(v=far), dict(k=ctypes.c_void_p(far.value + 2 * 3 * 1024)),
               dict(v=ctypes.c_void_p(far.value + 2 * (6144 + 4088)), stride=6144, qos=6144)):
        assert _append_rotated(c, r, qo=far, **kw) == _lib.KV_ERR_ARG, kw


def test_attention_counts_rounds_in_32_bits():
    """All problems' rounds of 128 rows, n_prob (max_len / 128 + 1), stay below 2^31."""
    far = dict(E2M1, max_len=1 << 24, table_stride=1 << 18, block_rows=64)
    assert (1 << 24) // 128 + 1 == 131073 and 16383 * 131073 < 1 << 31 < 16384 * 131073
    for n, code in ((16384, _lib.KV_ERR_SHAPE), (65535, _lib.KV_ERR_SHAPE), (16383, _lib.KV_ERR_WORKSPACE)):
        c = ctypes.byref(_cache(n_prob=n, **far))
        assert _attend(c, n_tok=n, max_q=1) == code, n


def test_append_rotated_checks():
    c, r = ctypes.byref(_cache(**E2M1)), _rot()
    for kw in (dict(pos=NULL), dict(k=NULL), dict(v=NULL), dict(slots=NULL), dict(q=NULL), dict(qo=NULL)):
        assert _append_rotated(c, r, **kw) == _lib.KV_ERR_NULL, kw
    assert _append_rotated(None, r) == _append_rotated(c, None) == _lib.KV_ERR_NULL
    for kw in (dict(k=ODD), dict(v=ODD), dict(q=ODD), dict(qo=ODD), dict(n=0), dict(stride=1020), dict(qs=4100), dict(qos=4090)):
        assert _append_rotated(c, r, **kw) == _lib.KV_ERR_ARG, kw
    assert _append_rotated(c, r, n=(1 << 25) + 1) == _lib.KV_ERR_SHAPE
    assert _append_rotated(ctypes.byref(_cache(d=64)), _rot(rot_dim=128)) == _lib.KV_ERR_SHAPE


def test_rows_checks():
    c = ctypes.byref(_cache(**E2M1))
    assert _rows(None) == _rows(c, off=NULL) == _rows(c, k=NULL, v=NULL) == _lib.KV_ERR_NULL
    row = 8 * 128 * 2
    for kw in (dict(), dict(v=ctypes.c_void_p(P.value + 9 * row - 16)), dict(k=ctypes.c_void_p(P.value + 8 * row))):
        assert _rows(c, n=9, **kw) == _lib.KV_ERR_ARG, kw  # keys and values overlap
    assert _rows(c, k=ODD) == _rows(c, v=ODD, k=NULL) == _rows(c, n=0) == _rows(c, n=-1) == _lib.KV_ERR_ARG


@pytest.mark.parametrize("kw,code", [x for x in BAD_CACHES if "qtype" not in x[0]])
def test_cache_checks(kw, code):
    c = ctypes.byref(_cache(**{**E2M1, **kw}))
    pr = HostProblem(lens=(4096,) * 4)
    assert _attend(c) == _append(c) == _compact(pr.ref(), c) == _rows(c) == _append_rotated(c, _rot()) == code
    assert _lib.lib().kv_paged_attention_workspace_bytes(c, 4, 1) == 0


def test_scales_of_4_bits_are_aligned():
    for name in ("k_scale", "v_scale"):
        four, eight = (ctypes.byref(_cache(qtype=t, **{name: P.value + 8})) for t in (_lib.KV_E2M1, _lib.KV_INT8))
        assert _attend(four, ws_bytes=0) == _append(four) == _rows(four) == _lib.KV_ERR_ARG
        assert _append(eight, n=0) == _lib.KV_ERR_ARG and _append(eight, slots=NULL) == _lib.KV_ERR_NULL  # not the scales


def test_other_code_types_are_refused():
    for t in (-1, 2, 3, 5):
        c = ctypes.byref(_cache(qtype=t))
        assert _attend(c) == _append(c) == _rows(c) == _append_rotated(c, _rot()) == _lib.KV_ERR_DTYPE


def test_workspace_is_that_of_8_bits():
    for kw in (dict(max_len=100), dict(n_blocks=4000, table_stride=2048, max_len=32768), dict(dtype=_lib.KV_F32)):
        for n, m in ((4, 1), (40, 9), (2000, 512)):
            need = [_lib.lib().kv_paged_attention_workspace_bytes(ctypes.byref(_cache(qtype=t, **kw)), n, m) for t in (0, 4)]
            assert (need[0] > 0) == (need[1] > 0)


def test_binding_checks():
    """Shapes and types that the binding itself refuses, on CPU tensors."""
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pool = torch.zeros(8, 2, 16, 32, dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    sc = torch.zeros(8, 2, 2, 16, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for args in ((pool, pool, torch.zeros(8, 2), sc), (pool.view(torch.uint8), pool.view(torch.uint8), sc, sc),
                 (pool, pool.view(torch.uint8), sc, sc), (pool, pool, sc, sc)):  # the last: host tensors
        with pytest.raises(ValueError):
            _lib.PagedCache("bf16", 4, *args, table, lens)
    f = torch.zeros(32, dtype=torch.float64)
    for args in (("half", f), ("other", f), ("half", f.float())):
        with pytest.raises(ValueError):
            _lib.Rotary(*args)
