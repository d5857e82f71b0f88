"""Rotary positions on the GPU against the definition in float64 (oracle/rotary.py): kv_rotate, and the queries and keys
of kv_paged_append_rotated.

An angle is the same product of doubles on both sides; cosine and sine are rounded to fp32 (2^-24 of each, and
2^-24 more where a rounding of the double before it tips it over, with their series' remainder far below), each of the two
products and their sum once: an element errs by at most 4 2^-24 (|a c| + |b s|), and its rounding to bf16 by 2^-8 of
itself (of what it was rounded from).  Results below the normal numbers may become 0: 2^-126.
"""
import numpy as np
import pytest

from oracle import paged, rotary
from paper_2609_30738_amd import _lib
from tests.test_gpu_paged import _bits, _dev, _dt, _host, _image, _pool, _q, _rng, _rows, _say

pytestmark = pytest.mark.gpu

LAYOUTS = ["half", "interleaved"]


def _rotary(family, rot, layout, params=(), base=1e4, inverse=False):
    f, factor = _lib.rotary_frequencies(family, rot, base, params)
    return _lib.Rotary(layout, _dev(f), factor, inverse), f, factor


def _positions(rng, T):
    """Near and far ones, 0, the ends of the range of a cache and negative ones."""
    p = rng.integers(0, 1 << 24, T)
    p[::2] = rng.integers(0, 40000, len(p[::2]))
    for i, x in enumerate((0, 1, (1 << 24) - 1, -1, -70000, (1 << 31) - 1)):
        if 3 * i < T:
            p[3 * i] = x
    return p.astype(np.int32)


def _near(got, x, pos, f, layout, factor, inverse, dtype, where):
    want, mag = rotary.rotate(_host(x), pos, f, layout, factor, inverse)
    bound = 4 * 2.0 ** -24 * mag + 2.0 ** -126
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    err = np.abs(_host(got) - want) - bound
    assert np.all(err <= 0), f"{where}: over the bound by {err.max():.3g} at {np.unravel_index(np.argmax(err), err.shape)}"
    rest = slice(2 * len(f), None)
    np.testing.assert_array_equal(_host(got)[..., rest], _host(x)[..., rest], err_msg=where)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 16), (128, 80), (128, 112), (64, 64), (64, 32), (64, 48), (64, 16)])
def test_rotate(dtype, layout, d, rot):
    """Tokens around a workgroup's group, odd numbers of heads, the angle's sign, factors, slices of wider rows."""
    import torch
    rng = _rng(d, rot, len(layout))
    for T, heads, family, params, inverse in ((1, 1, "plain", (), False), (7, 5, "yarn", (4.0, 8192.0, 32.0, 1.0), True),
                                              (33, 3, "ntk", (4.0,), False), (130, 9, "bands", (8.0, 8192.0, 1.0, 4.0), True)):
        r, f, factor = _rotary(family, rot, layout, params, inverse=inverse)
        pos = _positions(rng, T)
        wide = _q(rng, T, heads + 3, d, dtype)
        x = wide[:, 1:heads + 1]
        out = torch.full((T, heads + 2, d), 7.0, dtype=x.dtype, device="cuda")
        _say("rotate", dtype, layout, d, rot, T, heads, family)
        _lib.rotate(r, x, _dev(pos), out[:, 2:])
        _near(out[:, 2:], x, pos, f, layout, factor, inverse, dtype, f"{family} {T}")
        assert (out[:, :2] == 7).all()
        same = x.contiguous()
        _lib.rotate(r, same, _dev(pos), same)  # in place
        assert torch.equal(same, out[:, 2:])
        beside = wide.clone()
        if heads >= 3:  # from one slice of a row to another
            _lib.rotate(r, beside[:, :1], _dev(pos), beside[:, heads + 2:])
            assert torch.equal(beside[:, heads + 2:], _alone(r, wide[:, :1], pos)) and torch.equal(beside[:, :heads + 2], wide[:, :heads + 2])


def _alone(r, x, pos):
    import torch
    out = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    _lib.rotate(r, x, _dev(pos), out)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,heads", [(5000, 40), (3, 300), (20000, 1), (700, 128)])
def test_rotate_many(dtype, T, heads):
    """Heads and tokens past what one round of the chip takes."""
    rng = _rng(T, heads)
    r, f, factor = _rotary("plain", 128, "half", base=5e5)
    pos = rng.integers(0, 131072, T).astype(np.int32)
    x = _q(rng, T, heads, 128, dtype)
    _say("rotate many", dtype, T, heads)
    _near(_alone(r, x, pos), x, pos, f, "half", factor, False, dtype, "many")


@pytest.mark.parametrize("layout", LAYOUTS)
def test_rotate_angles(layout):
    """Elements 1 and 0 give cosine and sine themselves: within a rounding of fp32, at quarter turns, around them and far out."""
    import torch
    f = np.array([np.pi / 2, 1.0, np.pi / 4, 2.0 ** -30, 1e-7, 0.1, 3.0, 0.75])
    pos = np.concatenate([np.arange(-600, 600), 2 ** np.arange(31), 2 ** np.arange(31) - 1, -(2 ** np.arange(31))]).astype(np.int32)
    x = torch.zeros(len(pos), 1, 64, device="cuda")
    x[..., 0:8] = 1
    if layout == "interleaved":
        x.zero_()
        x[..., 0:16:2] = 1
    _say("angles", layout)
    y = _host(_alone(_lib.Rotary(layout, _dev(f)), x, pos))[:, 0]
    c, s = (y[:, 0:8], y[:, 8:16]) if layout == "half" else (y[:, 0:16:2], y[:, 1:16:2])
    angle = pos.astype(np.float64)[:, None] * f
    # half a rounding, and 2^-52 of a double series and reduction beside a number that may be small
    for got, want in ((c, np.cos(angle)), (s, np.sin(angle))):
        assert np.all(np.abs(got - want) <= 1.0001 * 2.0 ** -24 * np.abs(want) + 2.0 ** -50)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rot", [128, 48])
def test_inverse_is_the_gradient(layout, rot):
    """<w, rotate(x)> against <inverse(w), x>, with fp32 rows: each side's elements err by 4 2^-24 of their terms; and the
    inverse of the rotation gives the row back."""
    rng = _rng(rot)
    T = 40
    r, f, factor = _rotary("yarn", rot, layout, (4.0, 8192.0, 32.0, 1.0))
    back = _lib.Rotary(layout, r.freq, factor, inverse=True)
    pos = rng.integers(0, 100000, T).astype(np.int32)
    x, w = _q(rng, T, 3, 128, "f32"), _q(rng, T, 3, 128, "f32")
    y, g = _alone(r, x, pos), _alone(back, w, pos)
    terms = rotary.rotate(_host(x), pos, f, layout, factor)[1], rotary.rotate(_host(w), pos, f, layout, factor)[1]
    bound = 4 * 2.0 ** -24 * (terms[0] * np.abs(_host(w)) + terms[1] * np.abs(_host(x))).sum()
    assert abs((_host(w) * _host(y)).sum() - (_host(g) * _host(x)).sum()) <= bound
    z = _host(_alone(back, y, pos))
    z[..., :rot] /= factor ** 2
    assert np.all(np.abs(z - _host(x)) <= 16 * 2.0 ** -24 * np.abs(_host(x)).max((-1), keepdims=True))


def test_rotate_numbers_that_are_none():
    """A NaN or an infinity reaches its pair alone."""
    import torch
    rng = _rng(3)
    r, f, _ = _rotary("plain", 64, "half")
    pos = np.array([5, 6, 7], np.int32)
    x = _q(rng, 3, 2, 128, "bf16")
    clean = _alone(r, x, pos)
    x[0, 1, 3], x[1, 0, 40], x[2, 0, 100] = float("nan"), float("inf"), float("-inf")
    y = _alone(r, x, pos)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[0, 1, [3, 35]] = want[1, 0, [8, 40]] = want[2, 0, 100] = True
    assert torch.equal(bad, want) and torch.equal(y[~bad], clean[~bad])


def test_rotate_past_32_bit_offsets():
    """Rows whose elements lie past 4 GiB, by a large stride."""
    import torch
    rng = _rng(4)
    T, stride = 70, 1 << 25
    r, f, _ = _rotary("plain", 128, "interleaved")
    big = torch.empty((T - 1) * stride + 256, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((T, 2, 128), (stride, 128, 1))
    src = _q(rng, T, 2, 128, "bf16")
    x.copy_(src)
    pos = rng.integers(0, 9999, T).astype(np.int32)
    _say("rotate past 4 GiB")
    _lib.rotate(r, x, _dev(pos), x)
    assert torch.equal(x.contiguous(), _alone(r, src, pos))


def test_rotate_binding_refuses():
    import torch
    rng = _rng(9)
    r, _, _ = _rotary("plain", 64, "half")
    x, pos = _q(rng, 4, 2, 64, "bf16"), _dev(np.zeros(4, np.int32))
    out = torch.empty_like(x)
    for bad in ((x.half(), pos, out), (x, pos.long(), out), (x, pos[:3], out), (x, pos, out.float()), (x, pos, out[:3]),
                (x, pos.cpu(), out), (x.cpu(), pos, out), (x[0], pos, out[0]), (x[:1].expand(4, 2, 64), pos, out),
                (x, pos, out.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            _lib.rotate(r, *bad)
    wide = _rotary("plain", 128, "half")[0]
    with pytest.raises(_lib.KvError):  # more than the head
        _lib.rotate(wide, x, pos, out)
    buf = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(_lib.KvError):  # a row further
        _lib.rotate(r, buf[:4], pos, buf[1:])
    _lib.rotate(r, x[:0], pos[:0], out[:0])  # nothing to do


# ------------------------------------------------------------------------------------------------
# appending with the rotation on the way
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype,qtype,d,rot", [("bf16", "e4m3", 128, 128), ("bf16", "int8", 64, 48), ("bf16", "e2m1", 128, 80),
                                               ("f32", "e4m3", 64, 64), ("f32", "int8", 128, 16), ("f32", "e2m1", 128, 128),
                                               ("bf16", "e2m1", 64, 16), ("f32", "e2m1", 64, 48), ("bf16", "e4m3", 128, 112)])
@pytest.mark.parametrize("R", [16, 32, 64, 128])
def test_append_rotated_is_rotation_then_append(layout, dtype, qtype, d, rot, R):
    """Bit for bit what kv_rotate of fp32 rows and appending them give, and the queries what kv_rotate gives: prompts
    around the sizes of blocks, then single rows and runs behind them, skipped slots, with queries and without."""
    import torch
    rng = _rng(R, d, rot, len(dtype))
    h_q, h_kv, lens = 6, 3, [0, 1, R - 1, R, R + 1, 300, 17]
    stride = 420 // R + 2
    n_blocks = 40 + 7 * stride
    a = _pool(_lib.PagedCache.allocate(dtype, qtype, h_q, h_kv, d, R, n_blocks, 7, stride))
    b = _pool(_lib.PagedCache.allocate("f32", qtype, h_q, h_kv, d, R, n_blocks, 7, stride))
    table = rng.permutation(n_blocks)[:7 * stride].reshape(7, stride)
    at = [0] * 7
    r, _, _ = _rotary("yarn", rot, layout, (2.0, 4096.0, 32.0, 1.0))
    for step, adds in enumerate([lens, [1] * 7, [5, 0, 1, 2, 0, 40, 3], [1] * 7]):
        slots = [table[p, i // R] * R + i % R for p in range(7) for i in range(at[p], at[p] + adds[p])]
        pos = [i + 1000 * p for p in range(7) for i in range(at[p], at[p] + adds[p])]
        if step == 2:
            slots += [-1, n_blocks * R, -5]  # a padded batch
            pos += [0, 1 << 30, -9]
        T = len(slots)
        qkv = _rows(rng, T, h_q + 2 * h_kv, d, dtype)
        q, k, v = qkv[:, :h_q], qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:]
        slots, pos = _dev(np.asarray(slots, np.int32)), _dev(np.asarray(pos, np.int32))
        want = _alone_at(r, q, pos)
        k32 = _alone_at(r, k.float(), pos)
        q_out = torch.empty(T, h_q, d, dtype=q.dtype, device="cuda") if step % 2 == 0 else None
        if step == 2:
            q_out = q  # in place
        _say("append rotated", layout, dtype, qtype, d, rot, R, step)
        _lib.paged_append(b, k32, v.float().contiguous(), slots)
        _lib.paged_append_rotated(a, r, pos, k, v, slots, q=q if q_out is not None else None, q_out=q_out)
        if q_out is not None:
            assert torch.equal(q_out, want), step
        for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), step
        at = [x + n for x, n in zip(at, adds)]


def _alone_at(r, x, pos):
    import torch
    out = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    _lib.rotate(r, x, pos, out)
    return out


@pytest.mark.parametrize("qtype", ["e4m3", "int8", "e2m1"])
def test_append_rotated_against_the_definition(qtype):
    """Rotated rows in float64, coded: the same codes but where the fp32 value lies on the other side of a rounding's
    border, whose distance from it is below the bound of the rotation; scales likewise."""
    rng = _rng(12)
    R, h_kv, d, T = 32, 2, 128, 100
    r, f, factor = _rotary("plain", 128, "half")
    pc = _pool(_lib.PagedCache.allocate("bf16", qtype, 4, h_kv, d, R, 4, 1, 4))
    k = _rows(rng, T, h_kv, d, "bf16")
    pos = rng.integers(0, 30000, T).astype(np.int32)
    _say("append rotated values", qtype)
    _lib.paged_append_rotated(pc, r, _dev(pos), k, k, _dev(np.arange(T, dtype=np.int32)))
    want, mag = rotary.rotate(_host(k), pos, f, "half", factor)
    table = np.arange(4)
    if qtype == "e2m1":
        got, _ = paged.cache_rows4(_bits(pc.k), _bits(pc.k_scale), table, T)
    else:
        codes, scales = _image(pc)
        got, _ = paged.cache_rows(codes[0], scales[0], table, T, qtype)
    got = got.transpose(1, 0, 2)
    slack = 4 * 2.0 ** -24 * mag
    if qtype == "int8":
        half = np.repeat(scales[0], R, 0)[:T][:, :, None] / 2
    elif qtype == "e4m3":
        half = np.maximum(np.abs(want) * 2.0 ** -4, np.repeat(scales[0], R, 0)[:T][:, :, None] * 2.0 ** -10)
    else:
        s = np.exp2(_bits(pc.k_scale).astype(float) - 127)  # [4, h_kv, 4, R]
        s = s.transpose(0, 3, 1, 2).reshape(4 * R, h_kv, 4).repeat(32, -1)[:T]
        half = np.maximum(np.abs(want) / 4, s / 4)  # steps of a half below 2, of 1 and 2 beyond
    assert np.all(np.abs(got - want) <= half * (1 + 1e-5) + slack)


def test_append_rotated_many_requests():
    """2000 single rows, and prompts of many blocks: more runs than workgroups, every slot once."""
    import torch
    rng = _rng(13)
    R, h_kv, d = 16, 8, 128
    for qtype in ("e4m3", "e2m1"):
        for T, single in ((2000, True), (9000, False)):
            n_blocks = 2100
            r, _, _ = _rotary("plain", 128, "half")
            a, b = (_pool(_lib.PagedCache.allocate(t, qtype, 32, h_kv, d, R, n_blocks, 1, 1)) for t in ("bf16", "f32"))
            perm = rng.permutation(n_blocks)
            i = np.arange(T)
            slots = perm[:T] * R if single else perm[i // R] * R + i % R
            slots, pos = _dev(slots.astype(np.int32)), _dev(rng.integers(0, 1 << 20, T).astype(np.int32))
            k, v, q = (_rows(rng, T, h, d, "bf16") for h in (h_kv, h_kv, 32))
            out = torch.empty_like(q)
            _say("append rotated many", qtype, T)
            _lib.paged_append_rotated(a, r, pos, k, v, slots, q=q, q_out=out)
            _lib.paged_append(b, _alone_at(r, k.float(), pos), v.float(), slots)
            for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            assert torch.equal(out, _alone_at(r, q, pos))


def test_append_rotated_numbers_that_are_none():
    """NaN and infinite elements, which the rotation spreads over their pairs: as appending the rotated rows."""
    import torch
    rng = _rng(14)
    R, d = 16, 64
    r, _, _ = _rotary("plain", 32, "interleaved")
    for qtype in ("e4m3", "int8", "e2m1"):
        a, b = (_pool(_lib.PagedCache.allocate("f32", qtype, 2, 1, d, R, 3, 1, 3)) for _ in range(2))
        k = _rows(rng, 40, 1, d, "f32")
        k[3, 0, 4], k[20, 0, 9], k[21, 0, 50], k[39, 0, 33] = float("nan"), float("inf"), float("-inf"), float("nan")
        pos, slots = _dev(np.arange(40, dtype=np.int32)), _dev(np.arange(40, dtype=np.int32))
        _lib.paged_append_rotated(a, r, pos, k, k, slots)
        _lib.paged_append(b, _alone_at(r, k, pos), k, slots)
        for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), qtype


def test_append_rotated_binding_refuses():
    import torch
    rng = _rng(15)
    r, _, _ = _rotary("plain", 64, "half")
    pc = _lib.PagedCache.allocate("bf16", "e2m1", 4, 2, 64, 16, 4, 1, 4)
    k, q = _q(rng, 3, 2, 64, "bf16"), _q(rng, 3, 4, 64, "bf16")
    pos, slots = (_dev(np.arange(3, dtype=np.int32)) for _ in range(2))
    for args, kw in (((pos.long(), k, k, slots), {}), ((pos[:2], k, k, slots), {}), ((pos, k, k[:2], slots), {}),
                     ((pos, k.float(), k, slots), {}), ((pos, k, k, slots[:2]), {}), ((pos, k, k, slots), dict(q=q)),
                     ((pos, k, k, slots), dict(q=q[:2], q_out=q[:2])), ((pos, k, k, slots), dict(q=k, q_out=k)),
                     ((pos, k, k, slots), dict(q=q, q_out=q.float()))):
        with pytest.raises(ValueError):
            _lib.paged_append_rotated(pc, r, *args, **kw)
    before = _bits(pc.k).copy()
    _lib.paged_append_rotated(pc, r, pos[:0], k[:0], k[:0], slots[:0], q=q[:0], q_out=torch.empty_like(q)[:0])
    assert np.array_equal(_bits(pc.k), before)


def test_captured_prompts_and_single_rows():
    """Prompts into 8-bit blocks of 128 rows (their turns take most of a workgroup's LDS) and single rows behind them, captured
    once and replayed with other rows and positions, other work between the replays: every replay equals the eager calls."""
    import torch
    rng = _rng(51)
    h_q, h_kv, d, R, lens = 4, 2, 128, 128, [200, 128, 3]
    r, _, _ = _rotary("plain", 128, "half")
    caches = [_pool(_lib.PagedCache.allocate("f32", "e4m3", h_q, h_kv, d, R, 9, 3, 3)) for _ in range(2)]
    blocks = rng.permutation(9).reshape(3, 3)
    first = [blocks[p, i // R] * R + i % R for p in range(3) for i in range(lens[p])]
    then = [blocks[p, lens[p] // R] * R + lens[p] % R for p in range(3)]
    slots = [_dev(np.asarray(x, np.int32)) for x in (first, then)]
    qkv = [torch.zeros(len(x), h_q + 2 * h_kv, d, device="cuda") for x in (first, then)]
    pos = [torch.zeros(len(x), dtype=torch.int32, device="cuda") for x in (first, then)]
    outs = [[torch.zeros(len(x), h_q, d, device="cuda") for x in (first, then)] for _ in range(2)]

    def step(pc, out):
        for i in range(2):
            _lib.paged_append_rotated(pc, r, pos[i], qkv[i][:, h_q:h_q + h_kv], qkv[i][:, h_q + h_kv:], slots[i], q=qkv[i][:, :h_q], q_out=out[i])

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(caches[0], outs[0])
    torch.cuda.synchronize()
    for i in range(4):
        for x, p in zip(qkv, pos):
            x.copy_(_dev(rng.standard_normal(x.shape).astype(np.float32) * 3.0 ** i))
            p.copy_(_dev(rng.integers(0, 1 << 20, len(p)).astype(np.int32)))
        _say("captured prompts", i)
        graph.replay()
        other = torch.randn(200, 200, device="cuda") @ torch.randn(200, 200, device="cuda")
        step(caches[1], outs[1])
        torch.cuda.synchronize()
        del other
        for a, b in zip(outs[0], outs[1]):
            assert torch.equal(a, b), i
        for n in ("k", "v", "k_scale", "v_scale"):
            x, y = (getattr(c, n).view(torch.uint8) for c in caches)
            assert torch.equal(x, y), (i, n)
