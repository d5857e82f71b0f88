"""The 8-bit paged cache on the host: the oracle's codes against torch's, and the refusals of the paged
entry points (nothing here launches a kernel: host addresses stand in for device pointers)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_30738_amd import _lib
from tests.test_abi_cpu import BUF, NULL, P, HostProblem

ODD = ctypes.c_void_p(BUF.ctypes.data + 4)


def test_oracle_e4m3_values_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(paged.values(codes, "e4m3"), want)


def test_oracle_rounding_is_torchs():
    """Every bf16 number up to 448, the midpoints of neighbouring e4m3 numbers and their fp32 neighbours."""
    x = (np.arange(1 << 15, dtype=np.uint32) << 16).view(np.float32)
    grid = paged.values(np.arange(0x7F), "e4m3").astype(np.float32)
    mid = (grid[1:] + grid[:-1]) / 2
    x = np.concatenate([x[np.isfinite(x)], mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(999))])
    x = np.concatenate([x[x <= 448], -x[x <= 448]])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(paged.encode(x, 1.0, "e4m3"), want)


@pytest.mark.parametrize("qtype", ["e4m3", "int8"])
def test_oracle_scale_is_the_least(qtype):
    top = paged.QMAX[qtype]
    for e in (-120, -3, 0, 7, 100):
        s = 2.0 ** e
        assert paged.least_scale(top * s, qtype) == s
        assert paged.least_scale(np.nextafter(np.float32(top * s), np.float32(np.inf)), qtype) == 2 * s
    assert paged.least_scale(0.0, qtype) == 0 and paged.least_scale(2.0 ** -149, qtype) == 2.0 ** -126


# ------------------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------------------

def _cache(**kw):
    a = dict(dtype=_lib.KV_BF16, qtype=_lib.KV_E4M3, n_prob=4, h_q=32, h_kv=8, d=128, block_rows=16, n_blocks=100,
             table_stride=20, max_len=320, k=P.value, v=P.value, k_scale=P.value, v_scale=P.value, table=P.value,
             len=P.value)
    a.update(kw)
    return _lib.KvPagedCache(**a)


BAD_CACHES = [
    (dict(dtype=5), _lib.KV_ERR_DTYPE), (dict(qtype=2), _lib.KV_ERR_DTYPE), (dict(n_prob=0), _lib.KV_ERR_ARG),
    (dict(n_prob=65536), _lib.KV_ERR_ARG), (dict(h_q=30), _lib.KV_ERR_SHAPE), (dict(h_q=4), _lib.KV_ERR_SHAPE),
    (dict(h_q=136), _lib.KV_ERR_SHAPE), (dict(h_q=0, h_kv=0), _lib.KV_ERR_SHAPE), (dict(d=96), _lib.KV_ERR_SHAPE),
    (dict(block_rows=8), _lib.KV_ERR_SHAPE), (dict(block_rows=48), _lib.KV_ERR_SHAPE),
    (dict(n_blocks=0), _lib.KV_ERR_SHAPE), (dict(n_blocks=1 << 27), _lib.KV_ERR_SHAPE),
    (dict(table_stride=0), _lib.KV_ERR_SHAPE), (dict(table_stride=1 << 27), _lib.KV_ERR_SHAPE),
    (dict(max_len=-1), _lib.KV_ERR_SHAPE), (dict(max_len=(1 << 24) + 1), _lib.KV_ERR_SHAPE),
    (dict(k=None), _lib.KV_ERR_NULL), (dict(v_scale=None), _lib.KV_ERR_NULL), (dict(table=None), _lib.KV_ERR_NULL),
    (dict(len=None), _lib.KV_ERR_NULL), (dict(v=P.value + 4), _lib.KV_ERR_ARG),
]


def _attend(c, q=P, stride=0, off=P, n_tok=4, max_q=1, scale=0.1, out=P, ws=P, ws_bytes=1 << 30):
    return _lib.lib().kv_paged_attention(c, q, stride, off, n_tok, max_q, scale, out, ws, ws_bytes, NULL)


def _append(c, k=P, v=P, stride=0, slots=P, n=4):
    return _lib.lib().kv_paged_append(c, k, v, stride, slots, n, NULL)


def _compact(pr, c, budget=64, tail=32, bh=NULL, bd=NULL, k=P, sel=P):
    return _lib.lib().kv_paged_compact(pr, k, P, sel, budget, tail, bh, bd, c, NULL)


def _tables(c, off=P, blk=P, slots=P, n_free=10, n_slots=10):
    return _lib.lib().kv_paged_tables(c, NULL, NULL, NULL, n_free, NULL, NULL, off, blk, slots, n_slots, NULL)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_cache_checks(kw, code):
    c = ctypes.byref(_cache(**kw))
    pr = HostProblem(lens=(4096,) * 4)
    assert _attend(c) == code and _append(c) == code and _compact(pr.ref(), c) == code
    assert _lib.lib().kv_paged_attention_workspace_bytes(c, 4, 1) == 0


def test_null_cache():
    assert _attend(None) == _append(None) == _tables(None) == _lib.KV_ERR_NULL
    assert _compact(HostProblem().ref(), None) == _lib.KV_ERR_NULL


def test_attention_checks():
    c = ctypes.byref(_cache())
    assert _attend(c, q=NULL) == _attend(c, out=NULL) == _lib.KV_ERR_NULL
    assert _attend(c, q=ODD) == _attend(c, out=ODD) == _lib.KV_ERR_ARG
    assert _attend(c, scale=float("nan")) == _attend(c, scale=float("inf")) == _lib.KV_ERR_ARG
    for n_tok, max_q in ((0, 1), (4, 0), (4, 5), (-1, -1)):
        assert _attend(c, n_tok=n_tok, max_q=max_q) == _lib.KV_ERR_ARG
        assert _lib.lib().kv_paged_attention_workspace_bytes(c, n_tok, max_q) == 0
    assert _attend(c, off=NULL, n_tok=5) == _lib.KV_ERR_ARG       # one token each, but five of them
    assert _attend(c, off=NULL, n_tok=8, max_q=2) == _lib.KV_ERR_ARG
    assert _attend(c, n_tok=1 << 24, max_q=1 << 24) == _lib.KV_ERR_SHAPE
    assert _attend(c, n_tok=1 << 25, max_q=(1 << 24) + 1) == _lib.KV_ERR_SHAPE
    f = ctypes.byref(_cache(dtype=_lib.KV_F32))
    assert _attend(f, n_tok=1 << 17, max_q=1 << 17) == _lib.KV_ERR_SHAPE
    assert _attend(c, stride=4095) == _attend(c, stride=4100) == _attend(c, stride=-8) == _lib.KV_ERR_ARG


def test_attention_of_the_longest_turns():
    """The largest turns that the launches take, by the workspace that they ask for, and one token more."""
    f = lambda c, n: _lib.lib().kv_paged_attention_workspace_bytes(ctypes.byref(c), n, n)  # noqa: E731
    # a unit's 4 columns a token, 8 heads: 8191 groups of 32 columns
    c = _cache(dtype=_lib.KV_F32, n_blocks=1000, table_stride=1000, max_len=16000)
    most = 8191 * 32 // 4
    assert f(c, most) == -(-most * 32 * 8 * 130 * 4 // 256) * 256 and f(c, most + 1) == 0
    assert _attend(ctypes.byref(c), n_tok=most + 1, max_q=most + 1) == _lib.KV_ERR_SHAPE
    assert _attend(ctypes.byref(c), n_tok=most, max_q=most, ws_bytes=0) == _lib.KV_ERR_WORKSPACE
    # two splits of 65536 rows: 32767 groups of 256 columns
    c = _cache(n_blocks=8192, table_stride=8192, max_len=131072)
    most = 32767 * 256 // 4
    assert f(c, most) == -(-most * 32 * 2 * 130 * 4 // 256) * 256 and f(c, most + 1) == 0
    assert _attend(ctypes.byref(c), n_tok=most + 1, max_q=most + 1) == _lib.KV_ERR_SHAPE
    assert _attend(ctypes.byref(c), n_tok=most, max_q=most, ws_bytes=0) == _lib.KV_ERR_WORKSPACE


def test_attention_scale_times_log2e():
    """The largest scales are finite and their product with log2(e) is not."""
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert _attend(ctypes.byref(_cache()), scale=scale) == _lib.KV_ERR_ARG


def test_attention_workspace():
    c = _cache(n_blocks=4000, table_stride=2048, max_len=32768)
    need = _lib.lib().kv_paged_attention_workspace_bytes(ctypes.byref(c), 4, 1)
    assert need > 0 and need % 256 == 0
    assert _attend(ctypes.byref(c), ws_bytes=need - 1) == _lib.KV_ERR_WORKSPACE
    assert _attend(ctypes.byref(c), ws=NULL, ws_bytes=need) == _lib.KV_ERR_WORKSPACE
    assert _attend(ctypes.byref(c), ws=ctypes.c_void_p(BUF.ctypes.data + 16), ws_bytes=need) == _lib.KV_ERR_WORKSPACE
    # a short bound needs none, whatever the table could hold
    c.max_len = 100
    assert _lib.lib().kv_paged_attention_workspace_bytes(ctypes.byref(c), 4, 1) == 0


def test_append_checks():
    c = ctypes.byref(_cache())
    assert _append(c, k=NULL) == _append(c, v=NULL) == _append(c, slots=NULL) == _lib.KV_ERR_NULL
    assert _append(c, k=ODD) == _append(c, v=ODD) == _append(c, n=0) == _lib.KV_ERR_ARG
    assert _append(c, stride=1020) == _append(c, stride=1028) == _lib.KV_ERR_ARG
    assert _append(c, stride=(1 << 26) + 8) == _attend(c, stride=(1 << 26) + 8) == _lib.KV_ERR_ARG
    f = ctypes.byref(_cache(dtype=_lib.KV_F32))
    assert _append(f, stride=1026) == _lib.KV_ERR_ARG


def test_compact_checks():
    pr = HostProblem(lens=(4096,) * 4)
    c = _cache()
    ref = ctypes.byref(c)
    assert _compact(pr.ref(), ref, k=NULL) == _compact(pr.ref(), ref, sel=NULL) == _lib.KV_ERR_NULL
    assert _compact(pr.ref(), ref, k=ODD) == _lib.KV_ERR_ARG
    assert _compact(HostProblem(lens=(4096,)).ref(), ref) == _lib.KV_ERR_SHAPE        # other problems
    assert _compact(HostProblem(lens=(4096,) * 4, h_kv=16).ref(), ref) == _lib.KV_ERR_SHAPE
    assert _compact(HostProblem(lens=(4096,) * 4, dtype=_lib.KV_F32).ref(), ref) == _lib.KV_ERR_DTYPE
    assert _compact(pr.ref(), ref, budget=0) == _lib.KV_ERR_BUDGET
    assert _compact(pr.ref(), ref, budget=4096) == _lib.KV_ERR_BUDGET
    assert _compact(pr.ref(), ref, budget=289) == _lib.KV_ERR_SHAPE                   # 20 blocks hold 320 rows
    b = np.asarray([64, 289, 64, 64], dtype=np.int32)
    bh = ctypes.c_void_p(b.ctypes.data)
    assert _compact(pr.ref(), ref, budget=300, bh=bh, bd=P) == _lib.KV_ERR_SHAPE
    assert _compact(pr.ref(), ref, budget=300, bh=bh) == _lib.KV_ERR_NULL
    assert _compact(pr.ref(), ref, budget=200, bh=bh, bd=P) == _lib.KV_ERR_BUDGET
    big = _cache(table_stride=1000, n_blocks=5000)
    assert _compact(HostProblem(lens=(20000,) * 4).ref(), ctypes.byref(big), budget=9000) == _lib.KV_ERR_BUDGET


def test_tables_checks():
    c = ctypes.byref(_cache())
    assert _tables(c, off=NULL) == _tables(c, blk=NULL) == _tables(c, slots=NULL) == _lib.KV_ERR_NULL
    assert _tables(c, n_free=-1) == _tables(c, n_slots=-1) == _lib.KV_ERR_ARG
    for kw, code in BAD_CACHES:
        if set(kw) & {"n_prob", "block_rows", "n_blocks", "table_stride", "table", "len"}:
            assert _tables(ctypes.byref(_cache(**kw))) == code


def test_tables_overlaps():
    """Arrays that overlap in a way that the kernels do not take: every pair, an input that reaches into an
    output by one value, and an output that does into another."""
    n, n_slots, stride, n_free = 4, 10, 20, 30
    size = dict(table=n * stride, len=n, len_in=n, add=n, free=n_free, taken_in=1, taken_out=1, tok_off=n + 1,
                blk_off=n + 1, slots=n_slots)
    outs = ("table", "len", "taken_out", "tok_off", "blk_off", "slots")
    buf = np.zeros(64 * 128, np.int32)
    base = {name: buf.ctypes.data + 4 * 128 * (2 * i + 4) for i, name in enumerate(size)}

    def call(**at):
        a = dict(base, **at)
        c = _cache(n_prob=n, table_stride=stride, table=a["table"], len=a["len"])
        return _lib.lib().kv_paged_tables(ctypes.byref(c), a["len_in"], a["add"], a["free"], n_free, a["taken_in"],
                                          a["taken_out"], a["tok_off"], a["blk_off"], a["slots"], n_slots, NULL)

    taken = {("taken_in", "taken_out"), ("taken_in", "blk_off")}
    for x in size:
        for y in outs:
            if x == y:
                continue
            # x's last value on y's first one, x's first on y's last
            ends = {base[y] - 4 * (size[x] - 1), base[y] + 4 * (size[y] - 1)}
            if (x, y) in taken:
                continue
            for at in ends - ({base[y] + 4 * n} if (x, y) == ("taken_out", "blk_off") else set()):
                if {x, y} == {"taken_out", "blk_off"} and x == "blk_off" and at == base[y] - 4 * n:
                    continue  # the count is the last offset
                assert call(**{x: at}) == _lib.KV_ERR_ARG, (x, y, at - base[y])
    assert call(taken_out=base["blk_off"] + 4 * (n - 1)) == _lib.KV_ERR_ARG
    assert call(len_in=base["len"] + 4) == call(add=base["len"] - 4) == _lib.KV_ERR_ARG


def test_binding_checks():
    """Shapes and types that the binding itself refuses, on CPU tensors."""
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    sc = torch.zeros(8, 2)
    pool = torch.zeros(8, 2, 16, 64, dtype=torch.int8)
    with pytest.raises(ValueError):
        _lib.PagedCache("bf16", 4, pool.float(), pool.float(), sc, sc, table, lens)
    with pytest.raises(ValueError):
        _lib.PagedCache("bf16", 4, pool, pool, sc.double(), sc, table, lens)
    with pytest.raises(ValueError):
        _lib.PagedCache("bf16", 4, pool, pool, sc, sc, table.long(), lens)
    with pytest.raises(ValueError):
        _lib.PagedCache("bf16", 4, pool, pool, sc, sc, table, lens[:1])
    with pytest.raises(ValueError):  # host tensors
        _lib.PagedCache("bf16", 4, pool, pool, sc, sc, table, lens)
