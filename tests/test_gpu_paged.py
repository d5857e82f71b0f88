"""The 8-bit paged cache on the GPU against the definitions in float64 (oracle/paged.py).

Tables, slots, codes and scales are compared bit for bit: a scale is a power of two and a code one
rounding of an exact quotient.

Attention.  The kernels multiply exact codes with exact (or split) operands and accumulate in fp32:
  - a logit errs by at most d 2^-24 sum |q k| (any order of d products), and its scaling and the
    exponential's argument by 4 2^-24 |t|, so a weight by the factor of both and 2 2^-24 of v_exp_f32;
  - a weight enters the product with V with 16 bits (bf16 queries of up to 16 columns, 2^-16), rounded to
    bf16 (more columns, half a step of 2^-8) or with 24 bits (fp32, 2^-23);
  - sums of n terms of one sign, n 2^-24 (weights) and n 2^-24 of sum w |v| (output).
The error is at most the sum of these times sum w |v|, and for bf16 outputs half a step, 2^-8 |o|.
Below the normal numbers it is absolute: a weight (and each of its terms, at most three, and its product with the
block's scale) under 2^-126 may become 0.  The kernels' weights are 2^(t - m - o) with t - m <= o, o = 8 or
24 octaves, the largest at least 2^-24, so their sum is at least 2^-24 and a row's share of the output errs
by at most 4 2^-126 / 2^-24 (|v| + 448), 448 being the largest code: rows 2^-100 (max |v| + 448) in all.
"""
import numpy as np
import pytest

from oracle import paged
from paper_2609_30738_amd import _lib

pytestmark = pytest.mark.gpu


def _rng(*seed):
    return np.random.default_rng(seed)


def _dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _host(t):
    """A device tensor as float64 (exact for every type here)."""
    return t.double().cpu().numpy()


def _bits(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def _say(*a):
    print("[gpu case]", *a, flush=True)


def _pool(pc):
    """Fill a cache's pools and scales with what memory may hold: codes of 0x7F and NaN scales."""
    import torch
    pc.k.view(torch.uint8).fill_(0x7F)
    pc.v.view(torch.uint8).fill_(0xFF)
    pc.k_scale.fill_(float("nan"))
    pc.v_scale.fill_(float("nan"))
    return pc


def _image(pc):
    return [_bits(pc.k), _bits(pc.v)], [pc.k_scale.cpu().numpy().astype(np.float64),
                                        pc.v_scale.cpu().numpy().astype(np.float64)]


def _same_image(pc, codes, scales, where):
    got_c, got_s = _image(pc)
    for name, a, b in zip("kv", got_c, codes):
        bad = np.argwhere(a != b)
        assert bad.size == 0, f"{where}: {len(bad)} {name} codes differ, first at {bad[0]}"
    for name, a, b in zip("kv", got_s, scales):
        np.testing.assert_array_equal(a, b, err_msg=f"{where} {name} scales")


# ------------------------------------------------------------------------------------------------
# tables
# ------------------------------------------------------------------------------------------------

def _run_tables(table, n_blocks, R, len_in, add, free, taken, n_slots, in_place=False):
    t, ln = _dev(table), _dev(np.asarray(len_in, np.int32))
    out_len = ln if in_place else _dev(np.full(len(len_in), -5, np.int32))
    pc = _lib.PagedCache.for_tables(R, n_blocks, t, out_len)
    z = lambda n: _dev(np.full(n, -7, np.int32))  # noqa: E731
    tk = _dev(np.asarray([taken], np.int32))
    to, bo, sl = z(len(len_in) + 1), z(len(len_in) + 1), z(n_slots)
    _lib.paged_tables(pc, ln, _dev(np.asarray(add, np.int32)), _dev(np.asarray(free, np.int32)), tk, tk, to, bo, sl)
    return [x.cpu().numpy() for x in (t, out_len, to, bo, sl, tk)]


@pytest.mark.parametrize("n", [1, 3, 64, 65, 1024, 1025, 2300])
@pytest.mark.parametrize("R", [16, 128])
@pytest.mark.parametrize("most", [1, 5, 300])
def test_tables(n, R, most):
    """One row each, a few, and prompts (past 4096 slots a launch of its own fills them); requests without
    new rows, a padded slot map, entries that stay, lengths in place."""
    rng = _rng(n, R, most)
    stride = 2 + 700 // R
    len_in = rng.integers(0, 400, n)
    add = np.ones(n, int) if most == 1 else rng.integers(0, most + 1, n)
    n_blocks = n * stride + 10
    ids = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((n, stride), -3, np.int32)  # entries behind a request's blocks are nobody's
    at = 0
    for p in range(n):
        b = -(-len_in[p] // R)
        table[p, :b] = ids[at:at + b]
        at += b
    free, taken = ids[at - min(at, 4):], min(at, 4)
    n_slots = int(add.sum()) + 37
    want = paged.tables(table, n_blocks, R, len_in, add, free, taken, n_slots)
    for in_place in (False, True):
        _say("tables", n, R, most, in_place)
        got = _run_tables(table, n_blocks, R, len_in, add, free, taken, n_slots, in_place)
        for name, a, b in zip(("table", "len", "tok_off", "blk_off", "slots"), got, want):
            np.testing.assert_array_equal(a, b, err_msg=name)
        assert got[5][0] == want[3][-1]


TABLE_FORMS = ["apart", "count in blk_off", "count and total in blk_off", "added rows in len", "lengths in place"]


@pytest.mark.parametrize("form", TABLE_FORMS)
@pytest.mark.parametrize("n,R,most", [(1, 16, 5000), (40, 32, 300), (1024, 16, 9), (1025, 128, 300), (2300, 16, 40)])
def test_tables_of_many_rows(n, R, most, form):
    """More slots than one workgroup takes, requests past a scan of 1024: inputs that are apart from the outputs
    (several workgroups), and every one that may be an output too."""
    import torch
    rng = _rng(n, R, most, 2)
    empty = form == "added rows in len"
    add = rng.integers(0, most + 1, n)
    add[0] = most
    len_in = np.zeros(n, int) if empty else rng.integers(0, 400, n)
    stride = -(-(400 + most) // R) - 1 if n > 1 else -(-(400 + most) // R)  # the longest may pass the table
    n_blocks = int((-(-(len_in + add) // R)).sum()) + 20
    ids = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((n, stride), -3, np.int32)
    at = 0
    for p in range(n):
        b = min(-(-len_in[p] // R), stride)
        table[p, :b] = ids[at:at + b]
        at += b
    free, taken = ids[at - min(at, 4):], min(at, 4)
    n_slots = int(add.sum()) + 2100
    want = paged.tables(table, n_blocks, R, len_in, add, free, taken, n_slots)
    t, added, lens = _dev(table), _dev(add.astype(np.int32)), _dev(len_in.astype(np.int32))
    out_len = added if empty else lens if form == "lengths in place" else _dev(np.full(n, -5, np.int32))
    before = None if empty else lens
    to, bo, sl = (_dev(np.full(m, -7, np.int32)) for m in (n + 1, n + 1, n_slots))
    tk, tk_out = _dev(np.asarray([taken], np.int32)), _dev(np.asarray([-9], np.int32))
    if form.startswith("count"):
        bo[n] = taken
        tk = bo[n:]
        if "total" in form:
            tk_out = bo[n:]
    pc = _lib.PagedCache.for_tables(R, n_blocks, t, out_len)
    _say("tables", n, R, most, form)
    _lib.paged_tables(pc, before, added, _dev(free), tk, tk_out, to, bo, sl)
    for name, a, b in zip(("table", "len", "tok_off", "blk_off", "slots"), (t, out_len, to, bo, sl), want):
        np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=name)
    assert int(tk_out) == want[3][-1]
    if form == "apart":
        assert int(tk) == taken and torch.equal(lens, _dev(len_in.astype(np.int32)))
        assert torch.equal(added, _dev(add.astype(np.int32)))


def test_tables_where_the_pool_or_the_table_ends():
    """A free list too short, entries of it outside the pool, rows past the table, fewer slots than rows."""
    R, n_blocks = 16, 50
    table = np.full((4, 3), -1, np.int32)
    table[0, 0], table[3, :2] = 7, (60, 8)   # block 60 does not exist
    len_in, add = [5, 0, 0, 20], [30, 60, 16, 4]
    free = np.array([1, 2, 99, 4], np.int32)
    for n_slots in (120, 40):
        want = paged.tables(table, n_blocks, R, len_in, add, free, 0, n_slots)
        got = _run_tables(table, n_blocks, R, len_in, add, free, 0, n_slots)
        for name, a, b in zip(("table", "len", "tok_off", "blk_off", "slots"), got, want):
            np.testing.assert_array_equal(a, b, err_msg=name)
        assert want[4].min() == -1 and got[5][0] == want[3][-1] > len(free)


def test_tables_defaults():
    """Empty caches, one row each, blocks 0, 1, 2, .., nothing taken."""
    import torch
    t, ln = _dev(np.full((5, 2), -1, np.int32)), _dev(np.zeros(5, np.int32))
    pc = _lib.PagedCache.for_tables(32, 4, t, ln)
    z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    to, bo, sl = z(6), z(6), z(5)
    _lib.paged_tables(pc, None, None, None, None, None, to, bo, sl)
    assert t[:, 0].tolist() == [0, 1, 2, 3, -1] and ln.tolist() == [1] * 5
    assert sl.tolist() == [0, 32, 64, 96, -1] and to.tolist() == bo.tolist() == list(range(6))
    _lib.paged_tables(pc, ln, None, None, bo[5:], None, to, bo, sl)  # the second row needs no block
    assert sl.tolist() == [1, 33, 65, 97, -1] and ln.tolist() == [2] * 5 and bo.tolist() == [5] * 6


# ------------------------------------------------------------------------------------------------
# appending
# ------------------------------------------------------------------------------------------------

def _rows(rng, T, h_kv, d, dtype):
    """Rows of unequal size (2^-12 .. 2^6), some zero, as device tensors of `dtype`."""
    x = rng.standard_normal((T, h_kv, d)) * 2.0 ** rng.integers(-12, 7, (T, h_kv, 1))
    x[rng.random((T, h_kv)) < 0.1] = 0
    return _dev(x.astype(np.float32), _dt(dtype))


@pytest.mark.parametrize("dtype,qtype,d", [("bf16", "e4m3", 128), ("bf16", "int8", 64), ("f32", "e4m3", 64),
                                           ("f32", "int8", 128), ("bf16", "int8", 128)])
@pytest.mark.parametrize("R", [16, 32, 64, 128])
def test_append(dtype, qtype, d, R):
    """Prompts of 0 to 300 rows, then single rows and runs behind them (scales that grow and that do not),
    from contiguous rows and from slices of wider ones, with skipped slots."""
    rng = _rng(R, d, len(dtype))
    h_kv, lens = 3, [0, 1, R - 1, R, R + 1, 300, 17]
    n_blocks, stride = 40 + 7 * (420 // R + 1), 420 // R + 2
    pc = _pool(_lib.PagedCache.allocate(dtype, qtype, 6, h_kv, d, R, n_blocks, 7, stride))
    codes, scales = _image(pc)
    table = rng.permutation(n_blocks)[:7 * stride].reshape(7, stride)
    at = [0] * 7
    for step, adds in enumerate([lens, [1] * 7, [5, 0, 1, 2, 0, 40, 3], [1] * 7, [1] * 7]):
        slots = [table[p, r // R] * R + r % R for p in range(7) for r in range(at[p], at[p] + adds[p])]
        if step == 2:
            slots += [-1, n_blocks * R, -5]  # a padded batch
        T = len(slots)
        wide = _rows(rng, T, 3 * h_kv, d, dtype)
        kn, vn = (wide[:, h_kv:2 * h_kv], wide[:, 2 * h_kv:]) if step % 2 else \
            (wide[:, :h_kv].contiguous(), wide[:, h_kv:2 * h_kv].contiguous())
        _say("append", dtype, qtype, d, R, step)
        _lib.paged_append(pc, kn, vn, _dev(np.asarray(slots, np.int32)))
        for c, s, x in zip(codes, scales, (kn, vn)):
            paged.append(c, s, _host(x), np.asarray(slots), qtype)
        _same_image(pc, codes, scales, f"step {step}")
        at = [a + b for a, b in zip(at, adds)]


@pytest.mark.parametrize("qtype", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_rounds_and_saturates(dtype, qtype):
    """Midpoints of neighbouring codes and their neighbours, subnormal codes, infinities, NaN, the largest
    and the smallest numbers, and blocks of zeros."""
    import torch
    R, d = 16, 128
    grid = paged.values(np.arange(0x7F), "e4m3") if qtype == "e4m3" else np.arange(128.0)
    mid = ((grid[1:] + grid[:-1]) / 2).astype(np.float32)
    pts = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(999)), grid])
    rows = np.zeros((8 * R, 1, d), np.float32)
    flat = np.concatenate([pts, -pts])
    for i in range(4):  # the same block at four scales, its largest number pinning the scale
        part = rows[i * R:(i + 1) * R].reshape(-1)
        n = part.size - 1
        part[:n] = np.resize(flat, n + 1)[:n] if i % 2 == 0 else np.resize(flat[::-1], n + 1)[:n]
        part[n] = grid[-1]
        part *= np.float32(2.0) ** [0, -20, 60, -118][i]
    rows[4 * R, 0, :6] = [np.inf, -np.inf, np.nan, 1.0, -0.0, 3e-45]
    rows[5 * R] = np.finfo(np.float32).max
    rows[6 * R] = 1e-44
    rows[6 * R + 1, 0, ::2] = -1e-39
    rows[7 * R + 3, 0, 5] = np.nan  # alone among zeros
    x = _dev(rows, _dt(dtype))
    pc = _pool(_lib.PagedCache.allocate(dtype, qtype, 1, 1, d, R, 9, 1, 9))
    codes, scales = _image(pc)
    slots = np.arange(8 * R) + R
    _say("append values", dtype, qtype)
    _lib.paged_append(pc, x, x.clone(), _dev(slots.astype(np.int32)))
    for c, s in zip(codes, scales):
        paged.append(c, s, _host(x), slots, qtype)
    got = _bits(pc.k)
    zero = lambda c: np.where((c & 0x7F) == 0, 0, c) if qtype == "e4m3" else c  # noqa: E731  (-0 is 0)
    np.testing.assert_array_equal(zero(got), zero(codes[0]))
    np.testing.assert_array_equal(zero(_bits(pc.v)), zero(codes[1]))
    np.testing.assert_array_equal(pc.k_scale.cpu().numpy(), scales[0].astype(np.float32))
    assert torch.equal(pc.k_scale[1:], pc.v_scale[1:])


def test_append_many_requests_and_long_prompts():
    """3000 single rows (fewer waves than runs), and one prompt of 9000 rows from the middle of a block."""
    R, h_kv, d = 32, 2, 64
    rng = _rng(8)
    for T, first in ((3000, None), (9000, 7)):
        n_blocks = 3100
        pc = _pool(_lib.PagedCache.allocate("bf16", "e4m3", 2, h_kv, d, R, n_blocks, 1, 1))
        if first is None:
            slots = rng.permutation(n_blocks)[:T] * R
        else:
            pc.k_scale.fill_(2.0 ** -6)  # the first block's rows in use
            pc.v_scale.fill_(2.0 ** 3)
            pc.k.view(__import__("torch").uint8).fill_(0x31)
            pc.v.view(__import__("torch").uint8).fill_(0xB2)
            b = rng.permutation(n_blocks)
            r = first + np.arange(T)
            slots = b[r // R] * R + r % R
        codes, scales = _image(pc)
        x, y = _rows(rng, T, h_kv, d, "bf16"), _rows(rng, T, h_kv, d, "bf16")
        _say("append", T)
        _lib.paged_append(pc, x, y, _dev(slots.astype(np.int32)))
        for c, s, n in zip(codes, scales, (x, y)):
            paged.append(c, s, _host(n), slots, "e4m3")
        _same_image(pc, codes, scales, f"T={T}")


# ------------------------------------------------------------------------------------------------
# compaction
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,qtype,d", [("bf16", "e4m3", 128), ("f32", "int8", 64), ("bf16", "int8", 64),
                                           ("f32", "e4m3", 128)])
@pytest.mark.parametrize("R,budget,tail", [(16, 64, 32), (32, 1, 0), (64, 100, 7), (128, 700, 31), (16, 700, 1)])
def test_compact(dtype, qtype, d, R, budget, tail):
    """Ragged problems, budgets of their own, positions outside the problem and given twice, a missing
    block."""
    rng = _rng(R, budget, d)
    h_kv, lens = 2, [budget + tail + 5, 1501, 999]
    b = np.asarray([budget, max(1, budget // 3), budget], np.int32)
    batch = _lib.Batch(dtype, 2 * h_kv, h_kv, d, 2, lens)
    tot = sum(lens)
    k, v = _rows(rng, tot, h_kv, d, dtype), _rows(rng, tot, h_kv, d, dtype)  # any split into [h_kv][L][d]
    sel = np.full((3, h_kv, budget), -1, np.int32)
    for p in range(3):
        for g in range(h_kv):
            sel[p, g, :b[p]] = rng.permutation(lens[p] - tail)[:b[p]]
    if budget > 4:
        sel[1, 0, 1] = lens[1]          # outside
        sel[2, 1, :2] = (-1, sel[2, 1, 2])  # outside, and a position twice
    stride = -(-(budget + tail) // R) + 1
    n_blocks = 3 * stride + 5
    pc = _pool(_lib.PagedCache.allocate(dtype, qtype, 2 * h_kv, h_kv, d, R, n_blocks, 3, stride))
    table = rng.permutation(n_blocks)[:3 * stride].reshape(3, stride).astype(np.int32)
    if stride > 2:
        table[0, 1] = -1
    pc.table.copy_(_dev(table))
    codes, scales = _image(pc)
    _say("compact", dtype, qtype, d, R, budget, tail)
    _lib.paged_compact(batch, k, v, _dev(sel), budget, tail, pc, _lib.Budgets(b))
    at = 0
    for p, L in enumerate(lens):
        for c, s, x in zip(codes, scales, (k, v)):
            xp = _host(x).reshape(-1)[at * h_kv * d:(at + L) * h_kv * d].reshape(h_kv, L, d)
            paged.compact(c, s, table[p], xp, sel[p][:, :b[p]], tail, qtype)
        at += L
    _same_image(pc, codes, scales, "compact")


def test_compact_is_compaction_then_append():
    """The same codes as compacting the rows and appending them, at the largest budget."""
    import torch
    rng = _rng(77)
    R, h_kv, d, L, budget, tail = 64, 2, 128, 9000, 8192, 32
    batch = _lib.Batch("bf16", 8, h_kv, d, 32, [L])
    k, v = _rows(rng, L, h_kv, d, "bf16"), _rows(rng, L, h_kv, d, "bf16")
    sel = _dev(np.stack([rng.permutation(L - tail)[:budget] for _ in range(h_kv)]).astype(np.int32))
    rows = budget + tail
    n_blocks = -(-rows // R)
    a, b = (_pool(_lib.PagedCache.allocate("bf16", "e4m3", 8, h_kv, d, R, n_blocks, 1, n_blocks)) for _ in range(2))
    a.table.copy_(torch.arange(n_blocks, device="cuda")[None])
    _say("compact 8192")
    _lib.paged_compact(batch, k, v, sel, budget, tail, a)
    ko, vo = torch.empty(h_kv, rows, d, dtype=torch.bfloat16, device="cuda"), torch.empty(h_kv, rows, d, dtype=torch.bfloat16, device="cuda")
    _lib.compact_cache(batch, k, v, sel, budget, tail, ko, vo)
    _lib.paged_append(b, ko.transpose(0, 1).contiguous(), vo.transpose(0, 1).contiguous(),
                      torch.arange(rows, dtype=torch.int32, device="cuda"))
    for x, y in ((a.k, b.k), (a.v, b.v)):
        x, y = x.view(torch.uint8).reshape(n_blocks, h_kv, R, d), y.view(torch.uint8).reshape(n_blocks, h_kv, R, d)
        assert torch.equal(x, y)
    assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------

def _cache(rng, dtype, qtype, h_q, h_kv, d, R, lens, spare=3, max_len=None, amp=1.0):
    """Random codes and scales in used rows, not-a-number codes and scales everywhere else."""
    import torch
    lens = np.asarray(lens)
    stride = max(1, -(-int(lens.max()) // R)) + 1
    n_blocks = int(sum(-(-L // R) for L in lens)) + spare
    pc = _pool(_lib.PagedCache.allocate(dtype, qtype, h_q, h_kv, d, R, n_blocks, len(lens), stride,
                                        int(lens.max()) if max_len is None else max_len))
    ids, at = rng.permutation(n_blocks), 0
    table = np.full((len(lens), stride), -1, np.int32)
    kc, vc = _bits(pc.k), _bits(pc.v)
    ks, vs = np.full((n_blocks, h_kv), np.nan, np.float32), np.full((n_blocks, h_kv), np.nan, np.float32)
    for p, L in enumerate(lens):
        for j in range(-(-int(L) // R)):
            b = table[p, j] = ids[at]
            at += 1
            n = min(R, int(L) - j * R)
            for c, s in ((kc, ks), (vc, vs)):
                x = rng.standard_normal((h_kv, n, d)) * amp
                if c is kc:
                    x *= np.where(rng.random((h_kv, n, 1)) < 0.02, 4.0, 1.0)
                for g in range(h_kv):
                    s[b, g] = paged.least_scale(paged.finite_max(x[g]), qtype)
                    c[b, g, :n] = paged.encode(x[g], float(s[b, g]), qtype)
    pc.k.view(torch.uint8).copy_(_dev(kc))
    pc.v.view(torch.uint8).copy_(_dev(vc))
    pc.k_scale.copy_(_dev(ks))
    pc.v_scale.copy_(_dev(vs))
    pc.table.copy_(_dev(table))
    pc.lens.copy_(_dev(lens.astype(np.int32)))
    return pc


def _attend(pc, q, scale, n_q=None, max_q=None, fill=7.0):
    """One call on q [T, h_q, d]; n_q: tokens per problem (None: one each)."""
    import torch
    out = torch.full(q.shape, fill, dtype=q.dtype, device="cuda")
    off = None if n_q is None else _dev(np.concatenate([[0], np.cumsum(n_q)]).astype(np.int32))
    max_q = 1 if n_q is None else int(max(1, max(n_q))) if max_q is None else max_q
    nb = _lib.paged_attention_workspace_bytes(pc, q.shape[0], max_q)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda") if nb else None
    _lib.paged_attention(pc, q, scale, out, off, max_q, ws)
    return out


def _check(pc, q, scale, n_q, out, where, max_q=None):
    """Every token's output against float64, within the bounds derived above."""
    dtype, qtype = pc.dtype_name, "e4m3" if pc.struct.qtype == _lib.KV_E4M3 else "int8"
    codes, scales = _image(pc)
    table, lens = pc.table.cpu().numpy(), pc.lens.cpu().numpy()
    qh, oh, d = _host(q), _host(out), pc.struct.d
    cap = min(table.shape[1] * pc.struct.block_rows, pc.struct.max_len)
    n_q = np.ones(len(lens), int) if n_q is None else np.asarray(n_q)
    at, eps = 0, 2.0 ** -24
    cols = max(1, int(n_q.max()) if max_q is None else max_q) * pc.struct.h_q // pc.struct.h_kv
    weight = 2.0 ** -23 if dtype == "f32" else 2.0 ** -16 if cols <= 16 else 2.0 ** -8
    for p, (L, n) in enumerate(zip(lens, n_q)):
        if n:
            rows = min(int(L), cap)
            k, has = paged.cache_rows(codes[0], scales[0], table[p], rows, qtype)
            v, _ = paged.cache_rows(codes[1], scales[1], table[p], rows, qtype)
            k, v = np.where(has[:, None], k, 0.0), np.where(has[:, None], v, 0.0)
            ref, mag, qk = paged.attention(qh[at:at + n], k, v, has, scale, int(L))
            rel = 2 * (d + 4) * eps * qk + (2 * rows + 8) * eps + weight
            bound = rel * mag + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else eps * np.abs(ref))
            bound = bound + rows * 2.0 ** -100 * ((np.nanmax(np.abs(v)) if rows else 0.0) + 448)
            got = oh[at:at + n]
            assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{where} p={p}: NaN in other places"
            err = np.abs(np.nan_to_num(got) - np.nan_to_num(ref)) - np.nan_to_num(bound)
            assert np.all(err <= 0), (f"{where} p={p} L={L} n={n}: off by {np.nanmax(np.abs(got - ref)):.3g}, over the "
                                      f"bound by {err.max():.3g} at {np.unravel_index(np.argmax(err), err.shape)}")
        at += n
    if at < q.shape[0]:
        assert np.all(oh[at:] == 7.0), f"{where}: rows behind the last token were written"


TYPES = [("bf16", "e4m3", 128), ("bf16", "int8", 64), ("f32", "e4m3", 64), ("f32", "int8", 128), ("bf16", "int8", 128),
         ("bf16", "e4m3", 64), ("f32", "e4m3", 128), ("f32", "int8", 64)]


def _q(rng, T, h_q, d, dtype):
    return _dev(rng.standard_normal((T, h_q, d)).astype(np.float32), _dt(dtype))


@pytest.mark.parametrize("dtype,qtype,d", TYPES)
@pytest.mark.parametrize("R", [16, 32, 64, 128])
@pytest.mark.parametrize("h_q,h_kv", [(8, 2), (3, 3), (32, 2), (5, 1)])
def test_attention_one_token(dtype, qtype, d, R, h_q, h_kv):
    """Lengths of 0, 1 and around a tile, a step, a wave's round, a block and a split."""
    rng = _rng(R, h_q, d, len(dtype))
    lens = [0, 1, 15, 16, 17, 31, 33, 128, 129, 300, 511]
    pc = _cache(rng, dtype, qtype, h_q, h_kv, d, R, lens)
    q = _q(rng, len(lens), h_q, d, dtype)
    _say("attention", dtype, qtype, d, R, h_q, h_kv)
    out = _attend(pc, q, d ** -0.5)
    _check(pc, q, d ** -0.5, None, out, "one token")
    assert not out[0].any()  # nothing to attend to


@pytest.mark.parametrize("dtype,qtype,d", TYPES)
@pytest.mark.parametrize("R", [16, 64])
def test_attention_split_rows(dtype, qtype, d, R):
    """Caches of up to 3000 rows in several splits, unequal lengths, one empty and one of a single row."""
    rng = _rng(R, d, 5)
    lens = [2999, 0, 1, 640, 1281, 127]
    pc = _cache(rng, dtype, qtype, 8, 2, d, R, lens)
    assert _lib.paged_attention_workspace_bytes(pc) > 0
    q = _q(rng, 6, 8, d, dtype)
    _say("attention splits", dtype, qtype, d, R)
    _check(pc, q, d ** -0.5, None, _attend(pc, q, d ** -0.5), "splits")


@pytest.mark.parametrize("dtype,qtype,d", TYPES)
@pytest.mark.parametrize("G", [1, 4, 16])
def test_attention_several_tokens(dtype, qtype, d, G):
    """Up to 9 tokens a problem: none, one, all rows of a cache, more tokens than rows (the first ones see
    nothing), a padded batch; G = 16 with 9 tokens takes several groups of columns."""
    rng = _rng(G, d, 6)
    lens, n_q = [40, 0, 9, 700, 4, 33], [3, 0, 9, 8, 7, 1]
    pc = _cache(rng, dtype, qtype, 2 * G, 2, d, 32, lens)
    q = _q(rng, sum(n_q) + 2, 2 * G, d, dtype)
    _say("attention tokens", dtype, qtype, d, G)
    _check(pc, q, d ** -0.5, n_q, _attend(pc, q, d ** -0.5, n_q), "tokens")


@pytest.mark.parametrize("dtype,qtype,d", TYPES)
@pytest.mark.parametrize("R,G", [(16, 4), (64, 4), (128, 1), (32, 8)])
def test_attention_prompt_turn(dtype, qtype, d, R, G):
    """Turns of up to 333 tokens over caches of up to 900 rows, and a whole prompt (as many tokens as rows)."""
    rng = _rng(R, G, d, 7)
    lens, n_q = [900, 333, 50, 0, 401], [130, 333, 1, 0, 64]
    pc = _cache(rng, dtype, qtype, 2 * G, 2, d, R, lens)
    q = _q(rng, sum(n_q) + 3, 2 * G, d, dtype)
    _say("attention turn", dtype, qtype, d, R, G)
    _check(pc, q, d ** -0.5, n_q, _attend(pc, q, d ** -0.5, n_q), "turn")


@pytest.mark.parametrize("qtype,d,h_q,n_tok", [("e4m3", 128, 16, 40), ("int8", 128, 8, 33), ("e4m3", 64, 64, 70)])
def test_attention_turns_of_many_problems(qtype, d, h_q, n_tok):
    """Enough problems that no rows are split: ragged lengths and tokens, a padded batch, negative and zero
    scales."""
    rng = _rng(d, h_q)
    n = 66
    lens = rng.integers(0, 200, n)
    n_q = np.minimum(rng.integers(0, n_tok + 1, n), lens)
    n_q[7] = n_tok
    pc = _cache(rng, "bf16", qtype, h_q, 8, d, 32, lens)
    assert _lib.paged_attention_workspace_bytes(pc, int(n_q.sum()) + 1, n_tok) == 0
    q = _q(rng, int(n_q.sum()) + 1, h_q, d, "bf16")
    for scale in (d ** -0.5, -0.2, 0.0):
        _say("attention many turns", qtype, d, h_q, scale)
        _check(pc, q, scale, n_q, _attend(pc, q, scale, n_q), f"many turns {scale}")


def test_attention_turn_over_more_blocks_than_a_split_holds():
    """5000 rows in blocks of 16 are more than a split of the four-wave prompt kernel takes (256 blocks): two
    splits although the batch fills the chip."""
    rng = _rng(31)
    lens = np.full(40, 30)
    lens[[3, 17]] = 5000, 4097
    n_q = np.zeros(40, int)
    n_q[[3, 9, 17]] = 12, 5, 3
    pc = _cache(rng, "bf16", "e4m3", 32, 8, 64, 16, lens)
    q = _q(rng, 20, 32, 64, "bf16")
    need = _lib.paged_attention_workspace_bytes(pc, 20, 12)
    assert need == -(-20 * 32 * 2 * 66 * 4 // 256) * 256
    _say("attention many blocks")
    _check(pc, q, 0.125, n_q, _attend(pc, q, 0.125, n_q), "many blocks")


@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_missing_blocks(dtype, n):
    """Entries outside the pool in the middle, at the end and for a whole request: their rows are not seen."""
    rng = _rng(9, n)
    lens = [300, 200, 90, 2000]
    pc = _cache(rng, dtype, "e4m3", 8, 2, 128, 32, lens)
    pc.table[0, 3] = -1
    pc.table[1, 6] = 1 << 30
    pc.table[2] = pc.struct.n_blocks
    pc.table[3, 10:20] = -(1 << 31)
    n_q = [n] * 4
    q = _q(rng, 4 * n, 8, 128, dtype)
    _say("attention missing", dtype, n)
    _check(pc, q, 0.09, n_q, _attend(pc, q, 0.09, n_q), "missing")


@pytest.mark.parametrize("n", [1, 4, 90])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_attention_nan_rows(dtype, d, n):
    """A NaN in a row's V or K reaches the tokens that see the row, and no others."""
    rng = _rng(10, n)
    lens = [200, 170, 100]
    pc = _cache(rng, dtype, "e4m3", 4, 2, d, 16, lens)
    import torch
    k, v = pc.k.view(torch.uint8), pc.v.view(torch.uint8)
    at = lambda p, r: (int(pc.table[p, r // 16]), r % 16)  # noqa: E731
    b, r = at(0, 200 - (n + 1) // 2)
    v[b, 1, r, 5] = 0x7F
    v[b, 1, r, 40] = 0xFF
    b, r = at(1, 169)
    k[b, 0, r, 3] = 0x7F
    b, r = at(2, 99)
    v[b, :, r, 0] = 0xFF
    q = _q(rng, 3 * n, 4, d, dtype)
    _say("attention nan", dtype, n)
    out = _attend(pc, q, 0.1, [n] * 3)
    _check(pc, q, 0.1, [n] * 3, out, "nan")
    assert torch.isnan(out).any() and not torch.isnan(out).all()


def test_attention_of_nan_queries_and_scales():
    """A NaN query gives NaN outputs in its token and head alone; a block of zeros has scale 0."""
    import torch
    rng = _rng(11)
    pc = _cache(rng, "bf16", "e4m3", 4, 2, 128, 16, [100, 700])
    b = int(pc.table[1, 2])
    pc.k.view(torch.uint8)[b] = 0
    pc.v.view(torch.uint8)[b] = 0
    pc.k_scale[b] = 0
    pc.v_scale[b] = 0
    q = _q(rng, 2, 4, 128, "bf16")
    q[1, 2, 7] = float("nan")
    for ml in (700, 1200):  # with and without splits
        pc.struct.max_len = ml
        out = _attend(pc, q, 0.1)
        assert torch.isnan(out[1, 2]).all() and not torch.isnan(out[0]).any() and not torch.isnan(out[1, [0, 1, 3]]).any()
    q[1, 2, 7] = 0
    _check(pc, q, 0.1, None, _attend(pc, q, 0.1), "zeros")


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 6, 40, 200])
def test_attention_of_queries_that_are_no_numbers(dtype, n, split):
    """NaN and infinite queries, over whole rows and over splits, for every kernel: NaN in their tokens and heads
    alone."""
    import torch
    rng = _rng(43, n)
    lens = [210, 700 if split else 450]
    pc = _cache(rng, dtype, "e4m3", 4, 2, 128, 16, lens)
    n_q = [n, max(1, n - 1)]
    q = _q(rng, sum(n_q), 4, 128, dtype)
    assert (_lib.paged_attention_workspace_bytes(pc, len(q), n) > 0) == split
    bad = torch.zeros(len(q), 4, dtype=torch.bool, device="cuda")
    for t, h, x in ((0, 2, np.nan), (n // 2, 1, np.inf), (len(q) - 1, 3, -np.inf), (len(q) - 1, 0, np.nan)):
        q[t, h, (7 * t + h) % 128] = x
        bad[t, h] = True
    _say("attention NaN queries", dtype, n, split)
    out = _attend(pc, q, 0.1, n_q)
    assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
    q[bad] = 0.5
    same = _attend(pc, q, 0.1, n_q)
    _check(pc, q, 0.1, n_q, torch.where(bad[..., None], same, out), "the others")


@pytest.mark.parametrize("profile", ["rising", "alternating", "late"])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dtype,qtype,d", [("bf16", "e4m3", 64), ("bf16", "int8", 128), ("bf16", "e4m3", 128),
                                           ("f32", "e4m3", 64)])
def test_attention_of_moving_logits(dtype, qtype, d, split, profile):
    """Logits that move by tens of octaves from one 32 rows to the next, up for some columns of a wave and
    down or hardly at all for others: the reference moves again and again, between tiles and between the
    halves of one.  Few tokens, and turns that four and eight waves take."""
    import torch
    rng = _rng(44, d)
    L = 900 if split else 470
    pc = _cache(rng, dtype, qtype, 4, 1, d, 32, [L, L - 45])
    u = np.where(rng.random(d) < 0.5, -1.0, 1.0)
    codes, _ = _image(pc)
    pc.k_scale.fill_(0.5)
    for p, rows in enumerate(pc.lens.tolist()):
        half = np.arange(rows) // 32
        if profile == "rising":
            level = -60 + 120.0 * half / half.max()
        elif profile == "alternating":
            level = np.where(half % 2 == 0, 60.0, -60.0) * (0.5 + 0.5 * half / half.max())
        else:
            level = np.where(np.arange(rows) < rows - 30, -60.0, 60.0)
        for r in range(rows):
            t = int(pc.table[p, r // 32])
            codes[0][t, 0, r % 32] = paged.encode(u * (level[r] + rng.integers(-2, 3, d)), 1.0, qtype)
    pc.k.view(torch.uint8).copy_(_dev(codes[0]))
    for n in (1, 9, 30, 90):
        n_q = [n, max(1, n - 4)]
        amp = rng.choice([1.0, -1.0, 0.5, 0.125, -0.03125], (sum(n_q), 4, 1))
        q = _dev((u * amp).astype(np.float32), _dt(dtype))
        assert (_lib.paged_attention_workspace_bytes(pc, len(q), n) > 0) == split
        scale = 16.0 / d
        _say("attention moving", dtype, qtype, d, split, profile, n)
        out = _attend(pc, q, scale, n_q)
        _check(pc, q, scale, n_q, out, f"{profile} n={n}")
        assert torch.equal(out, _attend(pc, q, scale, n_q))  # the same bits again


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("dtype,qtype,d,R,G", [("bf16", "e4m3", 128, 16, 4), ("bf16", "int8", 64, 64, 4),
                                               ("bf16", "int8", 128, 32, 1), ("f32", "e4m3", 64, 32, 4)])
def test_attention_of_other_scales(dtype, qtype, d, R, G, which):
    """Scales that are no powers of two (another coder's): taken as they are for up to 32 columns and fp32; a
    turn of more gives NaN to the tokens that see the block, and to no others."""
    import torch
    rng = _rng(33, d, R)
    L, j = 333, 3
    for n, max_len in ((2, None), (8, 2000), (L, None), (L, 4000)):
        pc = _cache(rng, dtype, qtype, 2 * G, 2, d, R, [L, 90])
        if max_len:
            wide = torch.full((2, max_len // R), -1, dtype=torch.int32, device="cuda")
            wide[:, :pc.table.shape[1]] = pc.table
            pc = _lib.PagedCache(dtype, 2 * G, pc.k, pc.v, pc.k_scale, pc.v_scale, wide, pc.lens, max_len)
        b = int(pc.table[0, j])
        scale = pc.k_scale if which == "k" else pc.v_scale
        scale[b] *= 1.37
        n_q = [n, min(n, 90)]
        q = _q(rng, sum(n_q), 2 * G, d, dtype)
        _say("attention other scales", dtype, qtype, d, R, which, n, max_len)
        out = _attend(pc, q, 0.1, n_q)
        if dtype == "f32" or n * G <= 32:
            _check(pc, q, 0.1, n_q, out, "as they are")
            continue
        sees = torch.arange(n, device="cuda") + L - n >= j * R
        assert torch.isnan(out[:n][sees]).all() and not torch.isnan(out[:n][~sees]).any()
        m = int((~sees).sum())  # the tokens before the block are a turn of their own
        pc.lens[0] = m
        _check(pc, torch.cat([q[:m], q[n:]]), 0.1, [m, n_q[1]], torch.cat([out[:m], out[n:]]), "before it", max_q=n)


@pytest.mark.parametrize("qtype,d", [("e4m3", 128), ("int8", 64)])
@pytest.mark.parametrize("n", [200, 30])
def test_attention_beside_the_largest_values(qtype, d, n):
    """A block of values that round to 2^128, an infinity in bf16 and fp32 (rows of the type's lowest value, say):
    NaN to the tokens of a turn that see it, nothing to the ones before it in the same tile."""
    import torch
    rng = _rng(45, d)
    L, R = 200, 16
    pc = _cache(rng, "bf16", qtype, 8, 2, d, R, [L, 90])
    low = torch.full((L, 2, d), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16, device="cuda")
    row = torch.randn(L, 2, d, device="cuda").to(torch.bfloat16)
    j = 11
    slots = int(pc.table[0, j]) * R + torch.arange(R, dtype=torch.int32, device="cuda")
    _lib.paged_append(pc, row[:R], low[:R], slots)
    n_q = [n, min(n, 90)]
    q = _q(rng, sum(n_q), 8, d, "bf16")
    _say("attention largest values", qtype, d, n)
    out = _attend(pc, q, 0.1, n_q)
    sees = torch.arange(n, device="cuda") + L - n >= j * R
    assert sees.any() and not sees.all()
    assert torch.isnan(out[:n][sees]).all() and torch.isfinite(out[:n][~sees]).all()
    m = int((~sees).sum())
    pc.lens[0] = L - n + m
    _check(pc, torch.cat([q[:m], q[n:]]), 0.1, [m, n_q[1]], torch.cat([out[:m], out[n:]]), "before it", max_q=n)


@pytest.mark.parametrize("dtype,qtype", [("bf16", "e4m3"), ("f32", "int8")])
def test_attention_rising_logits(dtype, qtype):
    """Logits that rise by tens of octaves along the rows: the reference is raised many times."""
    rng = _rng(12)
    pc = _cache(rng, dtype, qtype, 4, 1, 64, 32, [1000, 260])
    q = _q(rng, 2, 4, 64, dtype)
    codes, _ = _image(pc)
    import torch
    u = np.sign(_host(q)[0, 0])
    for p, L in ((0, 1000), (1, 260)):
        for r in range(L):
            t = int(pc.table[p, r // 32])
            codes[0][t, 0, r % 32] = paged.encode(u * np.linspace(-60, 60, L)[r], 1.0, qtype)
            pc.k_scale[t] = 0.5
    pc.k.view(torch.uint8).copy_(_dev(codes[0]))
    _say("attention rising", dtype, qtype)
    _check(pc, q, 0.1, None, _attend(pc, q, 0.1), "rising")
    _check(pc, q, -0.1, None, _attend(pc, q, -0.1), "falling")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_attention_of_large_values(dtype, d):
    """Values of 2^118 in every row: the sums stay finite, and the output is 2^118."""
    import torch
    rng = _rng(13)
    for n in (1, 40):
        pc = _cache(rng, dtype, "e4m3", 4, 2, d, 16, [400, 3000])
        pc.v.view(torch.uint8).fill_(0x70)  # 128
        pc.v_scale.fill_(2.0 ** 111)
        q = _q(rng, 2 * n, 4, d, dtype)
        _say("attention large", dtype, n)
        out = _attend(pc, q, 0.1, [n] * 2)
        np.testing.assert_allclose(_host(out), 2.0 ** 118, rtol=2.0 ** -8 if dtype == "bf16" else 1e-4)


def test_attention_strided_queries_and_wide_bounds():
    """Queries as slices of a projection's output; max_len and max_q above what the batch needs, tok_off with
    a problem outside the call's rows."""
    import torch
    rng = _rng(14)
    pc = _cache(rng, "bf16", "e4m3", 8, 2, 128, 32, [300, 64, 900], max_len=5000)
    wide = _q(rng, 12, 12, 128, "bf16")
    q = wide[:, :8]
    n_q = [5, 3, 2]
    out = _attend(pc, q, 0.08, n_q, max_q=11)
    _check(pc, q, 0.08, n_q, out, "strided", max_q=11)
    plain = _attend(pc, q.contiguous(), 0.08, n_q, max_q=11)
    assert torch.equal(out, plain)
    off = torch.tensor([0, 5, 13, 13], dtype=torch.int32, device="cuda")  # the second reaches past 12 rows
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    ws = torch.empty(max(256, _lib.paged_attention_workspace_bytes(pc, 12, 11)), dtype=torch.uint8, device="cuda")
    _lib.paged_attention(pc, q, 0.08, o, off, 11, ws)
    assert torch.equal(o[:5], out[:5]) and (o[5:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_q,max_len", [(2, 300), (2, 2000), (9, 300), (9, 2000)])
def test_attention_of_offsets_that_are_none(dtype, max_q, max_len):
    """Offsets that fall, by so much that the number of columns leaves 32 bits, or lie anywhere: the problems
    between them are left out, and the ones beside them are not."""
    import torch
    rng = _rng(41, max_q)
    lens = [40, 50, 60, 33, 70, 80, 90]
    pc = _cache(rng, dtype, "e4m3", 32, 2, 64, 16, lens, max_len=max_len)
    if max_len > 300:  # splits: a table of as many blocks
        wide = torch.full((len(lens), 125), -1, dtype=torch.int32, device="cuda")
        wide[:, :pc.table.shape[1]] = pc.table
        pc = _lib.PagedCache(dtype, 32, pc.k, pc.v, pc.k_scale, pc.v_scale, wide, pc.lens, max_len)
    q = _q(rng, 12, 32, 64, dtype)
    big = (1 << 27) + 1
    off = torch.tensor([0, 2, big, 0, (1 << 31) - 1, -(1 << 31), 10, 12], dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    nb = _lib.paged_attention_workspace_bytes(pc, 12, max_q)
    assert (nb > 0) == (max_len > 1000)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
    _say("attention offsets", dtype, max_q, max_len)
    _lib.paged_attention(pc, q, 0.1, out, off, max_q, ws)
    assert (out[2:10] == 7).all()
    first = _lib.PagedCache(dtype, 32, pc.k, pc.v, pc.k_scale, pc.v_scale, pc.table[:1], pc.lens[:1], max_len)
    last = _lib.PagedCache(dtype, 32, pc.k, pc.v, pc.k_scale, pc.v_scale, pc.table[6:], pc.lens[6:], max_len)
    _check(first, q[:2], 0.1, [2], out[:2], "first", max_q)
    _check(last, q[10:], 0.1, [2], out[10:], "last", max_q)


def test_binding_refuses_overlapping_tokens_and_other_types():
    import torch
    rng = _rng(32)
    pc = _cache(rng, "bf16", "e4m3", 4, 2, 64, 16, [20, 30])
    q = _q(rng, 2, 4, 64, "bf16")
    out = torch.empty_like(q)
    rows = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (q[:1].expand(2, 4, 64), q.float(), q[:, :2], q.transpose(0, 1).contiguous().transpose(0, 1), q.cpu()):
        with pytest.raises(ValueError):
            _lib.paged_attention(pc, bad, 0.1, out)
    for bad in (out.float(), out[:1], torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda")[:, :4]):
        with pytest.raises(ValueError):
            _lib.paged_attention(pc, q, 0.1, bad)
    with pytest.raises(ValueError):
        _lib.paged_append(pc, rows, rows[:1], slots)
    with pytest.raises(ValueError):
        _lib.paged_append(pc, rows, rows, slots.long())
    with pytest.raises(ValueError):
        _lib.paged_append(pc, rows, torch.zeros(2, 6, 64, dtype=torch.bfloat16, device="cuda")[:, :2], slots)
    with pytest.raises(_lib.KvError):  # a workspace too small
        pc.struct.max_len = 30
        far = _lib.PagedCache("bf16", 4, pc.k, pc.v, pc.k_scale, pc.v_scale, torch.zeros(2, 400, dtype=torch.int32, device="cuda"), pc.lens)
        _lib.paged_attention(far, q, 0.1, out, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))


def test_streams(monkeypatch):
    """The current stream and one that is given, with torch's raw stream query and without it."""
    import torch
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(2):
        pc = _lib.PagedCache.for_tables(16, 4, _dev(np.zeros((2, 2), np.int32)), _dev(np.zeros(2, np.int32)))
        with torch.cuda.stream(side):
            assert pc._stream(None) == side.cuda_stream and pc._stream(other) == other.cuda_stream
        assert pc._stream(None) == torch.cuda.current_stream().cuda_stream
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)


def test_steps_without_tokens():
    """A step in which no request gets a row: tables, appending and attention take it, and change nothing;
    arguments of other types are refused all the same."""
    import torch
    rng = _rng(42)
    pc = _cache(rng, "bf16", "e4m3", 4, 2, 64, 16, [20, 30])
    codes, scales = _image(pc)
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    to, bo = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2))
    slots = torch.empty(0, dtype=torch.int32, device="cuda")
    qkv = torch.empty(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    _say("no tokens")
    _lib.paged_tables(pc, pc.lens, none, None, None, None, to, bo, slots)
    _lib.paged_append(pc, qkv[:, 4:6], qkv[:, 6:], slots)
    _lib.paged_attention(pc, qkv[:, :4], 0.1, out, to, 1)
    assert pc.lens.tolist() == [20, 30] and to.tolist() == bo.tolist() == [0, 0, 0]
    _same_image(pc, codes, scales, "no tokens")
    with pytest.raises(ValueError):
        _lib.paged_append(pc, qkv[:, 4:6].float(), qkv[:, 6:], slots)
    with pytest.raises(ValueError):
        _lib.paged_attention(pc, qkv[:, :4], 0.1, out.float(), to, 1)
    with pytest.raises(_lib.KvError):  # one token each, and there are none
        _lib.paged_attention(pc, qkv[:, :4], 0.1, out)


def test_attention_past_32_bit_offsets():
    """Blocks whose codes lie past 4 GiB of the pool, written and read."""
    import torch
    h_kv, R, d = 8, 128, 128
    n_blocks = (1 << 32) // (h_kv * R * d) + 40
    rng = _rng(15)
    pc = _lib.PagedCache.allocate("bf16", "e4m3", 16, h_kv, d, R, n_blocks, 2, 5)
    lens = [600, 333]
    far = n_blocks - 1 - np.arange(10).reshape(2, 5)
    pc.table.copy_(_dev(far.astype(np.int32)))
    pc.lens.copy_(_dev(np.asarray(lens, np.int32)))
    slots = np.concatenate([far[p, np.arange(L) // R] * R + np.arange(L) % R for p, L in enumerate(lens)])
    x, y = (_dev(rng.standard_normal((sum(lens), h_kv, d)).astype(np.float32), torch.bfloat16) for _ in range(2))
    _say("attention past 4 GiB", n_blocks)
    _lib.paged_append(pc, x, y, _dev(slots.astype(np.int32)))
    q = _q(rng, 4, 16, d, "bf16")
    out = _attend(pc, q, 0.09, [3, 1])
    lo = n_blocks - 10
    near = _lib.PagedCache("bf16", 16, pc.k[lo:].clone(), pc.v[lo:].clone(), pc.k_scale[lo:].clone(),
                           pc.v_scale[lo:].clone(), pc.table - lo, pc.lens, pc.struct.max_len)
    codes, scales = [np.zeros((10, h_kv, R, d), np.uint8) for _ in range(2)], [np.zeros((10, h_kv)) for _ in range(2)]
    for c, s, n in zip(codes, scales, (x, y)):
        paged.append(c, s, _host(n), slots - lo * R, "e4m3")
    used = np.zeros((10, R), bool)
    used.reshape(-1)[slots - lo * R] = True
    for c, pool in zip(codes, (near.k, near.v)):
        assert np.array_equal(_bits(pool)[used[:, None].repeat(h_kv, 1)], c[used[:, None].repeat(h_kv, 1)])
    _check(near, q, 0.09, [3, 1], out, "far blocks")


# ------------------------------------------------------------------------------------------------
# together
# ------------------------------------------------------------------------------------------------

def test_serving_run():
    """Prompts, an eviction of one request's worth of rows, generated tokens and a further turn: tables,
    appending, compaction and attention together, on a stream of its own, every step against float64."""
    import torch
    rng = _rng(20)
    h_q, h_kv, d, R, qtype = 8, 2, 128, 16, "e4m3"
    n, stride, n_blocks = 3, 40, 100
    pc = _lib.PagedCache.allocate("bf16", qtype, h_q, h_kv, d, R, n_blocks, n, stride, 640)
    free = _dev(rng.permutation(n_blocks).astype(np.int32))
    taken = torch.zeros(1, dtype=torch.int32, device="cuda")
    to, bo = (torch.empty(n + 1, dtype=torch.int32, device="cuda") for _ in range(2))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        L, budget, tail = 400, 50, 8
        batch = _lib.Batch("bf16", h_q, h_kv, d, 8, [L] * n)
        k, v = _rows(rng, n * L, h_kv, d, "bf16"), _rows(rng, n * L, h_kv, d, "bf16")
        sel = _dev(np.stack([[rng.permutation(L - tail)[:budget] for _ in range(h_kv)] for _ in range(n)]).astype(np.int32))
        b = np.asarray([50, 31, 9], np.int32)
        add = _dev(b + tail)
        _lib.paged_tables(pc, None, add, free, taken, taken, to, bo, torch.empty(n * 60, dtype=torch.int32, device="cuda"))
        _lib.paged_compact(batch, k, v, sel, budget, tail, pc, _lib.Budgets(b))
        for step, adds in enumerate([[1, 1, 1], [1, 1, 1], [40, 0, 150], [1, 1, 1], [4, 5, 6]]):
            T = sum(adds)
            slots = torch.empty(T + 1, dtype=torch.int32, device="cuda")
            _lib.paged_tables(pc, pc.lens, _dev(np.asarray(adds, np.int32)), free, taken, taken, to, bo, slots)
            qkv = _dev(rng.standard_normal((T + 1, h_q + 2 * h_kv, d)).astype(np.float32), torch.bfloat16)
            _lib.paged_append(pc, qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:], slots)
            q = qkv[:, :h_q]
            out = torch.full((T + 1, h_q, d), 7.0, dtype=torch.bfloat16, device="cuda")
            nb = _lib.paged_attention_workspace_bytes(pc, T + 1, max(adds))
            ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
            _lib.paged_attention(pc, q, d ** -0.5, out, to, max(adds), ws)
            stream.synchronize()
            _say("run step", step, pc.lens.tolist())
            _check(pc, q, d ** -0.5, adds, out, f"step {step}")
    assert pc.lens.tolist() == [int(x) + tail + a for x, a in zip(b, (47, 8, 159))]
    used = sum(-(-x // R) for x in pc.lens.tolist())
    assert int(taken) == used


def test_captured_step():
    """A generation step (tables, append, attention) captured once and replayed with other tokens, other
    work between the replays: the lengths and tables advance on the device, and every replay equals the
    eager calls."""
    import torch
    rng = _rng(21)
    h_q, h_kv, d, R, n, stride = 8, 2, 64, 16, 5, 60
    lens = [3, 15, 16, 500, 901]
    a = _cache(rng, "bf16", "int8", h_q, h_kv, d, R, lens, spare=40, max_len=960)
    b = _lib.PagedCache("bf16", h_q, a.k.clone(), a.v.clone(), a.k_scale.clone(), a.v_scale.clone(), a.table.clone(),
                        a.lens.clone(), 960)
    used = set(a.table[a.table >= 0].tolist())
    free = _dev(np.asarray([i for i in range(a.struct.n_blocks) if i not in used], np.int32))
    qkv = torch.zeros(n, h_q + 2 * h_kv, d, dtype=torch.bfloat16, device="cuda")

    def buffers(pc):
        z = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")  # noqa: E731
        nb = _lib.paged_attention_workspace_bytes(pc)
        assert nb > 0
        return dict(taken=z(1), to=z(n + 1), bo=z(n + 1), slots=z(n),
                    out=torch.zeros(n, h_q, d, dtype=torch.bfloat16, device="cuda"),
                    ws=torch.empty(nb, dtype=torch.uint8, device="cuda"))

    def step(pc, x):
        _lib.paged_tables(pc, pc.lens, None, free, x["taken"], x["taken"], x["to"], x["bo"], x["slots"])
        _lib.paged_append(pc, qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:], x["slots"])
        _lib.paged_attention(pc, qkv[:, :h_q], 0.125, x["out"], ws=x["ws"])

    xa, xb = buffers(a), buffers(b)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(a, xa)
    torch.cuda.synchronize()
    assert a.lens.tolist() == lens  # capture ran nothing
    for i in range(20):
        qkv.copy_(_dev(rng.standard_normal(qkv.shape).astype(np.float32) * 2.0 ** (i % 5), torch.bfloat16))
        graph.replay()
        other = torch.randn(300, 300, device="cuda") @ torch.randn(300, 300, device="cuda")
        step(b, xb)
        torch.cuda.synchronize()
        del other
        for name in ("taken", "to", "bo", "slots", "out"):
            assert torch.equal(xa[name], xb[name]), (i, name)
        assert torch.equal(a.lens, b.lens) and torch.equal(a.table, b.table)
        if i % 7 == 0:
            _check(a, qkv[:, :h_q], 0.125, None, xa["out"], f"replay {i}")
    assert a.lens.tolist() == [x + 20 for x in lens]


@pytest.mark.parametrize("n", [4, 60])
def test_captured_turns_share_a_workspace(n):
    """Two captured calls of several tokens each that share a workspace (one after the other on their stream),
    replayed three times over other queries with eager work between, against eager calls."""
    import torch
    rng = _rng(22, n)
    h_q, h_kv, d = 8, 2, 128
    pcs = [_cache(rng, "bf16", "e4m3", h_q, h_kv, d, 32, lens) for lens in ([1500, 300], [900, 1200])]
    n_q = [n, n - 1]
    T = 2 * n - 1
    off = _dev(np.asarray([0, n, T], np.int32))
    q = [_q(rng, T, h_q, d, "bf16") for _ in range(2)]
    out = [torch.zeros_like(x) for x in q]
    need = max(_lib.paged_attention_workspace_bytes(pc, T, n) for pc in pcs)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            for pc, x, o in zip(pcs, q, out):
                _lib.paged_attention(pc, x, 0.09, o, off, n, ws)
    torch.cuda.synchronize()
    for i in range(3):
        for x in q:
            x.copy_(_q(rng, T, h_q, d, "bf16"))
        _say("captured turns", n, i)
        graph.replay()
        torch.cuda.synchronize()
        for pc, x, o in zip(pcs, q, out):
            assert torch.equal(_attend(pc, x, 0.09, n_q), o), i
    _check(pcs[1], q[1], 0.09, n_q, out[1], "captured")
