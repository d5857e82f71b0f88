"""The 4-bit paged cache on the GPU against the definitions in float64 (oracle/paged.py), and reading caches of every code
type back.

Codes, scales and rows that are read back are compared bit for bit.  Attention: the kernels multiply codes times their
scales, which are exact in bf16, with exact (or split) operands and accumulate in fp32, as over 8 bits: the bounds of
test_gpu_paged.py hold as they are derived there, with 6 for the largest code.
"""
import numpy as np
import pytest

from oracle import paged
from paper_2609_30738_amd import _lib
from tests.test_gpu_paged import _attend, _bits, _dev, _dt, _host, _q, _rng, _rows, _say

pytestmark = pytest.mark.gpu


def _fill(pc):
    """A cache's pools as memory may leave them: every byte 0xFF (codes of -6, scales that are no numbers)."""
    import torch
    for t in (pc.k, pc.v, pc.k_scale, pc.v_scale):
        t.view(torch.uint8).fill_(0xFF)
    return pc


def _image4(pc):
    return [_bits(pc.k), _bits(pc.v)], [_bits(pc.k_scale), _bits(pc.v_scale)]


def _same(pc, codes, scales, where):
    got_c, got_s = _image4(pc)
    for what, got, want in (("codes", got_c, codes), ("scales", got_s, scales)):
        for name, a, b in zip("kv", got, want):
            bad = np.argwhere(a != b)
            assert bad.size == 0, f"{where}: {len(bad)} {name} {what} differ, first at {bad[0]}"


# ------------------------------------------------------------------------------------------------
# writing
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("R", [16, 32, 64, 128])
def test_append(dtype, d, R):
    """Prompts of 0 to 300 rows, then single rows and runs behind them, from contiguous rows and from slices of wider
    ones, with skipped slots; other rows stay as they were."""
    rng = _rng(R, d, len(dtype), 4)
    h_kv, lens = 3, [0, 1, R - 1, R, R + 1, 300, 17]
    stride = 420 // R + 2
    n_blocks = 40 + 7 * stride
    pc = _fill(_lib.PagedCache.allocate(dtype, "e2m1", 6, h_kv, d, R, n_blocks, 7, stride))
    codes, scales = _image4(pc)
    table = rng.permutation(n_blocks)[:7 * stride].reshape(7, stride)
    at = [0] * 7
    for step, adds in enumerate([lens, [1] * 7, [5, 0, 1, 2, 0, 40, 3], [1] * 7]):
        slots = [table[p, r // R] * R + r % R for p in range(7) for r in range(at[p], at[p] + adds[p])]
        if step == 2:
            slots += [-1, n_blocks * R, -5]  # a padded batch
        T = len(slots)
        wide = _rows(rng, T, 3 * h_kv, d, dtype)
        kn, vn = (wide[:, h_kv:2 * h_kv], wide[:, 2 * h_kv:]) if step % 2 else \
            (wide[:, :h_kv].contiguous(), wide[:, h_kv:2 * h_kv].contiguous())
        _say("append4", dtype, d, R, step)
        _lib.paged_append(pc, kn, vn, _dev(np.asarray(slots, np.int32)))
        for c, s, x in zip(codes, scales, (kn, vn)):
            paged.append4(c, s, _host(x), np.asarray(slots))
        _same(pc, codes, scales, f"step {step}")
        at = [a + b for a, b in zip(at, adds)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [16, 64])
def test_append_in_any_order(dtype, R):
    """Tokens in no order of their slots, single ones of many blocks, rows written again."""
    rng = _rng(R, 5)
    n_blocks, T = 30, 400
    pc = _fill(_lib.PagedCache.allocate(dtype, "e2m1", 2, 2, 64, R, n_blocks, 1, 1))
    codes, scales = _image4(pc)
    for _ in range(2):
        slots = rng.permutation(n_blocks * R)[:T]
        x, y = _rows(rng, T, 2, 64, dtype), _rows(rng, T, 2, 64, dtype)
        _say("append4 any order", dtype, R)
        _lib.paged_append(pc, x, y, _dev(slots.astype(np.int32)))
        for c, s, n in zip(codes, scales, (x, y)):
            paged.append4(c, s, _host(n), slots)
    _same(pc, codes, scales, "any order")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_rounds_and_saturates(dtype):
    """Midpoints of neighbouring codes and their neighbours at many scales, infinities, NaN, the largest and the smallest
    numbers, groups of zeros."""
    R, d = 16, 128
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float32)
    mid = (grid[1:] + grid[:-1]) / 2
    eps = np.float32(2.0 ** -7 if dtype == "bf16" else 2.0 ** -23)
    pts = np.concatenate([grid, mid, mid * (1 - eps), mid * (1 + eps), grid * (1 + eps), grid * (1 - eps)])
    rows = np.zeros((8 * R, 1, d), np.float32)
    flat = np.concatenate([pts, -pts])
    for i, e in enumerate((0, -20, 60, -118, 100, -124)):
        part = rows[i * R:(i + 1) * R].reshape(-1, 32)
        part[:, 1:] = np.resize(flat, (part.shape[0], 31))
        part[:, 0] = 6
        part *= np.float32(2.0) ** e
    rows[6 * R, 0, :6] = [np.inf, -np.inf, np.nan, 1.0, -0.0, 3e-45]
    rows[6 * R, 0, 40] = np.nan  # alone among zeros
    rows[6 * R, 0, 70] = -np.inf
    rows[6 * R + 1] = np.finfo(np.float32).max
    rows[6 * R + 1, 0, 5] = -1.0
    rows[6 * R + 2] = 1e-44
    rows[6 * R + 3, 0, ::2] = -1e-39
    rows[6 * R + 4, 0, 96:] = 6 * 2.0 ** 125
    rows[6 * R + 5] = np.nan
    x = _dev(rows, _dt(dtype))
    pc = _fill(_lib.PagedCache.allocate(dtype, "e2m1", 1, 1, d, R, 9, 1, 9))
    codes, scales = _image4(pc)
    slots = np.arange(8 * R) + R
    _say("append4 values", dtype)
    _lib.paged_append(pc, x, x.clone(), _dev(slots.astype(np.int32)))
    for c, s in zip(codes, scales):
        paged.append4(c, s, _host(x), slots)
    _same(pc, codes, scales, "values")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("R,budget,tail", [(16, 64, 32), (32, 1, 0), (64, 100, 7), (128, 700, 31), (16, 700, 1)])
def test_compact(dtype, d, R, budget, tail):
    """Ragged problems, budgets of their own, positions outside the problem and given twice, a missing block."""
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
        sel[1, 0, 1] = lens[1]
        sel[2, 1, :2] = (-1, sel[2, 1, 2])
    stride = -(-(budget + tail) // R) + 1
    n_blocks = 3 * stride + 5
    pc = _fill(_lib.PagedCache.allocate(dtype, "e2m1", 2 * h_kv, h_kv, d, R, n_blocks, 3, stride))
    table = rng.permutation(n_blocks)[:3 * stride].reshape(3, stride).astype(np.int32)
    if stride > 2:
        table[0, 1] = -1
    pc.table.copy_(_dev(table))
    codes, scales = _image4(pc)
    _say("compact4", dtype, d, R, budget, tail)
    _lib.paged_compact(batch, k, v, _dev(sel), budget, tail, pc, _lib.Budgets(b))
    at = 0
    for p, L in enumerate(lens):
        for c, s, x in zip(codes, scales, (k, v)):
            xp = _host(x).reshape(-1)[at * h_kv * d:(at + L) * h_kv * d].reshape(h_kv, L, d)
            paged.compact4(c, s, table[p], xp, sel[p][:, :b[p]], tail)
        at += L
    _same(pc, codes, scales, "compact")


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------

def _cache4(rng, dtype, h_q, h_kv, d, R, lens, spare=3, max_len=None, stride=None):
    """Random codes and scales in used rows, bytes of 0xFF everywhere else."""
    import torch
    lens = np.asarray(lens)
    stride = max(1, -(-int(lens.max()) // R)) + 1 if stride is None else stride
    n_blocks = int(sum(-(-L // R) for L in lens)) + spare
    pc = _fill(_lib.PagedCache.allocate(dtype, "e2m1", h_q, h_kv, d, R, n_blocks, len(lens), stride,
                                        int(lens.max()) if max_len is None else max_len))
    ids, at = rng.permutation(n_blocks), 0
    table = np.full((len(lens), stride), -1, np.int32)
    codes, scales = _image4(pc)
    for p, L in enumerate(lens):
        for j in range(-(-int(L) // R)):
            b = table[p, j] = ids[at]
            at += 1
            n = min(R, int(L) - j * R)
            for c, s in zip(codes, scales):
                c[b, :, :n] = rng.integers(0, 256, (h_kv, n, d // 2))
                s[b, :, :, :n] = 125 + rng.integers(-3, 2, (h_kv, d // 32, n))
            if rng.random() < 0.3:
                scales[0][b, :, :, rng.integers(n)] += 2  # a key that stands out
    for t, x in zip((pc.k, pc.v, pc.k_scale, pc.v_scale), codes + scales):
        t.view(torch.uint8).copy_(_dev(x))
    pc.table.copy_(_dev(table))
    pc.lens.copy_(_dev(lens.astype(np.int32)))
    return pc


def _check4(pc, q, scale, n_q, out, where, max_q=None):
    """Every token's output against float64, within the bounds derived in test_gpu_paged.py."""
    dtype = pc.dtype_name
    codes, scales = _image4(pc)
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
            (k, has), (v, _) = (paged.cache_rows4(c, s, table[p], rows) for c, s in zip(codes, scales))
            k, v = np.where(has[:, None], k, 0.0), np.where(has[:, None], v, 0.0)
            ref, mag, qk = paged.attention(qh[at:at + n], k, v, has, scale, int(L))
            rel = 2 * (d + 4) * eps * qk + (2 * rows + 8) * eps + weight
            bound = rel * mag + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else eps * np.abs(ref))
            bound = bound + rows * 2.0 ** -100 * ((np.abs(v).max() if rows else 0.0) + 6)
            err = np.abs(oh[at:at + n] - ref) - bound
            assert np.all(err <= 0), (f"{where} p={p} L={L} n={n}: over the bound by {np.max(err):.3g} at "
                                      f"{np.unravel_index(np.argmax(err), err.shape)}")
        at += n
    if at < q.shape[0]:
        assert np.all(oh[at:] == 7.0), f"{where}: rows behind the last token were written"


TYPES = [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("R", [16, 32, 64, 128])
@pytest.mark.parametrize("h_q,h_kv", [(8, 2), (3, 3), (32, 2), (5, 1)])
def test_attention_one_token(dtype, d, R, h_q, h_kv):
    """Lengths of 0, 1 and around a tile, a step, a wave's round, a block and a split."""
    rng = _rng(R, h_q, d, len(dtype))
    lens = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 128, 129, 255, 257, 300, 511]
    pc = _cache4(rng, dtype, h_q, h_kv, d, R, lens)
    q = _q(rng, len(lens), h_q, d, dtype)
    _say("attention4", dtype, d, R, h_q, h_kv)
    out = _attend(pc, q, d ** -0.5)
    _check4(pc, q, d ** -0.5, None, out, "one token")
    assert not out[0].any()  # nothing to attend to


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("R", [16, 64])
def test_attention_split_rows(dtype, d, R):
    """Caches of up to 3000 rows in several splits, unequal lengths, one empty and one of a single row."""
    rng = _rng(R, d, 5)
    lens = [2999, 0, 1, 640, 1281, 127]
    pc = _cache4(rng, dtype, 8, 2, d, R, lens)
    assert _lib.paged_attention_workspace_bytes(pc) > 0
    q = _q(rng, 6, 8, d, dtype)
    _say("attention4 splits", dtype, d, R)
    out = _attend(pc, q, d ** -0.5)
    _check4(pc, q, d ** -0.5, None, out, "splits")
    assert __import__("torch").equal(out, _attend(pc, q, d ** -0.5))  # the same bits again


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("G", [1, 4, 16])
def test_attention_several_tokens(dtype, d, G):
    """Up to 9 tokens a problem: none, one, all rows of a cache, more tokens than rows (the first ones see nothing), a
    padded batch; G = 16 with 9 tokens takes several groups of columns."""
    rng = _rng(G, d, 6)
    lens, n_q = [40, 0, 9, 700, 4, 33], [3, 0, 9, 8, 7, 1]
    pc = _cache4(rng, dtype, 2 * G, 2, d, 32, lens)
    q = _q(rng, sum(n_q) + 2, 2 * G, d, dtype)
    _say("attention4 tokens", dtype, d, G)
    _check4(pc, q, d ** -0.5, n_q, _attend(pc, q, d ** -0.5, n_q), "tokens")


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("R,G", [(16, 4), (64, 4), (128, 1), (32, 8)])
def test_attention_prompt_turn(dtype, d, R, G):
    """Turns of up to 333 tokens over caches of up to 900 rows, and a whole prompt (as many tokens as rows)."""
    rng = _rng(R, G, d, 7)
    lens, n_q = [900, 333, 50, 0, 401], [130, 333, 1, 0, 64]
    pc = _cache4(rng, dtype, 2 * G, 2, d, R, lens)
    q = _q(rng, sum(n_q) + 3, 2 * G, d, dtype)
    _say("attention4 turn", dtype, d, R, G)
    _check4(pc, q, d ** -0.5, n_q, _attend(pc, q, d ** -0.5, n_q), "turn")


@pytest.mark.parametrize("d,h_q,n_tok", [(128, 16, 40), (128, 8, 33), (64, 64, 70), (64, 24, 14)])
def test_attention_turns_of_many_problems(d, h_q, n_tok):
    """Enough problems that no rows are split: ragged lengths and tokens, a padded batch, negative and zero scales."""
    rng = _rng(d, h_q)
    n = 66
    lens = rng.integers(0, 200, n)
    n_q = np.minimum(rng.integers(0, n_tok + 1, n), lens)
    n_q[7] = n_tok
    pc = _cache4(rng, "bf16", h_q, 8, d, 32, lens)
    q = _q(rng, int(n_q.sum()) + 1, h_q, d, "bf16")
    for scale in (d ** -0.5, -0.2, 0.0):
        _say("attention4 many turns", d, h_q, scale)
        _check4(pc, q, scale, n_q, _attend(pc, q, scale, n_q), f"many turns {scale}")


@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_missing_blocks(dtype, n):
    """Entries outside the pool in the middle, at the end and for a whole request: their rows are not seen."""
    rng = _rng(9, n)
    lens = [300, 200, 90, 2000]
    pc = _cache4(rng, dtype, 8, 2, 128, 32, lens)
    pc.table[0, 3] = -1
    pc.table[1, 6] = 1 << 30
    pc.table[2] = pc.struct.n_blocks
    pc.table[3, 10:20] = -(1 << 31)
    q = _q(rng, 4 * n, 8, 128, dtype)
    _say("attention4 missing", dtype, n)
    _check4(pc, q, 0.09, [n] * 4, _attend(pc, q, 0.09, [n] * 4), "missing")


@pytest.mark.parametrize("n", [1, 6, 40, 200])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_attention_any_scale_byte(dtype, d, n):
    """The ends of the scales' range in rows that some tokens see and others do not: bytes 0 and 1 (next to nothing) in keys
    and values; in masked rows 0xFF and 252.  A value of the largest scale in a visible row stays with the tokens that see
    it."""
    import torch
    rng = _rng(21, n)
    L = 210
    pc = _cache4(rng, dtype, 4, 2, d, 16, [L, 170])
    ks, vs = pc.k_scale.view(torch.uint8), pc.v_scale.view(torch.uint8)
    at = lambda p, r: (int(pc.table[p, r // 16]), r % 16)  # noqa: E731
    for r in (3, 100, L - 1):
        b, i = at(0, r)
        ks[b, :, 0, i], vs[b, 1, :, i] = 0, 1
    q = _q(rng, 2 * n, 4, d, dtype)
    _say("attention4 scales", dtype, n)
    _check4(pc, q, 0.1, [n] * 2, _attend(pc, q, 0.1, [n] * 2), "small scales")
    last = at(0, L - 1)
    before = _attend(pc, q, 0.1, [n] * 2)
    vs[last[0], :, :, last[1]] = 255  # never written: infinities, NaN or a large value
    pc.v.view(torch.uint8)[last[0], :, last[1]] = 0x77
    out = _attend(pc, q, 0.1, [n] * 2)
    others = torch.arange(2 * n, device="cuda") != n - 1  # the last token of the first problem sees the row
    assert torch.equal(out[others], before[others])



@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 6, 40, 200])
def test_attention_of_queries_that_are_no_numbers(dtype, n, split):
    """NaN and infinite queries, over whole rows and over splits, for every kernel: NaN in their tokens and heads
    alone."""
    import torch
    rng = _rng(43, n)
    pc = _cache4(rng, dtype, 4, 2, 128, 16, [210, 700 if split else 450])
    n_q = [n, max(1, n - 1)]
    q = _q(rng, sum(n_q), 4, 128, dtype)
    assert (_lib.paged_attention_workspace_bytes(pc, len(q), n) > 0) == split
    bad = torch.zeros(len(q), 4, dtype=torch.bool, device="cuda")
    for t, h, x in ((0, 2, np.nan), (n // 2, 1, np.inf), (len(q) - 1, 3, -np.inf), (len(q) - 1, 0, np.nan)):
        q[t, h, (7 * t + h) % 128] = x
        bad[t, h] = True
    _say("attention4 NaN queries", dtype, n, split)
    out = _attend(pc, q, 0.1, n_q)
    assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
    q[bad] = 0.5
    same = _attend(pc, q, 0.1, n_q)
    _check4(pc, q, 0.1, n_q, torch.where(bad[..., None], same, out), "the others")


@pytest.mark.parametrize("profile", ["rising", "alternating", "late"])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_attention_of_moving_logits(dtype, d, split, profile):
    """Logits that move by tens of octaves from one 32 rows to the next, up for some columns of a wave and down or hardly
    at all for others: the reference moves again and again."""
    import torch
    rng = _rng(44, d)
    L = 900 if split else 470
    pc = _cache4(rng, dtype, 4, 1, d, 32, [L, L - 45])
    u = np.where(rng.random(d) < 0.5, -1.0, 1.0)
    codes, scales = _image4(pc)
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
            codes[0][t, 0, r % 32], scales[0][t, 0, :, r % 32] = paged.encode4(u * (level[r] + rng.integers(-2, 3, d)) / 2)
    pc.k.view(torch.uint8).copy_(_dev(codes[0]))
    pc.k_scale.view(torch.uint8).copy_(_dev(scales[0]))
    for n in (1, 9, 30, 90):
        n_q = [n, max(1, n - 4)]
        amp = rng.choice([1.0, -1.0, 0.5, 0.125, -0.03125], (sum(n_q), 4, 1))
        q = _dev((u * amp).astype(np.float32), _dt(dtype))
        scale = 16.0 / d
        _say("attention4 moving", dtype, d, split, profile, n)
        out = _attend(pc, q, scale, n_q)
        _check4(pc, q, scale, n_q, out, f"{profile} n={n}")
        assert torch.equal(out, _attend(pc, q, scale, n_q))


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("scale", [-0.2, 0.0, -1e-40, 3.0])
def test_attention_of_any_scale(dtype, d, n, scale):
    """Negative, zero, denormal and large scales; short caches and ones of several rounds."""
    rng = _rng(d, n, 31)
    for lens in ([70, 300, 9], [1500, 0, 640]):
        pc = _cache4(rng, dtype, 8, 2, d, 32, lens)
        q = _q(rng, 3 * n, 8, d, dtype)
        _say("attention4 scale", dtype, d, n, scale, lens)
        _check4(pc, q, scale, [n] * 3, _attend(pc, q, scale, [n] * 3), f"scale {scale} {lens}")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("n", [257, 600, 1025])
@pytest.mark.parametrize("tokens", [1, 5])
def test_attention_of_many_unequal_problems(dtype, d, n, tokens):
    """More requests than a wave looks at at once, most of a few rows or none and some long ones, the first and the last
    among them, requests without tokens between: shares begin and end in any of them."""
    rng = _rng(n, d, tokens)
    lens = np.where(rng.random(n) < 0.2, 0, rng.integers(1, 40, n))
    lens[[0, 255, 256, n - 1]] = 700, 1, 2500, 641
    pc = _cache4(rng, dtype, 4, 1, d, 16, lens)
    n_q = None if tokens == 1 else rng.integers(0, tokens + 1, n)
    if tokens > 1:
        n_q[[0, n - 1]] = tokens
    T = n if n_q is None else int(n_q.sum())
    q = _q(rng, T, 4, d, dtype)
    assert _lib.paged_attention_workspace_bytes(pc, T, tokens) > 0
    _say("attention4 many unequal", dtype, d, n, tokens)
    _check4(pc, q, 0.1, n_q, _attend(pc, q, 0.1, n_q), "many unequal", tokens)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("n", [230, 600])
@pytest.mark.parametrize("tokens", [1, 3])
def test_attention_of_more_problems_than_shares(dtype, d, n, tokens):
    """Many more requests than the workgroups that share a kv head's rows: short ones, empty ones, ones without tokens, long
    ones that several workgroups share beside each other, at the start and at the end."""
    rng = _rng(n, d, tokens, 7)
    lens = np.where(rng.random(n) < 0.1, 0, rng.integers(1, 200, n))
    lens[[0, 100, 101, 102, n - 1]] = 1900, 5000, 129, 3001, 1400
    pc = _cache4(rng, dtype, 16, 8, d, 32, lens)
    n_q = None if tokens == 1 else rng.integers(0, tokens + 1, n)
    if tokens > 1:
        n_q[[0, 100, 101, n - 1]] = tokens
    T = n if n_q is None else int(n_q.sum())
    q = _q(rng, T, 16, d, dtype)
    _say("attention4 many problems", dtype, d, n, tokens)
    out = _attend(pc, q, 0.1, n_q)
    _check4(pc, q, 0.1, n_q, out, "many problems", tokens)
    assert __import__("torch").equal(out, _attend(pc, q, 0.1, n_q))


def test_attention_of_as_many_columns_as_the_chip_holds():
    """256 fp32 tokens of 32 heads: a workgroup to a kv head's 32 columns goes over all problems, and nothing is joined."""
    rng = _rng(33)
    pc = _cache4(rng, "f32", 32, 8, 128, 64, [1300, 0, 290], max_len=1400)
    n_q = [256, 0, 40]
    q = _q(rng, 300, 32, 128, "f32")
    assert _lib.paged_attention_workspace_bytes(pc, 300, 256) > 0
    _say("attention4 many columns")
    _check4(pc, q, 0.09, n_q, _attend(pc, q, 0.09, n_q), "many columns")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_q", [2, 9])
@pytest.mark.parametrize("max_len", [300, 2000])
def test_attention_of_offsets_that_are_none(dtype, max_q, max_len):
    """Offsets that fall, by so much that the number of columns leaves 32 bits, or lie anywhere: the problems between them
    are left out, and the ones beside them are not."""
    import torch
    rng = _rng(41, max_q)
    pc = _cache4(rng, dtype, 32, 2, 64, 16, [40, 50, 60, 33, 70, 80, 90], max_len=max_len, stride=125)
    q = _q(rng, 12, 32, 64, dtype)
    off = torch.tensor([0, 2, (1 << 27) + 1, 0, (1 << 31) - 1, -(1 << 31), 10, 12], dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    nb = _lib.paged_attention_workspace_bytes(pc, 12, max_q)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda") if nb else None
    _say("attention4 offsets", dtype, max_q, max_len)
    _lib.paged_attention(pc, q, 0.1, out, off, max_q, ws)
    assert (out[2:10] == 7).all()
    for at, p in ((slice(0, 2), slice(0, 1)), (slice(10, 12), slice(6, 7))):
        one = _lib.PagedCache(dtype, 32, pc.k, pc.v, pc.k_scale, pc.v_scale, pc.table[p], pc.lens[p], max_len)
        _check4(one, q[at], 0.1, [2], out[at], "beside", max_q)


def test_attention_turn_over_more_blocks_than_a_split_holds():
    """5000 rows in blocks of 16: two splits although the batch fills the chip."""
    rng = _rng(31)
    lens = np.full(40, 30)
    lens[[3, 17]] = 5000, 4097
    n_q = np.zeros(40, int)
    n_q[[3, 9, 17]] = 12, 5, 3
    pc = _cache4(rng, "bf16", 32, 8, 64, 16, lens)
    q = _q(rng, 20, 32, 64, "bf16")
    _say("attention4 many blocks")
    _check4(pc, q, 0.125, n_q, _attend(pc, q, 0.125, n_q), "many blocks")


def test_attention_strided_queries_and_wide_bounds():
    """Queries as slices of a projection's output; max_len and max_q above what the batch needs, tok_off with a problem
    outside the call's rows."""
    import torch
    rng = _rng(14)
    pc = _cache4(rng, "bf16", 8, 2, 128, 32, [300, 64, 900], max_len=5000, stride=157)
    wide = _q(rng, 12, 12, 128, "bf16")
    q = wide[:, :8]
    n_q = [5, 3, 2]
    out = _attend(pc, q, 0.08, n_q, max_q=11)
    _check4(pc, q, 0.08, n_q, out, "strided", max_q=11)
    assert torch.equal(out, _attend(pc, q.contiguous(), 0.08, n_q, max_q=11))
    off = torch.tensor([0, 5, 13, 13], dtype=torch.int32, device="cuda")  # the second reaches past 12 rows
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    ws = torch.empty(max(256, _lib.paged_attention_workspace_bytes(pc, 12, 11)), dtype=torch.uint8, device="cuda")
    _lib.paged_attention(pc, q, 0.08, o, off, 11, ws)
    assert torch.equal(o[:5], out[:5]) and (o[5:] == 7).all()


def test_past_32_bit_offsets():
    """Blocks whose codes lie past 4 GiB of the pool: written, attended to and read back."""
    import torch
    h_kv, R, d = 8, 128, 128
    n_blocks = (1 << 32) // (h_kv * R * d // 2) + 40
    rng = _rng(15)
    pc = _lib.PagedCache.allocate("bf16", "e2m1", 16, h_kv, d, R, n_blocks, 2, 5)
    lens = [600, 333]
    far = n_blocks - 1 - np.arange(10).reshape(2, 5)
    pc.table.copy_(_dev(far.astype(np.int32)))
    pc.lens.copy_(_dev(np.asarray(lens, np.int32)))
    slots = np.concatenate([far[p, np.arange(L) // R] * R + np.arange(L) % R for p, L in enumerate(lens)])
    x, y = (_dev(rng.standard_normal((sum(lens), h_kv, d)).astype(np.float32), torch.bfloat16) for _ in range(2))
    _say("past 4 GiB", n_blocks)
    _lib.paged_append(pc, x, y, _dev(slots.astype(np.int32)))
    q = _q(rng, 4, 16, d, "bf16")
    out = _attend(pc, q, 0.09, [3, 1])
    lo = n_blocks - 10
    at = lambda t: t.view(torch.uint8)[lo:].clone().view(t.dtype)  # noqa: E731
    near = _lib.PagedCache("bf16", 16, at(pc.k), at(pc.v), at(pc.k_scale), at(pc.v_scale), pc.table - lo, pc.lens,
                           pc.struct.max_len)
    codes, scales = _image4(near)
    want_c, want_s = [c.copy() for c in codes], [s.copy() for s in scales]
    for c, s, n in zip(want_c, want_s, (x, y)):
        paged.append4(c, s, _host(n), slots - lo * R)
    _same(near, want_c, want_s, "far blocks")
    _check4(near, q, 0.09, [3, 1], out, "far blocks")
    off = _dev(np.array([0, 600, 933], np.int64))
    rows = [torch.empty(933 * h_kv * d, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    _lib.paged_rows(pc, off, rows[0], rows[1])
    _lib.paged_rows(near, off, rows[2], rows[3])
    assert torch.equal(rows[0], rows[2]) and torch.equal(rows[1], rows[3])


# ------------------------------------------------------------------------------------------------
# reading back
# ------------------------------------------------------------------------------------------------

def _cache_of(rng, dtype, qtype, h_kv, d, R, lens, **kw):
    if qtype == "e2m1":
        return _cache4(rng, dtype, 2 * h_kv, h_kv, d, R, lens, **kw)
    from tests.test_gpu_paged import _cache
    return _cache(rng, dtype, qtype, 2 * h_kv, h_kv, d, R, lens, **kw)


def _rows_of(pc, p, n):
    """Rows of problem p by the oracle, zeros where it has none: [2][h_kv, n, d]."""
    table, L = pc.table.cpu().numpy()[p], int(pc.lens[p])
    out = []
    for c, s in ((pc.k, pc.k_scale), (pc.v, pc.v_scale)):
        if pc.struct.qtype == _lib.KV_E2M1:
            x, has = paged.cache_rows4(_bits(c), _bits(s), table, min(n, L))
        else:
            x, has = paged.cache_rows(_bits(c), s.cpu().numpy(), table, min(n, L), "e4m3" if pc.struct.qtype == _lib.KV_E4M3 else "int8")
        full = np.zeros((x.shape[0], n, x.shape[2]))
        full[:, :min(n, L)] = np.where(has[:, None], x, 0.0)
        out.append(full)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("qtype", ["e2m1", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("R", [16, 32, 128])
def test_rows(dtype, qtype, d, R):
    """Whole caches, fewer rows than a cache holds, more (zeros), none, missing blocks; problems whose offsets are none are
    left out, and nothing else is written.  The values are exact in every type."""
    import torch
    rng = _rng(R, d, len(qtype))
    h_kv, lens = 3, [70, 1, 0, 200, 129, 64, 40]
    pc = _cache_of(rng, dtype, qtype, h_kv, d, R, lens, max_len=230)
    pc.table[3, 1] = -1
    pc.table[4, 0] = 1 << 29
    take = [70, 1, 5, 220, 100, 0, 0]
    off = np.concatenate([[0], np.cumsum(take)])
    n = int(off[-1])
    k, v = (torch.full(((n + 3) * h_kv * d,), 7.0, dtype=_dt(dtype), device="cuda") for _ in range(2))
    _say("rows", dtype, qtype, d, R)
    _lib.paged_rows(pc, _dev(off.astype(np.int64)), k, v)
    for p, m in enumerate(take):
        want = _rows_of(pc, p, m)
        for got, w, name in zip((k, v), want, "kv"):
            part = _host(got)[off[p] * h_kv * d:off[p + 1] * h_kv * d].reshape(h_kv, m, d)
            np.testing.assert_array_equal(part, w, err_msg=f"{name} of {p}")
    assert (k[n * h_kv * d:] == 7).all() and (v[n * h_kv * d:] == 7).all()
    # offsets that fall, span more than max_len or leave the output
    k2, v2 = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    bad = np.array([0, 70, 60, 60 + 300, 1 << 40, -(1 << 40), 10, 1 << 62], np.int64)
    _lib.paged_rows(pc, _dev(bad), k2, None)
    _lib.paged_rows(pc, _dev(bad), None, v2)
    m = 70 * h_kv * d
    for got, full in ((k2, k), (v2, v)):
        assert torch.equal(got[:m], full[:m]) and (got[m:] == 7).all()


def test_rows_of_other_scales():
    """8-bit blocks of another coder's scales: code times scale, rounded once."""
    import torch
    rng = _rng(51)
    for dtype in ("bf16", "f32"):
        pc = _cache_of(rng, dtype, "int8", 2, 64, 16, [50])
        pc.k_scale *= 1.37
        k = torch.empty(50 * 2 * 64, dtype=_dt(dtype), device="cuda")
        _lib.paged_rows(pc, _dev(np.array([0, 50], np.int64)), k, None)
        codes = pc.k[pc.table[0].long().clamp(min=0)]
        want = codes.float() * pc.k_scale[pc.table[0].long().clamp(min=0)][..., None, None]
        want = want.transpose(0, 1).reshape(2, -1, 64)[:, :50].to(_dt(dtype))
        assert torch.equal(k.view(2, 50, 64), want)


def test_rows_binding_refuses():
    import torch
    rng = _rng(52)
    pc = _cache_of(rng, "bf16", "e2m1", 2, 64, 16, [50])
    off = _dev(np.array([0, 50], np.int64))
    k = torch.empty(50 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    for args, kw in (((off.int(), k, k), {}), ((off[:1], k, k), {}), ((off, k.float(), k), {}), ((off, None, None), {}),
                     ((off, k[:100], k), dict(n_rows=50)), ((off, k.cpu(), k), {})):
        with pytest.raises(ValueError):
            _lib.paged_rows(pc, *args, **kw)


# ------------------------------------------------------------------------------------------------
# together
# ------------------------------------------------------------------------------------------------

def test_serving_run():
    """An eviction into 4 bits, generated tokens and a further turn with rotated queries and keys, on a stream of its own,
    every step against float64; then the caches read back and evicted again by the whole pass."""
    import torch
    rng = _rng(20)
    h_q, h_kv, d, R = 8, 2, 128, 16
    n, stride, n_blocks, L0 = 3, 40, 130, 400
    pc = _fill(_lib.PagedCache.allocate("bf16", "e2m1", h_q, h_kv, d, R, n_blocks, n, stride, 640))
    f, factor = _lib.rotary_frequencies("yarn", 64, 1e4, (4.0, 256.0, 32.0, 1.0))
    rot = _lib.Rotary("half", _dev(f), factor)
    free = _dev(rng.permutation(n_blocks).astype(np.int32))
    taken = torch.zeros(1, dtype=torch.int32, device="cuda")
    to, bo = (torch.empty(n + 1, dtype=torch.int32, device="cuda") for _ in range(2))
    codes, scales = _image4(pc)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        budget, tail = 50, 8
        batch = _lib.Batch("bf16", h_q, h_kv, d, 8, [L0] * n)
        k, v = _rows(rng, n * L0, h_kv, d, "bf16"), _rows(rng, n * L0, h_kv, d, "bf16")
        sel = _dev(np.stack([[rng.permutation(L0 - tail)[:budget] for _ in range(h_kv)] for _ in range(n)]).astype(np.int32))
        b = np.asarray([50, 31, 9], np.int32)
        _lib.paged_tables(pc, None, _dev(b + tail), free, taken, taken, to, bo, torch.empty(n * 60, dtype=torch.int32, device="cuda"))
        _lib.paged_compact(batch, k, v, sel, budget, tail, pc, _lib.Budgets(b))
        seen = np.full(n, L0)  # positions: those of the whole text, not the rows kept
        for step, adds in enumerate([[1, 1, 1], [1, 1, 1], [40, 0, 150], [1, 1, 1], [4, 5, 6]]):
            T = sum(adds)
            slots = torch.empty(T + 1, dtype=torch.int32, device="cuda")
            _lib.paged_tables(pc, pc.lens, _dev(np.asarray(adds, np.int32)), free, taken, taken, to, bo, slots)
            pos = np.concatenate([seen[p] + np.arange(a) for p, a in enumerate(adds)] + [[0]]).astype(np.int32)
            seen = seen + adds
            qkv = _dev(rng.standard_normal((T + 1, h_q + 2 * h_kv, d)).astype(np.float32), torch.bfloat16)
            q = qkv[:, :h_q]
            _lib.paged_append_rotated(pc, rot, _dev(pos), qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:], slots, q=q, q_out=q)
            out = torch.full((T + 1, h_q, d), 7.0, dtype=torch.bfloat16, device="cuda")
            nb = _lib.paged_attention_workspace_bytes(pc, T + 1, max(adds))
            ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
            _lib.paged_attention(pc, q, d ** -0.5, out, to, max(adds), ws)
            stream.synchronize()
            _say("run step", step, pc.lens.tolist())
            _check4(pc, q, d ** -0.5, adds, out, f"step {step}")
        lens = pc.lens.tolist()
        assert lens == [int(x) + tail + a for x, a in zip(b, (47, 8, 159))]
        # read back, and evicted again
        again = _lib.Batch("bf16", h_q, h_kv, d, 8, lens)
        total = sum(lens)
        k2, v2 = (torch.empty(total * h_kv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        _lib.paged_rows(pc, _dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)), k2, v2)
        for p, m in enumerate(lens):
            at = sum(lens[:p]) * h_kv * d
            for got, w in zip((k2, v2), _rows_of(pc, p, m)):
                np.testing.assert_array_equal(_host(got)[at:at + m * h_kv * d].reshape(h_kv, m, d), w)
        keep, win = 12, _q(rng, n * 8, h_q, d, "bf16").view(n, 8, h_q, d).transpose(1, 2).contiguous()
        lam = torch.zeros(n, device="cuda")
        rm, rs = (torch.empty(n, h_q, 8, device="cuda") for _ in range(2))
        si = torch.empty(n, h_kv, keep, dtype=torch.int32, device="cuda")
        ko, vo = (torch.empty(n, h_kv, keep + 8, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ws = torch.empty(_lib.candidates_workspace_bytes(again, keep, 4, 8), dtype=torch.uint8, device="cuda")
        _lib.evict_pass(again, win, k2, v2, d ** -0.5, lam, lam, keep, 4, 8, rm, rs, si, ws, None, ko, vo)
        small = _fill(_lib.PagedCache.allocate("bf16", "e2m1", h_q, h_kv, d, R, 8, n, 2))
        small.table.copy_(_dev(np.array([[3, 1], [0, 5], [7, 2]], np.int32)))
        _lib.paged_compact(again, k2, v2, si, keep, 8, small)
        stream.synchronize()
    # what was coded once is coded again without loss
    small.lens.fill_(keep + 8)
    for p in range(n):
        for got, w in zip(_rows_of(small, p, keep + 8), (ko, vo)):
            np.testing.assert_array_equal(got, _host(w[p]))


def test_captured_step():
    """A generation step (tables, rotated append, attention, reading back) captured once and replayed with other tokens and
    positions, other work between the replays: every replay equals the eager calls."""
    import torch
    rng = _rng(21)
    h_q, h_kv, d, R, n, stride = 8, 2, 64, 16, 5, 60
    lens = [3, 15, 16, 500, 901]
    a = _cache4(rng, "bf16", h_q, h_kv, d, R, lens, spare=40, max_len=960, stride=stride)
    cl = lambda t: t.view(torch.uint8).clone().view(t.dtype)  # noqa: E731
    b = _lib.PagedCache("bf16", h_q, cl(a.k), cl(a.v), cl(a.k_scale), cl(a.v_scale), a.table.clone(), a.lens.clone(), 960)
    used = set(a.table[a.table >= 0].tolist())
    free = _dev(np.asarray([i for i in range(a.struct.n_blocks) if i not in used], np.int32))
    qkv = torch.zeros(n, h_q + 2 * h_kv, d, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    rot = _lib.Rotary("interleaved", _dev(_lib.rotary_frequencies("plain", 32)[0]))
    off = _dev(np.array([0, 40, 80, 120, 640, 1600], np.int64))

    def buffers(pc):
        z = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")  # noqa: E731
        nb = _lib.paged_attention_workspace_bytes(pc)
        assert nb > 0
        e = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        return dict(taken=z(1), to=z(n + 1), bo=z(n + 1), slots=z(n), out=e(n, h_q, d), q=e(n, h_q, d),
                    k=e(1600 * h_kv * d), v=e(1600 * h_kv * d), ws=torch.empty(nb, dtype=torch.uint8, device="cuda"))

    def step(pc, x):
        _lib.paged_tables(pc, pc.lens, None, free, x["taken"], x["taken"], x["to"], x["bo"], x["slots"])
        _lib.paged_append_rotated(pc, rot, pos, qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:], x["slots"], q=qkv[:, :h_q], q_out=x["q"])
        _lib.paged_attention(pc, x["q"], 0.125, x["out"], ws=x["ws"])
        _lib.paged_rows(pc, off, x["k"], x["v"])

    xa, xb = buffers(a), buffers(b)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(a, xa)
    torch.cuda.synchronize()
    assert a.lens.tolist() == lens  # capture ran nothing
    for i in range(20):
        qkv.copy_(_dev(rng.standard_normal(qkv.shape).astype(np.float32) * 2.0 ** (i % 5), torch.bfloat16))
        pos.copy_(_dev(rng.integers(0, 1 << 20, n).astype(np.int32)))
        graph.replay()
        other = torch.randn(300, 300, device="cuda") @ torch.randn(300, 300, device="cuda")
        step(b, xb)
        torch.cuda.synchronize()
        del other
        for name in ("taken", "to", "bo", "slots", "q", "out", "k", "v"):
            assert torch.equal(xa[name], xb[name]), (i, name)
        assert torch.equal(a.lens, b.lens) and torch.equal(a.table, b.table)
        if i % 7 == 0:
            _check4(a, xa["q"], 0.125, None, xa["out"], f"replay {i}")
    assert a.lens.tolist() == [x + 20 for x in lens]


@pytest.mark.parametrize("n", [4, 60])
def test_captured_turns_share_a_workspace(n):
    """Two captured calls of several tokens each that share a workspace, replayed three times over other queries with eager
    work between, against eager calls."""
    import torch
    rng = _rng(22, n)
    h_q, h_kv, d = 8, 2, 128
    pcs = [_cache4(rng, "bf16", h_q, h_kv, d, 32, lens) for lens in ([1500, 300], [900, 1200])]
    n_q, T = [n, n - 1], 2 * n - 1
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
    _check4(pcs[1], q[1], 0.09, n_q, out[1], "captured")
