"""The 8-bit paged cache's operators, as cases to time and compare: block tables and slots from
request lengths, appending new rows, compacting an eviction's kept rows into blocks, and attention
over the blocks for single tokens, a few tokens and whole prompt turns.

A cache holds K and V as 8-bit codes (e4m3 or int8) in blocks of R rows of one kv head, pools
[n_blocks][h_kv][R][d], with one fp32 scale per block and head: value = code * scale.  Row r of
problem p is row r % R of block table[p][r // R].  A written scale is the least power of two s with
max|x| <= 448 s (e4m3) or 127 s (int8) over the block's rows; code = x / s rounded to nearest even.

The head layout is the one of the package's workloads (32 query heads on 8 kv heads of 128), with
smaller and larger groups and d = 64 beside it.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
RAGGED_LENS = tuple(int(x) for x in np.random.default_rng([4, 0]).integers(2048, 31745, 8))


# ------------------------------------------------------------------------------------------------
# Cases
# ------------------------------------------------------------------------------------------------

def listed():
    return [
        # the step of a serving loop: every request of a large batch of evicted caches gets one row
        dict(name="tables_step", kind="tables", n_prob=256, cached=160, add=1, block_rows=16, lens_seed=1),
        # admission of a batch of prompts of up to 32k tokens
        dict(name="tables_prompts", kind="tables", n_prob=64, cached=0, add=32768, block_rows=32, lens_seed=2),
        # one generated token of each of 64 requests, into the layer's blocks
        dict(_append(64, 130, 1, 16, 3), name="append_step"),
        # a layer's K and V of eight prompts of unequal odd lengths, as prefill leaves them
        dict(_append(8, 0, 31744, 64, 4), name="append_prompts"),
        # what the eviction of an 8k prompt keeps, all layers in one call
        dict(_compact(32, 8192, 64, 16), name="compact_kept"),
        # a generous budget that falls with depth, at 32k, in int8
        dict(_compact(32, 32768, 1024, 32, beta=4.0, qtype="int8"), name="compact_pyramid"),
        # one generated token over the kept rows of all layers
        dict(_attend(32, 100, 1, 16, 5), name="decode_kept"),
        # one generated token over full caches of 32k rows
        dict(_attend(32, 32768, 1, 64, 6), name="decode_full"),
        # a ragged batch, one request still empty, eight query heads to a kv head, small int8 blocks
        dict(_attend(24, 24001, 1, 16, 7, ragged=True, h_q=64, qtype="int8"), name="decode_ragged"),
        # fp32 queries and heads of 64
        dict(_attend(4, 4097, 1, 32, 8, dtype="f32", h_q=16, d=64), name="decode_f32"),
        # up to five drafted tokens of each request, verified in one call
        dict(_attend(16, 6001, 5, 32, 9, ragged=True), name="verify"),
        # a further turn of up to 4096 tokens over caches of up to 16k rows
        dict(_attend(3, 16384, 4096, 64, 10, ragged=True), name="prompt_turn"),
    ]


def _append(n_prob, cached, add, block_rows, lens_seed, dtype="bf16", qtype="e4m3", h_q=32, h_kv=8, d=128):
    """Up to `cached` rows per request before the call, up to `add` new ones."""
    return dict(kind="append", n_prob=n_prob, cached=cached, add=add, block_rows=block_rows,
                lens_seed=lens_seed, dtype=dtype, qtype=qtype, h_q=h_q, h_kv=h_kv, d=d)


def _compact(layers, L, budget, block_rows, tail=32, beta=1.0, dtype="bf16", qtype="e4m3", h_kv=8, d=128):
    """`budget` rows a layer on average, falling with depth for beta > 1, and the last `tail`."""
    return dict(kind="compact", layers=layers, L=L, budget=budget, tail=tail, beta=beta,
                block_rows=block_rows, dtype=dtype, qtype=qtype, h_q=4 * h_kv, h_kv=h_kv, d=d)


def _attend(n_prob, rows, tokens, block_rows, lens_seed, ragged=False, dtype="bf16", qtype="e4m3", h_q=32,
            h_kv=8, d=128):
    """The last (up to) `tokens` rows of caches of up to `rows` rows attend."""
    return dict(kind="attend", n_prob=n_prob, rows=rows, tokens=tokens, block_rows=block_rows, ragged=ragged,
                lens_seed=lens_seed, dtype=dtype, qtype=qtype, h_q=h_q, h_kv=h_kv, d=d)


def draw(rng):
    def log_int(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    while True:
        kind = rng.choice(["tables", "append", "compact", "decode", "decode", "verify", "turn"])
        ls = rng.randrange(1 << 20)
        R = rng.choice([16, 32, 64, 128])
        types = dict(dtype=rng.choice(["bf16", "bf16", "f32"]), qtype=rng.choice(["e4m3", "e4m3", "int8"]),
                     d=rng.choice([128, 128, 64]))
        if kind == "tables":
            c = dict(kind="tables", n_prob=log_int(1, 2048), cached=rng.choice([0, log_int(1, 4096)]),
                     add=rng.choice([1, log_int(2, 32768)]), block_rows=R, lens_seed=ls)
        elif kind == "append":
            c = _append(log_int(1, 256), rng.choice([0, log_int(1, 2000)]), rng.choice([1, log_int(2, 16384)]), R, ls,
                        **types)
        elif kind == "compact":
            L = log_int(600, 32768)
            c = _compact(log_int(1, 32), L, log_int(16, min(2048, L // 4)), R, tail=rng.choice([8, 16, 32]),
                         beta=rng.choice([1.0, 4.0]), **types)
        else:
            tokens = {"decode": 1, "verify": log_int(2, 16), "turn": log_int(17, 4096)}[kind]
            rows = log_int(max(1, tokens), 32768)
            n = log_int(1, 64) if kind != "turn" else log_int(1, 6)
            if kind == "turn":
                types["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"]) if tokens < 300 else "bf16"
            c = _attend(n, rows, tokens, R, ls, ragged=rng.random() < 0.6, h_q=8 * rng.choice([1, 2, 3, 4, 4, 8]),
                        **types)
        w = work(c)
        if c["kind"] != "attend":
            if w["bytes"] <= 7e8:
                return c
        elif w["bytes"] <= 2.1e9 and w["flops"] <= 1.4e12 and c["n_prob"] * c["h_q"] * c["tokens"] * c["rows"] <= 6.4e9:
            return c


def _cached_and_added(c):
    """Rows per request before the call, and new rows: unequal, some requests at the ends of the range."""
    rng = np.random.default_rng(c["lens_seed"])
    n = c["n_prob"]
    if c["kind"] == "append" and c["add"] == 31744:  # the workloads' own ragged batch
        return np.zeros(n, np.int64), np.resize(np.asarray(RAGGED_LENS), n)
    cached = rng.integers((c["cached"] + 1) // 2, c["cached"] + 1, n)
    add = np.ones(n, np.int64) if c["add"] == 1 else rng.integers(1, c["add"] + 1, n)
    add[0] = c["add"]
    if n > 3 and c["add"] > 1:
        add[2] = 0
    return cached, add


def _rows_and_tokens(c):
    """Cache lengths, and how many of their last rows attend."""
    rng = np.random.default_rng(c["lens_seed"])
    n, rows = c["n_prob"], c["rows"]
    if not c["ragged"]:
        lens = np.maximum(1, rows - (rows // 8) * (np.arange(n) % 4) // 3)
        tokens = np.minimum(np.full(n, c["tokens"]), lens)
    else:
        lens = rng.integers(max(1, rows // 8), rows + 1, n)
        lens[0] = rows
        tokens = np.minimum(rng.integers(1, c["tokens"] + 1, n), lens)
        tokens[0] = min(c["tokens"], rows)
        if n > 3:
            lens[2] = 0
            tokens[2] = 1 if c["tokens"] == 1 else 0
    return lens, tokens


def _budgets(c):
    """Rows kept per layer: linear in depth about the mean."""
    n, b = c["layers"], c["budget"]
    lo = max(1, int(b / c["beta"]))
    t = np.linspace(1.0, -1.0, n) if n > 1 else np.zeros(1)
    return np.minimum(np.rint(b + t * (b - lo)).astype(np.int64), c["L"] - c["tail"])


def _blocks(rows, R):
    return -(-np.asarray(rows) // R)


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _qdtype(c):
    return torch.float8_e4m3fn if c["qtype"] == "e4m3" else torch.int8


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEVICE).to(dtype)


def _table(gen, per_prob, spare):
    """A table with every problem's blocks from one random order of the pool's, -1 behind them."""
    total = int(per_prob.sum())
    ids = torch.randperm(total + spare, device=DEVICE, generator=gen).to(torch.int32)
    stride = max(1, int(per_prob.max()))
    used = torch.arange(stride, device=DEVICE)[None] < _dev(per_prob)[:, None]
    table = torch.full((len(per_prob), stride), -1, dtype=torch.int32, device=DEVICE)
    table[used] = ids[:total]
    return table, ids[total:].contiguous(), total + spare


def prepare(case, seed):
    c, gen = case, _gen(seed)
    s = dict(case=c)
    if c["kind"] == "tables":
        cached, add = _cached_and_added(c)
        R = c["block_rows"]
        have, need = _blocks(cached, R), _blocks(cached + add, R)
        table, free, n_blocks = _table(gen, have, int((need - have).sum()) + 64)
        full = torch.full((c["n_prob"], int(need.max()) + 1), -1, dtype=torch.int32, device=DEVICE)
        full[:, :table.shape[1]] = table
        n_slots = -(-int(add.sum()) // 64) * 64  # batches of tokens are padded
        s.update(table=full, free=free, n_blocks=n_blocks, len_in=_dev(cached), add=_dev(add),
                 taken_in=torch.full((1,), 5, dtype=torch.int32, device=DEVICE))
        e = lambda n: torch.zeros(n, dtype=torch.int32, device=DEVICE)  # noqa: E731
        s.update(len=e(c["n_prob"]), taken=e(1), tok_off=e(c["n_prob"] + 1), blk_off=e(c["n_prob"] + 1),
                 slots=e(n_slots))
        if own:
            s["pc"] = _handle(c, s, 1)
        return s
    R, h_kv, d, dt = c["block_rows"], c["h_kv"], c["d"], _dtype(c)
    rnd = lambda *n: torch.randn(*n, device=DEVICE, generator=gen)  # noqa: E731
    if c["kind"] == "append":
        cached, add = _cached_and_added(c)
        have, need = _blocks(cached, R), _blocks(cached + add, R)
        s["table"], _, n = _table(gen, np.maximum(need, 1), 3)
        s["len"] = _dev(cached + add)
        _fill(s, c, gen, n, cached)
        # new rows as a projection leaves them: q, k and v of a token in one row; some tokens larger
        T = int(add.sum())
        qkv = rnd(T, c["h_q"] + 2 * h_kv, d)
        qkv *= torch.where(torch.rand(T, 1, 1, device=DEVICE, generator=gen) < 0.05, 6.0, 1.0)
        qkv = qkv.to(dt)
        s["k_new"], s["v_new"] = qkv[:, c["h_q"]:c["h_q"] + h_kv], qkv[:, c["h_q"] + h_kv:]
        row = torch.arange(T, device=DEVICE) - _dev(np.repeat(np.cumsum(add) - add - cached, add), torch.int64)
        p = _dev(np.repeat(np.arange(c["n_prob"]), add), torch.int64)
        s["slots"] = (s["table"][p, row // R] * R + row % R).to(torch.int32)
        if own:
            s["pc"] = _handle(c, s, int((cached + add).max()))
        return s
    if c["kind"] == "compact":
        P, L, tail = c["layers"], c["L"], c["tail"]
        b = _budgets(c)
        B = int(b.max())
        k, v = torch.empty(P, h_kv, L, d, dtype=dt, device=DEVICE), torch.empty(P, h_kv, L, d, dtype=dt, device=DEVICE)
        for p in range(P):
            k[p], v[p] = rnd(h_kv, L, d), rnd(h_kv, L, d)
        sel = torch.rand(P, h_kv, L - tail, device=DEVICE, generator=gen).topk(B).indices.to(torch.int32)
        sel[torch.arange(B, device=DEVICE).expand(P, h_kv, B) >= _dev(b)[:, None, None]] = -1
        rows = b + tail
        s["table"], _, n = _table(gen, _blocks(rows, R), 3)
        z = lambda: torch.zeros(n, h_kv, R, d, dtype=torch.uint8, device=DEVICE).view(_qdtype(c))  # noqa: E731
        s.update(k=k, v=v, sel=sel, budget=B, b_host=b, b_dev=_dev(b), kq=z(), vq=z(), len=_dev(rows),
                 ks=torch.zeros(n, h_kv, device=DEVICE), vs=torch.zeros(n, h_kv, device=DEVICE))
        if own:
            from paper_2609_30738_amd import _lib
            s["pc"] = _handle(c, s, int(rows.max()))
            s["batch"] = _lib.Batch(c["dtype"], c["h_q"], h_kv, d, 8, [L] * P, device=DEVICE)
            s["budgets"] = _lib.Budgets(b, DEVICE)
        return s
    lens, tokens = _rows_and_tokens(c)
    s["table"], _, n = _table(gen, np.maximum(_blocks(lens, R), 1), 3)
    s["len"] = _dev(lens)
    _fill(s, c, gen, n, lens)
    off = np.concatenate([[0], np.cumsum(tokens)])
    pad = 3 if c["tokens"] > 1 else 0  # rows behind the last token of a padded batch
    T = int(off[-1]) + pad
    # queries as a projection leaves them, q, k and v of a token in one row
    s["q"] = rnd(T, c["h_q"] + 2 * h_kv, d).to(dt)[:, :c["h_q"]]
    s["tok_off"] = _dev(off)
    s["max_q"], s["max_len"] = int(tokens.max()), int(lens.max())
    s["scale"] = 1.0 / math.sqrt(d)
    s["out"] = torch.zeros(T, c["h_q"], d, dtype=dt, device=DEVICE)
    if own:
        from paper_2609_30738_amd import _lib
        s["pc"] = _handle(c, s, s["max_len"])
        nb = _lib.paged_attention_workspace_bytes(s["pc"], T, s["max_q"])
        s["ws"] = torch.empty(nb, dtype=torch.uint8, device=DEVICE) if nb else None
    return s


def _fill(s, c, gen, n, lens):
    """Pools whose used rows hold quantised normal values (a few dominant keys among them); the rows
    behind each problem's last one hold what memory happened to hold: not-a-number codes."""
    R, h_kv, d = c["block_rows"], c["h_kv"], c["d"]
    for name in ("k", "v"):
        q = torch.empty(n, h_kv, R, d, dtype=torch.uint8, device=DEVICE)
        sc = torch.empty(n, h_kv, device=DEVICE)
        for i in range(0, n, 4096):
            x = torch.randn(min(4096, n - i), h_kv, R, d, device=DEVICE, generator=gen)
            if name == "k":
                x *= torch.where(torch.rand(*x.shape[:3], 1, device=DEVICE, generator=gen) < 3e-4, 4.0, 1.0)
            sc[i:i + 4096] = _scale_of(x.abs().amax((2, 3)), c)
            q[i:i + 4096] = _codes(x, sc[i:i + 4096][..., None, None], c).view(torch.uint8)
        lens_d = _dev(lens, torch.int64)
        at = s["table"].long().gather(1, (lens_d[:, None] // R).clamp(max=s["table"].shape[1] - 1))[:, 0]
        part = lens_d < R * (s["table"] >= 0).sum(1)
        behind = torch.arange(R, device=DEVICE)[None] >= (lens_d % R)[:, None]
        keep = q[at[part]]
        q[at[part]] = torch.where(behind[part][:, None, :, None], torch.full_like(keep, 0x7F), keep)
        s[name + "q"], s[name + "s"] = q.view(_qdtype(c)), sc


def _handle(c, s, max_len):
    from paper_2609_30738_amd import _lib
    if c["kind"] == "tables":
        return _lib.PagedCache.for_tables(c["block_rows"], s["n_blocks"], s["table"], s["len"])
    return _lib.PagedCache(c["dtype"], c["h_q"], s["kq"], s["vq"], s["ks"], s["vs"], s["table"], s["len"], max_len)


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2609_30738_amd import _lib
    c = s["case"]
    if c["kind"] == "tables":
        _lib.paged_tables(s["pc"], s["len_in"], s["add"], s["free"], s["taken_in"], s["taken"], s["tok_off"],
                          s["blk_off"], s["slots"])
    elif c["kind"] == "append":
        _lib.paged_append(s["pc"], s["k_new"], s["v_new"], s["slots"])
    elif c["kind"] == "compact":
        _lib.paged_compact(s["batch"], s["k"], s["v"], s["sel"], s["budget"], c["tail"], s["pc"], s["budgets"])
    else:
        off = s["tok_off"] if c["tokens"] > 1 else None
        _lib.paged_attention(s["pc"], s["q"], s["scale"], s["out"], tok_off=off, max_q=s["max_q"], ws=s["ws"])
    return _outputs(s)


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "tables":
        return {n: s[n] for n in ("table", "len", "taken", "tok_off", "blk_off", "slots")}
    if kind == "attend":
        return dict(out=s["out"])
    return dict(k=s["kq"], v=s["vq"], k_scale=s["ks"], v_scale=s["vs"])


def _run_plain(s):
    dict(tables=_plain_tables, append=_plain_append, compact=_plain_compact, attend=_plain_attend)[s["case"]["kind"]](s)
    return _outputs(s)


def _plain_tables(s):
    R, table = s["case"]["block_rows"], s["table"]
    old, add = s["len_in"].long(), s["add"].long()
    have, need = (old + R - 1) // R, (old + add + R - 1) // R
    zero = torch.zeros(1, dtype=torch.int64, device=DEVICE)
    tok_off = torch.cat([zero, add.cumsum(0)])
    blk_off = torch.cat([zero, (need - have).cumsum(0)]) + s["taken_in"]
    j = torch.arange(table.shape[1], device=DEVICE)[None]
    new = (j >= have[:, None]) & (j < need[:, None])
    at = (blk_off[:-1, None] + j - have[:, None]).clamp(0, s["free"].numel() - 1)
    table.copy_(torch.where(new, s["free"][at], table))
    i = torch.arange(s["slots"].numel(), device=DEVICE)
    p = torch.searchsorted(tok_off, i, right=True).sub_(1).clamp_(max=old.numel() - 1)
    row = old[p] + i - tok_off[p]
    b = table[p, (row // R).clamp(max=table.shape[1] - 1)]
    s["slots"].copy_(torch.where(i < tok_off[-1], b * R + row % R, -1))
    s["tok_off"].copy_(tok_off)
    s["blk_off"].copy_(blk_off)
    s["taken"].copy_(blk_off[-1:])
    s["len"].copy_(old + add)


def _scale_of(amax, c):
    """The least power of two s with amax <= qmax s; 0 for 0."""
    m, e = torch.frexp(amax)
    bits, top = (9, 0.875) if c["qtype"] == "e4m3" else (7, 127 / 128)
    e = (e - bits + (m > top)).clamp(min=-126).to(torch.int32)
    return torch.where(amax > 0, ((e + 127) << 23).view(torch.float32), torch.zeros_like(amax))


def _codes(x, scale, c):
    """x / scale (a power of two) rounded to nearest even, as codes."""
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    y = x * inv
    return y.to(torch.float8_e4m3fn) if c["qtype"] == "e4m3" else y.round().to(torch.int8)


def _values(codes):
    """8-bit codes as fp32."""
    return codes.to(torch.float32)


def _take(pool, ids):
    """Blocks of a pool by their numbers."""
    return pool.view(torch.uint8)[ids].view(pool.dtype)


def _plain_append(s):
    c = s["case"]
    R = c["block_rows"]
    slots = s["slots"].long()
    block, row = slots // R, slots % R
    first = torch.ones_like(slots, dtype=torch.bool)
    first[1:] = (slots[1:] != slots[:-1] + 1) | (row[1:] == 0)
    for new, pool, scale in ((s["k_new"], s["kq"], s["ks"]), (s["v_new"], s["vq"], s["vs"])):
        x = new.float()
        amax = torch.zeros_like(scale).index_reduce_(0, block, x.abs().amax(2), "amax")
        # blocks that get rows, with the number of rows they held before
        b, held = block[first], row[first]
        old = torch.where(held[:, None] > 0, scale[b], torch.zeros_like(scale[b]))
        to = torch.maximum(old, _scale_of(amax[b], c))
        # the old rows of blocks in use move to the new scale
        u = held > 0
        keep = torch.arange(R, device=DEVICE)[None, None, :, None] < held[u][:, None, None, None]
        codes = _take(pool, b[u])
        moved = _codes(_values(codes) * old[u][..., None, None], to[u][..., None, None], c)
        bytes_ = pool.view(torch.uint8)
        bytes_[b[u]] = torch.where(keep, moved.view(torch.uint8), codes.view(torch.uint8))
        scale[b] = to
        bytes_[block, :, row] = _codes(x, scale[block][..., None], c).view(torch.uint8)


def _plain_compact(s):
    c = s["case"]
    P, h_kv, L, d = s["k"].shape
    R, tail, nb = c["block_rows"], c["tail"], s["table"].shape[1]
    b = s["b_dev"].long()[:, None, None]
    t = torch.arange(s["budget"], device=DEVICE)
    pos = torch.where(t < b, s["sel"].long(), L).sort(-1).values
    r = torch.arange(nb * R, device=DEVICE).expand(P, h_kv, nb * R)
    pos = torch.where(r < b, pos.gather(2, r.clamp(max=s["budget"] - 1)), L - tail + r - b)
    used = (r < b + tail)[..., None]
    pos = pos.clamp(0, L - 1)[..., None].expand(-1, -1, -1, d)
    ids = s["table"].long()
    live = ids >= 0
    for src, pool, scale in ((s["k"], s["kq"], s["ks"]), (s["v"], s["vq"], s["vs"])):
        x = torch.where(used, src.gather(2, pos).float(), torch.zeros((), device=DEVICE))
        x = x.view(P, h_kv, nb, R, d).transpose(1, 2)[live]
        scale[ids[live]] = _scale_of(x.abs().amax((2, 3)), c)
        codes = _codes(x, scale[ids[live]][..., None, None], c).view(torch.uint8)
        u = used.view(P, h_kv, nb, R, 1).transpose(1, 2)[live]
        pool.view(torch.uint8)[ids[live]] = torch.where(u, codes, _take(pool, ids[live]).view(torch.uint8))


def _plain_attend(s):
    c = s["case"]
    P, h_q, h_kv, d, R = c["n_prob"], c["h_q"], c["h_kv"], c["d"], c["block_rows"]
    G, n_max, L = h_q // h_kv, s["max_q"], s["table"].shape[1] * R
    ids = s["table"].long().clamp(min=0)
    lens, off = s["len"].long(), s["tok_off"].long()
    row = torch.arange(L, device=DEVICE)
    used = (row < lens[:, None])[:, None, :, None]

    def rows(pool, scale):
        x = _values(_take(pool, ids)).mul_(scale[ids][..., None, None])  # [P, blocks, h_kv, R, d]
        return torch.where(used, x.transpose(1, 2).reshape(P, h_kv, L, d), torch.zeros((), device=DEVICE))

    k = rows(s["kq"], s["ks"])
    j = torch.arange(n_max, device=DEVICE)
    n = off[1:] - off[:-1]
    live = j < n[:, None]                                                   # [P, n_max]
    tok = (off[:-1, None] + j).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][tok].float().view(P, n_max, h_kv, G, d).permute(0, 2, 1, 3, 4).reshape(P, h_kv, n_max * G, d)
    t = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    del k
    last = (lens - n)[:, None] + j                                          # last visible row of a token
    unseen = (row > last[..., None]).repeat_interleave(G, 1)[:, None]      # [P, 1, n_max G, L]
    t = t.masked_fill_(unseen, -math.inf)
    m = t.amax(-1, keepdim=True)
    t = t.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    z = t.sum(-1, keepdim=True)
    o = torch.matmul(t, rows(s["vq"], s["vs"])).div_(torch.where(z > 0, z, torch.ones_like(z)))
    o = o.view(P, h_kv, n_max, G, d).permute(0, 2, 1, 3, 4).reshape(P, n_max, h_q, d)
    s["out"][tok[live]] = o[live].to(s["out"].dtype)


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    R = c["block_rows"]
    if c["kind"] == "tables":
        cached, add = _cached_and_added(c)
        blocks = int((_blocks(cached + add, R) - _blocks(cached, R)).sum())
        held = int(((cached % R > 0) & (add > 0)).sum())  # blocks in use that get further rows
        return {"bytes": 8 * c["n_prob"] + 4 * held + 8 * blocks + 4 * int(add.sum()) + 12 * c["n_prob"], "flops": 0}
    e, h_kv, d = 2 if c["dtype"] == "bf16" else 4, c["h_kv"], c["d"]
    if c["kind"] == "append":
        cached, add = _cached_and_added(c)
        T = int(add.sum())
        blocks = int((_blocks(cached + add, R) - cached // R)[add > 0].sum())
        return {"bytes": 2 * T * h_kv * d * (e + 1) + 4 * T + 8 * blocks * h_kv, "flops": 2 * T * h_kv * d}
    if c["kind"] == "compact":
        rows = _budgets(c) + c["tail"]
        n = int(rows.sum()) * h_kv
        return {"bytes": 2 * n * d * (e + 1) + 4 * int(_budgets(c).sum()) * h_kv
                + 8 * int(_blocks(rows, R).sum()) * h_kv, "flops": 2 * n * d}
    lens, tokens = _rows_and_tokens(c)
    seen = sum(int(n) * int(L - n) + int(n) * (int(n) + 1) // 2 for L, n in zip(lens, tokens) if L >= n)
    T = int(tokens.sum())
    read = int(lens[tokens > 0].sum())
    return {"bytes": 2 * read * h_kv * d + 8 * int(_blocks(lens, R).sum()) * h_kv + 2 * T * c["h_q"] * d * e,
            "flops": 4 * seen * c["h_q"] * d}


# ------------------------------------------------------------------------------------------------
# The same from the definition, in 64 bits
# ------------------------------------------------------------------------------------------------

def _decode64(codes):
    """Codes as the numbers they stand for, from their bits."""
    if codes.dtype == torch.int8:
        return codes.double()
    u = codes.view(torch.uint8).int()
    e, f = (u >> 3) & 15, (u & 7).double()
    x = torch.where(e > 0, (1.0 + f / 8) * torch.exp2((e - 7).double()), f * 2.0 ** -9)
    x = torch.where((u & 0x7F) == 0x7F, torch.full_like(x, math.nan), x)
    return torch.where(u >= 128, -x, x)


def _grid64(x, c):
    """x rounded to the nearest number of 8 bits, ties to the even one, and held as such a number."""
    if c["qtype"] == "int8":
        return x.round()
    step = torch.exp2(x.abs().clamp(min=2.0 ** -6).log2().floor() - 3)
    # log2 may fall on the wrong side of a power of two: the step follows the number itself
    step = torch.where(x.abs().clamp(min=2.0 ** -6) >= 16 * step, 2 * step, step)
    step = torch.where(x.abs().clamp(min=2.0 ** -6) < 8 * step, step / 2, step)
    return (x / step).round() * step


def _least_scale64(amax, c):
    qmax = 448.0 if c["qtype"] == "e4m3" else 127.0
    e = torch.ceil(torch.log2((amax / qmax).clamp(min=2.0 ** -126)))
    e = torch.where(amax <= qmax * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax > qmax * torch.exp2(e), e + 1, e)
    return torch.where(amax > 0, torch.exp2(e.clamp(min=-126)), torch.zeros_like(amax))


def exact(case, seed):
    c = case
    if c["kind"] == "tables":
        return None  # whole numbers alone
    s = prepare(c, seed)
    R = c["block_rows"]
    if c["kind"] == "attend":
        return dict(out=_attend64(s, c))
    if c["kind"] == "append":
        cached, add = _cached_and_added(c)
        at, out = 0, {}
        k, v = s["k_new"].double(), s["v_new"].double()
        pools = [_decode64(s["kq"]), _decode64(s["vq"])]
        scales = [s["ks"].double(), s["vs"].double()]
        n_blk = int(_blocks(cached + add, R).sum()) + c["n_prob"]
        if n_blk > 4000:
            return None
        for p in range(c["n_prob"]):
            r, end = int(cached[p]), int(cached[p] + add[p])
            while r < end:
                b, lo = int(s["table"][p, r // R]), r % R
                n = min(R - lo, end - r)
                for x, pool, sc in ((k, pools[0], scales[0]), (v, pools[1], scales[1])):
                    new = x[at:at + n].transpose(0, 1)
                    was = sc[b] if lo else torch.zeros_like(sc[b])
                    to = torch.maximum(was, _least_scale64(new.abs().amax((1, 2)), c))
                    div = torch.where(to > 0, to, torch.ones_like(to))[:, None, None]
                    if lo:
                        pool[b, :, :lo] = _grid64(pool[b, :, :lo] * was[:, None, None] / div, c)
                    pool[b, :, lo:lo + n] = _grid64(new / div, c)
                    sc[b] = to
                at += n
                r += n
        out = dict(k_scale=scales[0], v_scale=scales[1])
        return dict(out, k=pools[0] if c["qtype"] == "e4m3" else None, v=pools[1] if c["qtype"] == "e4m3" else None)
    b = s["b_host"]
    pools = [_decode64(s["kq"]), _decode64(s["vq"])]
    scales = [s["ks"].double(), s["vs"].double()]
    for p in range(c["layers"]):
        n = int(b[p])
        kept = s["sel"][p, :, :n].long().sort(1).values
        rows = torch.cat([kept, torch.arange(c["L"] - c["tail"], c["L"], device=DEVICE).expand(c["h_kv"], -1)], 1)
        for x, pool, sc in ((s["k"][p], pools[0], scales[0]), (s["v"][p], pools[1], scales[1])):
            x = x.gather(1, rows[..., None].expand(-1, -1, c["d"])).double()
            for j, i in enumerate(range(0, x.shape[1], R)):
                at = int(s["table"][p, j])
                part = x[:, i:i + R]
                sc[at] = _least_scale64(part.abs().amax((1, 2)), c)
                pool[at, :, :part.shape[1]] = _grid64(part / sc[at][:, None, None], c)
    e4m3 = c["qtype"] == "e4m3"
    return dict(k=pools[0] if e4m3 else None, v=pools[1] if e4m3 else None, k_scale=scales[0], v_scale=scales[1])


def _attend64(s, c):
    lens, tokens = _rows_and_tokens(c)
    R, h_kv, d, G = c["block_rows"], c["h_kv"], c["d"], c["h_q"] // c["h_kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    at = 0
    for p in range(c["n_prob"]):
        L, n = int(lens[p]), int(tokens[p])
        if L and n:
            ids = s["table"][p, :-(-L // R)].long()
            seen = torch.arange(L, device=DEVICE)[None] <= (L - n + torch.arange(n, device=DEVICE))[:, None]
            for g in range(h_kv):
                k, v = (( _decode64(_take(s[x + "q"], ids)[:, g]) * s[x + "s"][ids, g].double()[:, None, None])
                        .reshape(-1, d)[:L] for x in "kv")
                q = s["q"][at:at + n, g * G:(g + 1) * G].double()
                for h in range(G):
                    t = (q[:, h] @ k.T * s["scale"]).masked_fill_(~seen, -math.inf)
                    out[at:at + n, g * G + h] = t.softmax(-1) @ v
        at += n
    return out
