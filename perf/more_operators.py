"""Cases to time and compare: the paged cache in 4 bits (appending, compaction, reading back, attention), rotary
positions, and appending to a paged cache with the rotation on the way.

Rotation of a row x at position p, frequencies f_i in radians a position, i < r / 2, factor s: with
c = s cos(p f_i), t = s sin(p f_i) the pair (a, b), elements (i, i + r / 2) in the half layout and (2 i, 2 i + 1) in the
interleaved one, becomes (a c - b t, b c + a t); elements from r on stay.

A 4-bit cache (e2m1) holds codes of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} in blocks of R rows, pools [n_blocks][h_kv][R][d / 2] bytes
with element 2 i in a byte's low half, and a scale 2^(b - 127) for 32 elements of a row, bytes b in
[n_blocks][h_kv][d / 32][R]: the least one with max|x| <= 6 2^(b - 127), 2 <= b <= 252.  An 8-bit one holds e4m3 or int8 codes
with one fp32 power of two for a block and head: the least s with max|x| <= 448 s or 127 s.  Codes are rounded to nearest even.
torch does not convert 4-bit tensors, so a pass that writes them ends with reading the caches back.

The head layout is the one of the package's workloads (32 query heads on 8 kv heads of 128), with smaller and larger groups
and d = 64 beside it.  A row's place in a cache that was evicted is not its position: positions are inputs.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
GROUP = 32  # elements of a row that share a 4-bit cache's scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------
# Cases
# ------------------------------------------------------------------------------------------------

def listed():
    return [
        # the queries of one generated token of 64 requests
        dict(_rotate(64, 32, 1), name="rotate_step"),
        # a layer's queries of a long prompt, half of each head rotated in neighbouring pairs, scaled for long contexts
        dict(_rotate(31744, 32, 2, layout="interleaved", rot=64, family="yarn"), name="rotate_prompt"),
        # one generated token of each of 64 requests into the layer's 8-bit blocks, keys and queries rotated
        dict(_append(64, 130, 1, 16, 3, q=True), name="append_step"),
        # a layer's q, k and v of eight prompts of unequal odd lengths, as the projection leaves them
        dict(_append(8, 0, 8191, 64, 4, q=True), name="append_prompts"),
        # the same two into 4-bit blocks, which are read back
        dict(_append(24, 130, 1, 16, 5, q=True, qtype="e2m1", layout="interleaved"), name="append4_step"),
        dict(_append(4, 0, 8191, 32, 6, qtype="e2m1", family="bands"), name="append4_prompts"),
        # what the eviction of an 8k prompt keeps, all layers in one call, into 4 bits and read back
        dict(_compact(32, 8192, 64, 16), name="compact4_kept"),
        # one generated token over the kept rows of all layers
        dict(_attend(32, 100, 1, 16, 7), name="decode4_kept"),
        # one generated token over full caches of 32k rows
        dict(_attend(32, 32768, 1, 64, 8), name="decode4_full"),
        # a ragged batch, one request still empty, eight query heads to a kv head, small blocks
        dict(_attend(24, 24001, 1, 16, 9, ragged=True, h_q=64), name="decode4_ragged"),
        # up to five drafted tokens of each request, verified in one call
        dict(_attend(16, 6001, 5, 32, 10, ragged=True), name="verify4"),
        # a further turn of up to 4096 tokens over caches of up to 16k rows
        dict(_attend(3, 16384, 4096, 64, 11, ragged=True), name="prompt_turn4"),
    ]


def _rotate(tokens, heads, lens_seed, layout="half", rot=128, family="plain", inverse=False, dtype="bf16", d=128):
    return dict(kind="rotate", tokens=tokens, h_q=heads, lens_seed=lens_seed, layout=layout, rot=rot, family=family,
                inverse=inverse, dtype=dtype, d=d)


def _append(n_prob, cached, add, block_rows, lens_seed, q=False, layout="half", rot=128, family="plain", dtype="bf16",
            qtype="e4m3", h_q=32, h_kv=8, d=128):
    """Up to `cached` rows per request before the call, up to `add` new ones; rot 0: not rotated."""
    return dict(kind="append", n_prob=n_prob, cached=cached, add=add, block_rows=block_rows, lens_seed=lens_seed, q=q,
                layout=layout, rot=rot, family=family, dtype=dtype, qtype=qtype, h_q=h_q, h_kv=h_kv, d=d)


def _compact(layers, L, budget, block_rows, tail=32, dtype="bf16", h_kv=8, d=128):
    """`budget` rows a layer and the last `tail`, into 4 bits, and read back."""
    return dict(kind="compact", layers=layers, L=L, budget=budget, tail=tail, block_rows=block_rows, dtype=dtype,
                qtype="e2m1", h_q=4 * h_kv, h_kv=h_kv, d=d)


def _rows(n_prob, rows, block_rows, lens_seed, qtype, dtype, h_kv, d):
    """Caches read back."""
    return dict(kind="rows", n_prob=n_prob, rows=rows, block_rows=block_rows, lens_seed=lens_seed, qtype=qtype, dtype=dtype,
                h_q=4 * h_kv, h_kv=h_kv, d=d)


def _attend(n_prob, rows, tokens, block_rows, lens_seed, ragged=False, dtype="bf16", h_q=32, h_kv=8, d=128):
    """The last (up to) `tokens` rows of 4-bit caches of up to `rows` rows attend."""
    return dict(kind="attend", n_prob=n_prob, rows=rows, tokens=tokens, block_rows=block_rows, ragged=ragged,
                lens_seed=lens_seed, dtype=dtype, qtype="e2m1", h_q=h_q, h_kv=h_kv, d=d)


def draw(rng):
    def log_int(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    while True:
        kind = rng.choice(["rotate", "append", "append", "compact", "rows", "decode", "decode", "verify", "turn"])
        ls = rng.randrange(1 << 20)
        R = rng.choice([16, 32, 64, 128])
        types = dict(dtype=rng.choice(["bf16", "bf16", "f32"]), d=rng.choice([128, 128, 64]))
        turn = dict(layout=rng.choice(["half", "interleaved"]), rot=16 * rng.choice([types["d"] // 16, rng.randint(1, types["d"] // 16)]),
                    family=rng.choice(["plain", "linear", "ntk", "yarn", "bands"]))
        if kind == "rotate":
            c = _rotate(log_int(1, 32768), rng.choice([1, 7, 8, 32, 40]), ls, inverse=rng.random() < 0.3, **turn, **types)
        elif kind == "append":
            qtype = rng.choice(["e2m1", "e4m3", "int8"])
            if qtype == "e2m1" and rng.random() < 0.3:
                turn["rot"] = 0
            c = _append(log_int(1, 256), rng.choice([0, log_int(1, 2000)]), rng.choice([1, log_int(2, 8192)]), R, ls,
                        q=turn["rot"] > 0 and rng.random() < 0.7, qtype=qtype, **turn, **types)
        elif kind == "compact":
            L = log_int(600, 32768)
            c = _compact(log_int(1, 32), L, log_int(16, min(2048, L // 4)), R, tail=rng.choice([8, 16, 32]), **types)
        elif kind == "rows":
            c = _rows(log_int(1, 64), log_int(1, 16384), R, ls, rng.choice(["e2m1", "e4m3", "int8"]), h_kv=8, **types)
        else:
            tokens = {"decode": 1, "verify": log_int(2, 16), "turn": log_int(17, 4096)}[kind]
            rows = log_int(max(1, tokens), 32768)
            n = log_int(1, 64) if kind != "turn" else log_int(1, 6)
            if kind == "turn":
                types["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"]) if tokens < 300 else "bf16"
            c = _attend(n, rows, tokens, R, ls, ragged=rng.random() < 0.6, h_q=8 * rng.choice([1, 2, 3, 4, 4, 8]), **types)
        w = work(c)
        if c["kind"] != "attend":
            if w["bytes"] <= 7e8:
                return c
        elif w["bytes"] <= 1.2e9 and w["flops"] <= 1.4e12 and c["n_prob"] * c["h_q"] * c["tokens"] * c["rows"] <= 6.4e9:
            return c


def _cached_and_added(c):
    """Rows per request before the call, and new rows: unequal, some requests at the ends of the range."""
    rng = np.random.default_rng(c["lens_seed"])
    n = c["n_prob"]
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
    if c["kind"] == "rows":
        lens = rng.integers((rows + 1) // 2, rows + 1, n)
        lens[0] = rows
        return lens, np.zeros(n, np.int64)
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


def _blocks(rows, R):
    return -(-np.asarray(rows) // R)


def _frequencies(c):
    """Radians a position of the r / 2 pairs, and the factor of the rotated elements: contexts of 8192 positions taken to
    four times as many."""
    r, base, F, old = c["rot"], 10000.0, 4.0, 8192.0
    i = np.arange(r // 2, dtype=np.float64)
    if c["family"] == "ntk":
        base = base * F ** (r / max(r - 2.0, 1.0))
    f = base ** (-2.0 * i / r)
    s = 1.0
    if c["family"] == "linear":
        f = f / F
    elif c["family"] == "yarn":
        at = lambda turns: r * math.log(old / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        f = f / F * (1.0 - keep) + f * keep
        s = 0.1 * math.log(F) + 1.0
    elif c["family"] == "bands":
        turns = old * f / (2 * math.pi)
        t = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1.0 - t) * f / F + t * f
    return f, float(np.float32(s))


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 7919 + 31)
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
    return table, total + spare


def _turning(c, s):
    f, factor = _frequencies(c)
    s["freq"], s["factor"] = torch.from_numpy(f).to(DEVICE), factor
    if own:
        from paper_2609_30738_amd import _lib
        s["rot"] = _lib.Rotary(c["layout"], s["freq"], factor, inverse=c.get("inverse", False))


def prepare(case, seed):
    c, gen = case, _gen(seed)
    s = dict(case=c)
    d, dt = c["d"], _dtype(c)
    rnd = lambda *n: torch.randn(*n, device=DEVICE, generator=gen)  # noqa: E731
    if c["kind"] == "rotate":
        T, H = c["tokens"], c["h_q"]
        _turning(c, s)
        # q, k and v of a token in one row, the queries first; positions of unequal requests
        s["x"] = rnd(T, H + 2, d).to(dt)[:, :H]
        s["pos"] = torch.randint(0, 32768, (T,), device=DEVICE, generator=gen, dtype=torch.int32)
        s["out"] = torch.zeros(T, H, d, dtype=dt, device=DEVICE)
        return s
    R, h_kv = c["block_rows"], c["h_kv"]
    if c["kind"] == "append":
        cached, add = _cached_and_added(c)
        s["table"], n = _table(gen, np.maximum(_blocks(cached + add, R), 1), 3)
        s["len"] = _dev(cached + add)
        _fill(s, c, gen, n, cached)
        # q, k and v of a token in one row, as a projection leaves them; some tokens larger
        T = int(add.sum())
        h = c["h_q"] if c["q"] else 1
        qkv = rnd(T, h + 2 * h_kv, d)
        qkv *= torch.where(torch.rand(T, 1, 1, device=DEVICE, generator=gen) < 0.05, 6.0, 1.0)
        qkv = qkv.to(dt)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :h], qkv[:, h:h + h_kv], qkv[:, h + h_kv:]
        s["q_out"] = torch.zeros(T, h, d, dtype=dt, device=DEVICE) if c["q"] else None
        row = torch.arange(T, device=DEVICE) - _dev(np.repeat(np.cumsum(add) - add - cached, add), torch.int64)
        p = _dev(np.repeat(np.arange(c["n_prob"]), add), torch.int64)
        s["slots"] = (s["table"][p, row // R] * R + row % R).to(torch.int32)
        # a cache that was evicted holds fewer rows than it has seen positions
        s["pos"] = (row + torch.where(_dev(cached, torch.int64) > 0, 8000, 0)[p]).to(torch.int32)
        if c["rot"]:
            _turning(c, s)
        _back(s, c, cached + add)
        return s
    if c["kind"] == "compact":
        P, L, tail, B = c["layers"], c["L"], c["tail"], min(c["budget"], c["L"] - c["tail"])
        k, v = torch.empty(P, h_kv, L, d, dtype=dt, device=DEVICE), torch.empty(P, h_kv, L, d, dtype=dt, device=DEVICE)
        for p in range(P):
            k[p], v[p] = rnd(h_kv, L, d), rnd(h_kv, L, d)
        sel = torch.rand(P, h_kv, L - tail, device=DEVICE, generator=gen).topk(B).indices.to(torch.int32)
        rows = np.full(P, B + tail)
        s["table"], n = _table(gen, _blocks(rows, R), 3)
        s.update(k=k, v=v, sel=sel, budget=B, len=_dev(rows))
        for name in ("k", "v"):
            s[name + "q"] = torch.zeros(n, h_kv, R, d // 2, dtype=torch.uint8, device=DEVICE)
            s[name + "s"] = torch.full((n, h_kv, d // GROUP, R), 127, dtype=torch.uint8, device=DEVICE).view(torch.float8_e8m0fnu)
        _back(s, c, rows)
        if own:
            from paper_2609_30738_amd import _lib
            s["batch"] = _lib.Batch(c["dtype"], c["h_q"], h_kv, d, 8, [L] * P, device=DEVICE)
        return s
    lens, tokens = _rows_and_tokens(c)
    s["table"], n = _table(gen, np.maximum(_blocks(lens, R), 1), 3)
    s["len"] = _dev(lens)
    _fill(s, c, gen, n, lens)
    if c["kind"] == "rows":
        _back(s, c, lens)
        return s
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


def _back(s, c, lens):
    """The handle, and room for the caches' rows: problem p at row_off[p] h_kv d elements, [h_kv][rows][d]."""
    if c["qtype"] == "e2m1" or c["kind"] == "rows":
        off = np.concatenate([[0], np.cumsum(lens)])
        s["row_off"] = _dev(off, torch.int64)
        s["row_prob"] = _dev(np.repeat(np.arange(len(lens)), lens), torch.int64)
        for name in ("k_rows", "v_rows"):
            s[name] = torch.zeros(int(off[-1]) * c["h_kv"] * c["d"], dtype=_dtype(c), device=DEVICE)
    if own:
        s["pc"] = _handle(c, s, int(np.max(lens)))


def _fill(s, c, gen, n, lens):
    """Pools whose used rows hold quantised normal values (a few dominant keys among them); the rows behind each
    problem's last one hold what memory happened to hold."""
    R, h_kv, d = c["block_rows"], c["h_kv"], c["d"]
    four = c["qtype"] == "e2m1"
    lens_d = _dev(lens, torch.int64)
    at = s["table"].long().gather(1, (lens_d[:, None] // R).clamp(max=s["table"].shape[1] - 1))[:, 0]
    part = lens_d < R * (s["table"] >= 0).sum(1)
    behind = (torch.arange(R, device=DEVICE)[None] >= (lens_d % R)[:, None])[part][:, None, :, None]
    for name in ("k", "v"):
        q = torch.empty(n, h_kv, R, d // 2 if four else d, dtype=torch.uint8, device=DEVICE)
        sc = torch.empty(n, h_kv, d // GROUP, R, dtype=torch.uint8, device=DEVICE) if four else torch.empty(n, h_kv, device=DEVICE)
        for i in range(0, n, 4096):
            x = torch.randn(min(4096, n - i), h_kv, R, d, device=DEVICE, generator=gen)
            if name == "k":
                x *= torch.where(torch.rand(*x.shape[:3], 1, device=DEVICE, generator=gen) < 3e-4, 4.0, 1.0)
            if four:
                q[i:i + 4096], b = _codes4(x)
                sc[i:i + 4096] = b.transpose(2, 3)
            else:
                sc[i:i + 4096] = _scale_of(x.abs().amax((2, 3)), c)
                q[i:i + 4096] = _codes(x, sc[i:i + 4096][..., None, None], c).view(torch.uint8)
        keep = q[at[part]]
        q[at[part]] = torch.where(behind, torch.full_like(keep, 0x7F), keep)
        if four:
            keep = sc[at[part]]
            sc[at[part]] = torch.where(behind.transpose(2, 3), torch.full_like(keep, 200), keep)
            s[name + "q"], s[name + "s"] = q, sc.view(torch.float8_e8m0fnu)
        else:
            s[name + "q"], s[name + "s"] = q.view(torch.float8_e4m3fn if c["qtype"] == "e4m3" else torch.int8), sc


def _handle(c, s, max_len):
    from paper_2609_30738_amd import _lib
    pool = (lambda x: x.view(torch.float4_e2m1fn_x2)) if c["qtype"] == "e2m1" else (lambda x: x)
    return _lib.PagedCache(c["dtype"], c["h_q"], pool(s["kq"]), pool(s["vq"]), s["ks"], s["vs"], s["table"], s["len"], max_len)


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2609_30738_amd import _lib
    c = s["case"]
    if c["kind"] == "rotate":
        _lib.rotate(s["rot"], s["x"], s["pos"], s["out"])
    elif c["kind"] == "append":
        if c["rot"]:
            _lib.paged_append_rotated(s["pc"], s["rot"], s["pos"], s["k_new"], s["v_new"], s["slots"],
                                      q=s["q"] if c["q"] else None, q_out=s["q_out"])
        else:
            _lib.paged_append(s["pc"], s["k_new"], s["v_new"], s["slots"])
    elif c["kind"] == "compact":
        _lib.paged_compact(s["batch"], s["k"], s["v"], s["sel"], s["budget"], c["tail"], s["pc"])
    elif c["kind"] == "attend":
        off = s["tok_off"] if c["tokens"] > 1 else None
        _lib.paged_attention(s["pc"], s["q"], s["scale"], s["out"], tok_off=off, max_q=s["max_q"], ws=s["ws"])
    if "row_off" in s:
        _lib.paged_rows(s["pc"], s["row_off"], s["k_rows"], s["v_rows"])
    return _outputs(s)


def _outputs(s):
    c = s["case"]
    if c["kind"] in ("rotate", "attend"):
        return dict(out=s["out"])
    out = dict(k_rows=s["k_rows"], v_rows=s["v_rows"]) if "row_off" in s else dict(k=s["kq"], v=s["vq"])
    if c["kind"] != "rows":
        out.update(k_scale=s["ks"], v_scale=s["vs"])
    if c["kind"] == "append" and c["q"]:
        out["q"] = s["q_out"]
    return out


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rotate":
        s["out"].copy_(_turned(s, s["x"], -1 if c["inverse"] else 1))
    elif c["kind"] == "append":
        k = _turned(s, s["k_new"]) if c["rot"] else s["k_new"].float()
        (_plain_append4 if c["qtype"] == "e2m1" else _plain_append)(s, k, s["v_new"].float())
        if c["q"]:
            s["q_out"].copy_(_turned(s, s["q"]))
    elif c["kind"] == "compact":
        _plain_compact(s)
    elif c["kind"] == "attend":
        _plain_attend(s)
    if "row_off" in s:
        _plain_rows(s)
    return _outputs(s)


def _turned(s, x, sign=1):
    """Rows x [T, heads, d] rotated, in 32 bits (the angles in 64)."""
    c = s["case"]
    r = c["rot"]
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = (angle.cos() * s["factor"]).float()[:, None], (angle.sin() * (sign * s["factor"])).float()[:, None]
    x = x.float()
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)


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


def _codes4(x):
    """Rows [.., d] in fp32 as 4-bit codes [.., d / 2] and their scales' bytes [.., d / 32]."""
    x = x.unflatten(-1, (-1, GROUP))
    m, e = torch.frexp(x.abs().amax(-1))
    # 6 = 0.75 2^3
    b = torch.where(m > 0, e - 3 + (m > 0.75) + 127, torch.zeros_like(e)).clamp(2, 252).to(torch.int32)
    y = x * ((254 - b) << 23).view(torch.float32)[..., None]
    a = y.abs()
    code = torch.signbit(y).to(torch.uint8) << 3
    for i, edge in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):  # halfway goes to the even code
        code += (a >= edge) if i % 2 else (a > edge)
    code = code.flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, b.to(torch.uint8)


def _values4(codes, scales):
    """Codes [.., R, d / 2] and scales [.., d / 32, R] as fp32 rows [.., R, d]."""
    grid = torch.tensor(GRID, device=codes.device)
    grid = torch.cat([grid, -grid])
    x = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], -1).flatten(-2)
    s = (scales.view(torch.uint8).int() << 23).view(torch.float32).transpose(-1, -2)
    return (x.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


def _take(pool, ids):
    """Blocks of a pool by their numbers."""
    return pool.view(torch.uint8)[ids].view(pool.dtype) if pool.element_size() == 1 else pool[ids]


def _block_values(s, name, ids):
    """Blocks by their numbers as fp32 [.., h_kv, R, d]."""
    codes, scale = _take(s[name + "q"], ids), _take(s[name + "s"], ids)
    return _values4(codes, scale) if s["case"]["qtype"] == "e2m1" else codes.float() * scale[..., None, None]


def _plain_append(s, k, v):
    c = s["case"]
    R = c["block_rows"]
    slots = s["slots"].long()
    block, row = slots // R, slots % R
    first = torch.ones_like(slots, dtype=torch.bool)
    first[1:] = (slots[1:] != slots[:-1] + 1) | (row[1:] == 0)
    for x, pool, scale in ((k, s["kq"], s["ks"]), (v, s["vq"], s["vs"])):
        amax = torch.zeros_like(scale).index_reduce_(0, block, x.abs().amax(2), "amax")
        # blocks that get rows, with the number of rows they held before
        b, held = block[first], row[first]
        old = torch.where(held[:, None] > 0, scale[b], torch.zeros_like(scale[b]))
        to = torch.maximum(old, _scale_of(amax[b], c))
        # the old rows of blocks in use move to the new scale
        u = held > 0
        keep = torch.arange(R, device=DEVICE)[None, None, :, None] < held[u][:, None, None, None]
        codes = _take(pool, b[u])
        moved = _codes(codes.float() * old[u][..., None, None], to[u][..., None, None], c)
        bytes_ = pool.view(torch.uint8)
        bytes_[b[u]] = torch.where(keep, moved.view(torch.uint8), codes.view(torch.uint8))
        scale[b] = to
        bytes_[block, :, row] = _codes(x, scale[block][..., None], c).view(torch.uint8)


def _plain_append4(s, k, v):
    R = s["case"]["block_rows"]
    slots = s["slots"].long()
    for x, name in ((k, "k"), (v, "v")):
        codes, b = _codes4(x)
        s[name + "q"][slots // R, :, slots % R] = codes
        s[name + "s"].view(torch.uint8)[slots // R, :, :, slots % R] = b


def _plain_compact(s):
    c = s["case"]
    P, h_kv, L, d = s["k"].shape
    R, tail, nb = c["block_rows"], c["tail"], s["table"].shape[1]
    n = s["budget"] + tail
    end = torch.arange(L - tail, L, device=DEVICE).expand(P, h_kv, tail)
    pos = torch.cat([s["sel"].long().sort(-1).values, end], -1)
    ids = s["table"].long()
    for name in ("k", "v"):
        codes, b = _codes4(s[name].gather(2, pos[..., None].expand(-1, -1, -1, d)).float())
        row = torch.arange(n, device=DEVICE)
        at = ids[:, row // R]  # [P, n]
        s[name + "q"][at, :, row % R] = codes.transpose(1, 2)
        s[name + "s"].view(torch.uint8)[at, :, :, row % R] = b.transpose(1, 2)


def _plain_rows(s):
    c = s["case"]
    h_kv, d, R = c["h_kv"], c["d"], c["block_rows"]
    p, off = s["row_prob"], s["row_off"]
    row = torch.arange(p.numel(), device=DEVICE) - off[p]
    n = s["len"].long()[p]
    # element [head][row][d] of problem p, in its place
    at = ((off[p] * h_kv + row)[:, None] + n[:, None] * torch.arange(h_kv, device=DEVICE)).flatten()
    ids = s["table"].long()[p, row // R]
    for name in ("k", "v"):
        x = s[name + "q"].view(torch.uint8)[ids, :, row % R].view(s[name + "q"].dtype)
        if c["qtype"] == "e2m1":
            x = _values4(x[:, :, None], s[name + "s"].view(torch.uint8)[ids, :, :, row % R][..., None])[:, :, 0]
        else:
            x = x.float() * s[name + "s"][ids][..., None]
        s[name + "_rows"].view(-1, d)[at] = x.reshape(-1, d).to(s[name + "_rows"].dtype)


def _plain_attend(s):
    c = s["case"]
    P, h_q, h_kv, d, R = c["n_prob"], c["h_q"], c["h_kv"], c["d"], c["block_rows"]
    G, n_max, L = h_q // h_kv, s["max_q"], s["table"].shape[1] * R
    ids = s["table"].long().clamp(min=0)
    lens, off = s["len"].long(), s["tok_off"].long()
    row = torch.arange(L, device=DEVICE)
    used = (row < lens[:, None])[:, None, :, None]

    def rows(name):
        x = _block_values(s, name, ids)  # [P, blocks, h_kv, R, d]
        return torch.where(used, x.transpose(1, 2).reshape(P, h_kv, L, d), torch.zeros((), device=DEVICE))

    k = rows("k")
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
    o = torch.matmul(t, rows("v")).div_(torch.where(z > 0, z, torch.ones_like(z)))
    o = o.view(P, h_kv, n_max, G, d).permute(0, 2, 1, 3, 4).reshape(P, n_max, h_q, d)
    s["out"][tok[live]] = o[live].to(s["out"].dtype)


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    e, d = 2 if c["dtype"] == "bf16" else 4, c["d"]
    if c["kind"] == "rotate":
        n = c["tokens"] * c["h_q"]
        return {"bytes": 2 * n * d * e + 4 * c["tokens"], "flops": 3 * n * c["rot"]}
    R, h_kv, four = c["block_rows"], c["h_kv"], c["qtype"] == "e2m1"
    held = d / 2 + d / GROUP if four else d  # bytes of a row in the cache (without the scales of 8-bit blocks)
    if c["kind"] == "append":
        cached, add = _cached_and_added(c)
        T = int(add.sum())
        n = 2 * T * h_kv * (d * e + held) + (4 + 4 * (c["rot"] > 0)) * T + 2 * T * c["h_q"] * d * e * c["q"]
        if four:  # the caches' rows read and written
            n += 2 * int((cached + add).sum()) * h_kv * (held + d * e)
        else:
            n += 8 * int((_blocks(cached + add, R) - cached // R)[add > 0].sum()) * h_kv
        return {"bytes": n, "flops": 3 * T * c["rot"] * (h_kv + c["h_q"] * c["q"]) + 2 * T * h_kv * d}
    if c["kind"] == "compact":
        n = c["layers"] * (min(c["budget"], c["L"] - c["tail"]) + c["tail"]) * h_kv
        return {"bytes": 4 * n * (d * e + held) + 4 * c["layers"] * c["budget"] * h_kv, "flops": 2 * n * d}
    lens, tokens = _rows_and_tokens(c)
    scales = 0 if four else 8 * int(_blocks(lens, R).sum()) * h_kv
    if c["kind"] == "rows":
        n = 2 * int(lens.sum()) * h_kv
        return {"bytes": n * (d * e + held) + scales, "flops": n * d}
    seen = sum(int(n) * int(L - n) + int(n) * (int(n) + 1) // 2 for L, n in zip(lens, tokens) if L >= n)
    read = int(lens[tokens > 0].sum())
    return {"bytes": 2 * read * h_kv * held + 2 * int(tokens.sum()) * c["h_q"] * d * e, "flops": 4 * seen * c["h_q"] * d}


# ------------------------------------------------------------------------------------------------
# The same from the definition, in 64 bits
# ------------------------------------------------------------------------------------------------

def _turned64(s, x, sign=1):
    """x as complex numbers, times factor exp(i p f)."""
    c = s["case"]
    r = c["rot"]
    x = x.double()
    z = torch.polar(torch.full((), s["factor"], dtype=torch.float64, device=DEVICE).expand(x.shape[0], r // 2).contiguous(),
                    sign * s["pos"].double()[:, None] * s["freq"])[:, None]
    if c["layout"] == "half":
        y = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * z
        return torch.cat([y.real, y.imag, x[..., r:]], -1)
    y = torch.view_as_complex(x[..., :r].reshape(*x.shape[:2], r // 2, 2).contiguous()) * z
    return torch.cat([torch.view_as_real(y).reshape(*x.shape[:2], r), x[..., r:]], -1)


def _decode64(codes):
    """8-bit codes as the numbers they stand for, from their bits."""
    if codes.dtype == torch.int8:
        return codes.double()
    u = codes.view(torch.uint8).int()
    e, f = (u >> 3) & 15, (u & 7).double()
    x = torch.where(e > 0, (1.0 + f / 8) * torch.exp2((e - 7).double()), f * 2.0 ** -9)
    x = torch.where((u & 0x7F) == 0x7F, torch.full_like(x, math.nan), x)
    return torch.where(u >= 128, -x, x)


def _values64(s, name, ids, g):
    """Blocks ids of head g as numbers [blocks, R, d]."""
    codes, scale = _take(s[name + "q"], ids)[:, g], _take(s[name + "s"], ids)[:, g]
    if s["case"]["qtype"] != "e2m1":
        return _decode64(codes) * scale.double()[:, None, None]
    u = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    e, f = u >> 1 & 3, (u & 1).double()
    x = torch.where(e > 0, (1.0 + f / 2) * torch.exp2((e - 1).double()), f / 2)
    x = torch.where(u >= 8, -x, x)
    p = torch.exp2(scale.view(torch.uint8).double() - 127).transpose(1, 2)
    return x * p.repeat_interleave(GROUP, -1)


def _grid64(x, top):
    """x rounded to the nearest number with so many steps to a binade (e4m3: 8 down to 2^-6, e2m1: 2 down to 1) or to whole
    ones (0), ties to even."""
    if top == 0:
        return x.round()
    least = 2.0 ** -6 if top == 8 else 1.0
    e = torch.frexp(x.abs().clamp(min=least))[1].double() - 1
    step = torch.exp2(e) / top
    return (x / step).round() * step


def _least64(amax, qmax, lowest=-126):
    e = torch.ceil(torch.log2((amax / qmax).clamp(min=2.0 ** lowest)))
    e = torch.where(amax <= qmax * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax > qmax * torch.exp2(e), e + 1, e)
    return torch.exp2(e.clamp(min=lowest))


def _coded4_64(x):
    """Rows [.., d] as a 4-bit cache holds them, and their scales [.., d / 32]."""
    x = x.unflatten(-1, (-1, GROUP))
    s = _least64(x.abs().amax(-1), 6.0, -125)
    return (_grid64(x / s[..., None], 2) * s[..., None]).flatten(-2), s


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "rotate":
        return dict(out=_turned64(s, s["x"], -1 if c["inverse"] else 1))
    if c["kind"] == "attend":
        return dict(out=_attend64(s, c))
    R = c["block_rows"]
    if c["kind"] == "append" and c["qtype"] != "e2m1":
        return _append64(s, c)
    out = {}
    lens = s["len"].tolist()
    if sum(-(-n // R) for n in lens) > 60000:
        return None
    for name in ("k", "v"):
        rows = []
        scale = s[name + "s"].double()
        t = 0
        for p, n in enumerate(lens):
            ids = s["table"][p, :-(-n // R)].long()
            if c["kind"] == "compact":
                kept = s["sel"][p].long().sort(1).values
                at = torch.cat([kept, torch.arange(c["L"] - c["tail"], c["L"], device=DEVICE).expand(c["h_kv"], -1)], 1)
                x, sc = _coded4_64(s[name][p].gather(1, at[..., None].expand(-1, -1, c["d"])).double())
                r0 = 0
            else:
                x = torch.stack([_values64(s, name, ids, g).reshape(-1, c["d"])[:n] for g in range(c["h_kv"])])
            if c["kind"] == "append":
                add = int(_cached_and_added(c)[1][p])
                new = s[name + "_new"][t:t + add]
                if name == "k" and c["rot"]:
                    sub = dict(s, pos=s["pos"][t:t + add])
                    new = _turned64(sub, new)
                new, sc = _coded4_64(new.double().transpose(0, 1))
                x = torch.cat([x[:, :n - add], new], 1)
                r0, t = n - add, t + add
            if c["kind"] != "rows" and n > r0:
                row = torch.arange(r0, n, device=DEVICE)
                scale[ids[row // R], :, :, row % R] = sc.transpose(0, 1)
            rows.append(x.flatten())
        out[name + "_rows"] = torch.cat(rows)
        out[name + "_scale"] = scale
    if c["kind"] == "rows":
        return dict(k_rows=out["k_rows"], v_rows=out["v_rows"])
    if c["kind"] == "append" and c["q"]:
        out["q"] = _turned64(s, s["q"])
    return out


def _append64(s, c):
    """New rows into 8-bit blocks, block by block."""
    cached, add = _cached_and_added(c)
    R, e4m3 = c["block_rows"], c["qtype"] == "e4m3"
    if int(_blocks(cached + add, R).sum()) + c["n_prob"] > 4000:
        return None
    pools, scales = [_decode64(s["kq"]), _decode64(s["vq"])], [s["ks"].double(), s["vs"].double()]
    k, v, at = _turned64(s, s["k_new"]), s["v_new"].double(), 0
    qmax, top = (448.0, 8) if e4m3 else (127.0, 0)
    for p in range(c["n_prob"]):
        r, end = int(cached[p]), int(cached[p] + add[p])
        while r < end:
            b, lo = int(s["table"][p, r // R]), r % R
            n = min(R - lo, end - r)
            for x, pool, sc in ((k, pools[0], scales[0]), (v, pools[1], scales[1])):
                new = x[at:at + n].transpose(0, 1)
                was = sc[b] if lo else torch.zeros_like(sc[b])
                amax = new.abs().amax((1, 2))
                to = torch.maximum(was, torch.where(amax > 0, _least64(amax, qmax), torch.zeros_like(amax)))
                div = torch.where(to > 0, to, torch.ones_like(to))[:, None, None]
                if lo:
                    pool[b, :, :lo] = _grid64(pool[b, :, :lo] * was[:, None, None] / div, top)
                pool[b, :, lo:lo + n] = _grid64(new / div, top)
                sc[b] = to
            at += n
            r += n
    out = dict(k=pools[0] if e4m3 else None, v=pools[1] if e4m3 else None, k_scale=scales[0], v_scale=scales[1])
    if c["q"]:
        out["q"] = _turned64(s, s["q"])
    return out


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
                k, v = (_values64(s, x, ids, g).reshape(-1, d)[:L] for x in "kv")
                q = s["q"][at:at + n, g * G:(g + 1) * G].double()
                for h in range(G):
                    t = (q[:, h] @ k.T * s["scale"]).masked_fill_(~seen, -math.inf)
                    out[at:at + n, g * G + h] = t.softmax(-1) @ v
        at += n
    return out
