"""Workloads of the paged packed KV cache: append with the position rotation on the way, attention with a sliding window and
first tokens that stay visible, and reading tokens back to 16 bits.

A pool holds packed pages of 128 tokens, [pool page][KV head][page bytes], in the library's page layout (token-wise groups); a
block table names the pool page of every 128 tokens of a sequence.  Calls are ragged: rows cu[b] .. cu[b + 1] - 1 of a call are
the LAST cu[b + 1] - cu[b] of the seq_len[b] tokens of sequence b, so row i stands at position seq_len[b] - (cu[b + 1] - cu[b]) +
i - cu[b].  Rows from cu[batch] on are padding and stay as they were.  A case is one pass of one of three kinds:

  append   rotate q and k by position, quantize k and v into the pool; returned: q and the stored values as 16-bit numbers;
  attend   a row at position p sees the tokens t <= p that are also t > p - window or t < sinks (window 0: all of them);
  restore  the tokens of every sequence back to 16 bits, as a preempted request is handed to a dense kernel.

Where `own` is false the operators are computed in their plain form: elementary torch operations in 32 bits, rounded once.
Shapes are those of the model-shaped caches that the rest of the repository is measured on.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 128
# query heads, KV heads, head_dim, type, key / value group, longest context
SHAPES = {"tiny": (8, 8, 64, "fp16", 32, 512), "1b": (32, 8, 64, "fp16", 64, 4096),
          "8b": (32, 8, 128, "bf16", 128, 32768), "70b": (64, 8, 128, "bf16", 128, 131072)}
WIDTHS = {"tiny": [(4, 2)], "1b": [(4, 2)], "8b": [(4, 2), (2, 4), (4, 4), (8, 4)], "70b": [(4, 2)]}
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
MAX_FLOPS, MAX_BYTES, MAX_PAIRS = 5.6e11, 8.5e8, 5.5e8      # of a drawn case: no more than the largest listed ones


def _case(kind, shape, name=None, **over):
    c = {"kind": kind, "shape": shape, "kb": WIDTHS[shape][0][0], "vb": WIDTHS[shape][0][1], "batch": 1, "tokens": SHAPES[shape][5],
         "rows": 1, "ragged": False, "window": 0, "sinks": 0, "rotary": SHAPES[shape][2], "interleaved": False, "pad": 0}
    c.update(over)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: one token of one sequence, where launches are everything
        _case("append", "tiny", "append_tiny_1", tokens=512),
        # a decoding step of a full batch: one token a sequence, long and uneven contexts
        _case("append", "8b", "append_8b_step64", batch=64, tokens=32768, ragged=True),
        # a continuous batch: chunks of prompts of uneven lengths that start inside a page, padded for a captured graph
        _case("append", "1b", "append_1b_mixed", batch=8, tokens=4001, rows=601, ragged=True, rotary=32, interleaved=True, pad=77),
        # prompts taken in whole
        _case("append", "8b", "append_8b_prefill", batch=4, tokens=8192, rows=8192),
        # one short sequence with a narrow window
        _case("attend", "tiny", "decode_tiny_window", tokens=509, window=100, sinks=4),
        # decoding over the whole context
        _case("attend", "8b", "decode_8b_32k", batch=16, tokens=32767),
        # streaming decode of a large uneven batch: a 4k window and four first tokens, equal widths, a padded batch
        _case("attend", "8b", "decode_8b_k4v4_window", batch=64, tokens=20001, vb=4, ragged=True, window=4096, sinks=4, pad=3),
        # eight query heads per KV head at a 128k context
        _case("attend", "70b", "decode_70b_128k", batch=4, tokens=131071),
        # three drafted tokens a sequence verified at once, window and sinks that end inside a page
        _case("attend", "1b", "draft_1b_window", batch=8, tokens=4096, rows=3, ragged=True, window=1000, sinks=16),
        # chunks of prompts on top of a cached context
        _case("attend", "8b", "chunk_8b_window", batch=2, tokens=16001, rows=700, ragged=True, window=4096, sinks=4),
        # a whole prompt against its own cache
        _case("attend", "8b", "prefill_8b_8k", tokens=8192, rows=8192),
        # preempted requests back to 16 bits
        _case("restore", "8b", "restore_8b_8k", batch=4, tokens=8001, rows=8001, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "restore"])
        shape = rng.choice(["8b", "8b", "8b", "70b", "1b", "tiny"])
        D, top = SHAPES[shape][2], SHAPES[shape][5]
        c = _case(kind, shape, batch=_log_int(rng, 1, 64), tokens=_log_int(rng, 1, top), ragged=rng.random() < 0.6, pad=rng.choice([0, 0, 1, 13]))
        c["kb"], c["vb"] = rng.choice(WIDTHS[shape])
        form = rng.random()
        if kind == "restore":
            c["rows"] = c["tokens"]
        elif form > 0.4:
            c["rows"] = min(c["tokens"], rng.randint(2, 8) if form < 0.55 else _log_int(rng, 2, 8192))
        if kind == "append":
            c["rotary"] = rng.choice([D, D, D // 2])
            c["interleaved"] = rng.random() < 0.3
        if kind == "attend" and rng.random() < 0.6:
            c["window"] = _log_int(rng, 1, c["tokens"])
            c["sinks"] = rng.choice([0, 1, 4, 16, 64, 200])
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and _padded_pairs(c) <= MAX_PAIRS:
            return c


# ------------------------------------------------------------------------------------------------- sizes of a case
def _sizes(c):
    """(tokens after the call, rows of the call) per sequence: the last sequence has all of them, the others at least half."""
    lens, rows = [], []
    for b in range(c["batch"]):
        cut = ((b + 1) * 7919) % 1009 / 1009.0 if c["ragged"] and b + 1 < c["batch"] else 0.0
        n = max(1, c["tokens"] - int(cut * (c["tokens"] // 2)))
        r = max(1, c["rows"] - int((1.0 - cut) * cut * 2 * c["rows"]))
        lens.append(n)
        rows.append(n if c["kind"] == "restore" else min(n, r))
    return lens, rows


def _visible_pages(c, n, r):
    """Logical pages of a sequence of n tokens that its last r rows see some token of."""
    low = max(0, n - r - c["window"] + 1) // PAGE if c["kind"] == "attend" and c["window"] else 0
    first = min(-(-c["sinks"] // PAGE), low)
    return list(range(first)) + list(range(low, -(-n // PAGE)))


def _visible(c, n, r):
    """(pairs of a row and a token that it sees, tokens that some row sees) of a sequence."""
    W, S = c["window"], c["sinks"]
    if not W:
        return r * n - r * (r - 1) // 2, n
    pairs = sum(min(p + 1, W) + min(S, max(0, p + 1 - W)) for p in range(n - r, n))
    low = max(0, n - r - W + 1)
    return pairs, n - low + min(S, low)


def _padded_pairs(c):
    """Entries of the plain form's score matrix, over the query heads (and its keys where those are more)."""
    if c["kind"] != "attend":
        return 0
    lens, rows = _sizes(c)
    pages = max(len(_visible_pages(c, n, r)) for n, r in zip(lens, rows))
    hq, hkv, D = SHAPES[c["shape"]][:3]
    return c["batch"] * pages * PAGE * max(max(rows) * hq // 4, hkv * D // 2)


def _packed(c):
    """Packed bytes of a token of a KV head."""
    D, g = SHAPES[c["shape"]][2], SHAPES[c["shape"]][4]
    return D * (c["kb"] + c["vb"]) // 8 + 8 * (D // g)


def work(case):
    c = case
    hq, hkv, D = SHAPES[c["shape"]][:3]
    lens, rows = _sizes(c)
    n = sum(rows)
    if c["kind"] == "append":
        table = 8 * (c["rotary"] // 2) * len({p for m, r in zip(lens, rows) for p in range(m - r, m)})
        return {"bytes": n * (2 * D * (2 * hq + 2 * hkv) + hkv * (2 * _packed(c) + 4 * D)) + table, "flops": n * D * (3 * hq + 15 * hkv)}
    if c["kind"] == "restore":
        return {"bytes": n * hkv * (_packed(c) + 4 * D), "flops": n * hkv * 4 * D}
    seen = [_visible(c, m, r) for m, r in zip(lens, rows)]
    return {"bytes": sum(t for _, t in seen) * hkv * _packed(c) + 4 * n * hq * D, "flops": 4 * D * hq * sum(p for p, _ in seen)}


# -------------------------------------------------------------------------------------------------------- the page
def _regions(c):
    """Byte sizes of a page's regions: key codes, key metadata, value codes, value metadata."""
    D, g = SHAPES[c["shape"]][2], SHAPES[c["shape"]][4]
    return PAGE * D * c["kb"] // 8, PAGE * (D // g) * 4, PAGE * D * c["vb"] // 8, PAGE * (D // g) * 4


def _quantize(x, bits, g):
    """Codes (fp32 whole numbers) and fp16 (scale, zero) of groups of g along the last axis."""
    y = x.unflatten(-1, (-1, g))
    mn, mx = y.amin(-1, keepdim=True) + 0.0, y.amax(-1, keepdim=True) + 0.0
    top = float((1 << bits) - 1)
    s16 = ((mx - mn) / torch.tensor(top, device=x.device)).clamp_(-65504.0, 65504.0).half()      # (a tensor: a true division)
    z16 = mn.clamp(-65504.0, 65504.0).half()
    s, z = s16.float(), z16.float()
    inv = torch.where(s != 0, 1.0 / s, torch.zeros_like(s))
    code = ((y - z) * inv).round_().clamp_(0.0, top)
    return code, s16, z16


def _values(code, s16, z16):
    """scale x code + zero, rounded once to 32 bits."""
    return (code.double() * s16.double() + z16.double()).float().flatten(-2)


def _pack_keys(code, bits):
    """uint8 codes [..., 128, D] -> bytes [..., 128 D bits / 8]."""
    D, f = code.shape[-1], 8 // bits
    w = D * bits // 128
    q = min(w, 4)
    y = code.unflatten(-1, (w // q, q, f, 4, 4))                   # token, quad, word, field, chunk, byte
    y = sum(y[..., i, :, :] << (bits * i) for i in range(f))
    return y.transpose(-2, -3).flatten(-5)


def _unpack_keys(data, bits, D):
    f = 8 // bits
    w = D * bits // 128
    q = min(w, 4)
    y = data.unflatten(-1, (PAGE, w // q, 4, q, 4))
    y = torch.stack([(y >> (bits * i)) & ((1 << bits) - 1) for i in range(f)], -1)
    n = y.dim() - 6
    return y.permute(*range(n), n, n + 1, n + 3, n + 5, n + 2, n + 4).flatten(-5)


def _pack_values(code, bits):
    D, f = code.shape[-1], 8 // bits
    # token = (block, half, high, t, low), channel = (word, field, row half, lane)
    y = code.unflatten(-1, (D // 16 // f, f, 2, 8)).unflatten(-5, (4, 2, 2, 4, 2))
    y = sum(y[..., i, :, :] << (bits * i) for i in range(f))
    n = y.dim() - 8
    k, hi, t, lo, w, r, g = (n + i for i in range(1, 8))
    return y.permute(*range(n), n, w, g, t, r, k, lo, hi).flatten(-8)


def _unpack_values(data, bits, D):
    f = 8 // bits
    y = data.unflatten(-1, (4, D // 16 // f, 8, 4, 2, 2, 2, 2))    # block, word, lane, t, row half, half, low, high
    y = torch.stack([(y >> (bits * i)) & ((1 << bits) - 1) for i in range(f)], -1)
    n = y.dim() - 9
    w, g, t, r, k, lo, hi, fi = (n + i for i in range(1, 9))
    return y.permute(*range(n), n, k, hi, t, lo, w, fi, r, g).flatten(-9, -5).flatten(-4)


def _unpack_page(data, c):
    """(code, scale, zero) in fp32 of keys and of values of packed pages [..., page bytes]."""
    D, g = SHAPES[c["shape"]][2], SHAPES[c["shape"]][4]
    k, km, v, vm = data.split(_regions(c), -1)
    out = []
    for codes, meta in ((_unpack_keys(k, c["kb"], D), km), (_unpack_values(v, c["vb"], D), vm)):
        m = meta.contiguous().view(torch.float16).unflatten(-1, (PAGE, D // g, 2)).float()
        out.append((codes.unflatten(-1, (-1, g)).float(), m[..., :1], m[..., 1:]))
    return out


# ---------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _spread_keys(c, x):
    """Keys [..., KV head, token, channel] as the model-shaped caches have them: heavy channels, the same for a head's tokens."""
    D = x.shape[-1]
    at = (torch.arange(x.shape[-3], device=x.device)[:, None] * 37 + torch.arange(8, device=x.device) * 29) % D
    heavy = torch.zeros(x.shape[-3], D, device=x.device).scatter_(1, at, 1.0)[:, None]
    return x * {"tiny": 1.0 + heavy, "1b": 1.0 + heavy, "8b": 1.0 + 3.0 * heavy, "70b": 3.0 + 0.0 * heavy}[c["shape"]]


def _table(c, lens, rows, gen):
    """Block table with the pages that a program still holds (-1: never written, or fallen out of the window), and the pool's size."""
    width = -(-max(lens) // PAGE)
    held = [_visible_pages(c, n, r) for n, r in zip(lens, rows)]
    count = sum(len(h) for h in held)
    pool = count + max(2, count // 16)
    ids = torch.randperm(pool, generator=gen, device="cuda")[:count].to(torch.int32)
    b = torch.tensor([b for b, h in enumerate(held) for _ in h], device="cuda")
    i = torch.tensor([i for h in held for i in h], device="cuda")
    table = torch.full((c["batch"], width), -1, dtype=torch.int32, device="cuda")
    table[b, i] = ids
    return table, pool, b, i, ids.long()


def prepare(case, seed):
    c = case
    hq, hkv, D, dt, g, _ = SHAPES[c["shape"]]
    lens, rows = _sizes(c)
    gen = _gen(seed)
    n = sum(rows) + c["pad"]
    s = {"case": dict(c), "max_rows": max(rows), "pages_seen": max(len(_visible_pages(c, m, r)) for m, r in zip(lens, rows)),
         "seq_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "cu": torch.tensor([0] + rows, dtype=torch.int32, device="cuda").cumsum(0, dtype=torch.int32)}
    table, pool, b, i, ids = _table(c, lens, rows, gen)
    s["table"] = table
    # the pool as an allocator hands it out: whatever was there (here: bytes that read as NaN scales)
    pages = torch.full((pool, hkv, sum(_regions(c))), 255, dtype=torch.uint8, device="cuda")
    s["pages"] = pages
    if c["kind"] == "append":
        # what the projection leaves: q, k and v of a token side by side
        x = torch.randn(n, hq + 2 * hkv, D, generator=gen, device="cuda")
        x[:, hq:hq + hkv] = _spread_keys(c, x[:, hq:hq + hkv].transpose(0, 1)).transpose(0, 1)
        s["qkv"] = x.to(DTYPES[dt])
        half = c["rotary"] // 2
        freq = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(max(lens), dtype=torch.float64, device="cuda")[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_out"] = torch.zeros(n, hq, D, dtype=DTYPES[dt], device="cuda")
    else:
        where = torch.arange(0, len(ids), 256, device="cpu").tolist()
        for lo in where:                                          # in pieces, so that the 32-bit copies stay small
            part, pb, pi = ids[lo:lo + 256], b[lo:lo + 256], i[lo:lo + 256]
            k = _spread_keys(c, torch.randn(len(part), hkv, PAGE, D, generator=gen, device="cuda"))
            v = torch.randn(len(part), hkv, PAGE, D, generator=gen, device="cuda")
            behind = (pi[:, None] * PAGE + torch.arange(PAGE, device="cuda") >= s["seq_len"][pb][:, None])[:, None, :, None]
            region = []
            for x, bits, pack in ((k, c["kb"], _pack_keys), (v, c["vb"], _pack_values)):
                code, s16, z16 = _quantize(x.to(DTYPES[dt]).float(), bits, g)
                meta = torch.cat([s16, z16], -1).flatten(-2)
                meta = torch.where(behind, torch.full_like(meta, float("nan")), meta)      # tokens never written
                region += [pack(code.flatten(-2).to(torch.uint8), bits), meta.flatten(-2).contiguous().view(torch.uint8)]
            pages[part] = torch.cat(region, -1)
    if c["kind"] == "attend":
        s["q"] = torch.randn(n, hq, D, generator=gen, device="cuda").to(DTYPES[dt])
        s["out"] = torch.full((n, hq, D), 0.5, dtype=DTYPES[dt], device="cuda")
    else:
        s["k_out"] = torch.zeros(n, hkv, D, dtype=DTYPES[dt], device="cuda")
        s["v_out"] = torch.zeros(n, hkv, D, dtype=DTYPES[dt], device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------ plain forms
def _row_positions(s):
    """Sequence and position of every row of the call (padding: sequence 0, position 0), and which rows are not padding."""
    cu, n = s["cu"].long(), (s["q"] if "q" in s else s["k_out"]).shape[0]
    i = torch.arange(n, device="cuda")
    b = torch.searchsorted(cu[1:], i, right=True).clamp_(max=len(cu) - 2)
    there = i < cu[-1]
    return torch.where(there, b, 0), torch.where(there, s["seq_len"].long()[b] - cu[b + 1] + i, 0), there


def _rotate(x, cos, sin, c):
    """x [rows, heads, D] in fp32; cos, sin [rows, rotary / 2].  Every product and sum rounded on its own."""
    r = c["rotary"]
    co, si = cos[:, None], sin[:, None]
    y = x.clone()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    first, second = a * co - b * si, b * co + a * si
    if c["interleaved"]:
        y[..., 0:r:2], y[..., 1:r:2] = first, second
    else:
        y[..., :r // 2], y[..., r // 2:r] = first, second
    return y


def _append_plain(s):
    c = s["case"]
    hq, hkv, D, dt, g, _ = SHAPES[c["shape"]]
    _, pos, there = _row_positions(s)
    x = s["qkv"].float()
    cos, sin = s["cos"][pos], s["sin"][pos]
    q, k = _rotate(x[:, :hq], cos, sin, c), _rotate(x[:, hq:hq + hkv], cos, sin, c)
    new = {"q": q, "k": _values(*_quantize(k, c["kb"], g)), "v": _values(*_quantize(x[:, hq + hkv:], c["vb"], g))}
    old = {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    return {i: torch.where(there[:, None, None], new[i].to(DTYPES[dt]), old[i]) for i in new}


def _restore_plain(s):
    c = s["case"]
    b, pos, there = _row_positions(s)
    ids = s["table"].long()[b, pos // PAGE]
    used, at = torch.unique(ids, return_inverse=True)
    new = [_values(*side)[at, :, pos % PAGE] for side in _unpack_page(s["pages"][used], c)]
    return {i: torch.where(there[:, None, None], x.to(y.dtype), y) for i, x, y in zip("kv", new, (s["k_out"], s["v_out"]))}


def _attend_plain(s):
    c = s["case"]
    hq, hkv, D, dt, g, _ = SHAPES[c["shape"]]
    W, S, R, n = c["window"], c["sinks"], s["max_rows"], s["seq_len"].long()
    rows = (s["cu"][1:] - s["cu"][:-1]).long()
    # the pages that a sequence's rows see, and the tokens in them
    low = (n - rows - W + 1).clamp(min=0) // PAGE if W else torch.zeros_like(n)
    first = torch.clamp(low, max=-(-S // PAGE))
    i = torch.arange(s["pages_seen"], device="cuda")[None]
    page = torch.where(i < first[:, None], i, i - first[:, None] + low[:, None])
    held = page * PAGE < n[:, None]
    ids = torch.where(held, s["table"].long().gather(1, page.clamp(max=s["table"].shape[1] - 1)), 0)
    token = (page[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten(1)
    real = (token < n[:, None]) & held.repeat_interleave(PAGE, 1)
    k, v = (torch.where(real[:, None, :, None], (code * sc + z).flatten(-2).transpose(1, 2).flatten(2, 3), 0.0) for code, sc, z in _unpack_page(s["pages"][ids], c))
    # queries [sequence, KV head, row x head of the group, D]
    r = torch.arange(R, device="cuda")[None]
    at = (s["cu"][:-1, None].long() + r).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = (q @ k.transpose(-1, -2)).mul_(D ** -0.5).unflatten(2, (R, -1))
    pos = (n - rows)[:, None] + r
    t = token[:, None]
    sees = (t <= pos[..., None]) & real[:, None] & (r < rows[:, None])[..., None]
    if W:
        sees &= (t > pos[..., None] - W) | (t < S)
    x.masked_fill_(~sees[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.flatten(2, 3) @ v).unflatten(2, (R, -1)) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 2, 1, 3, 4).flatten(2, 3).to(DTYPES[dt])                     # [sequence, row, query head, D]
    out = s["out"].clone()
    there = (r < rows[:, None])
    out[at[there]] = o[there]
    return out


# ------------------------------------------------------------------------------------------------- the library's calls
def _handle(s):
    """What a serving program keeps: the configuration, the cache's handle and the scratch memory."""
    if "handle" not in s:
        from paper_2502_15075_b200 import kvq
        c = s["case"]
        hq, hkv, D, dt, g, _ = SHAPES[c["shape"]]
        cfg = kvq.make_config(c["batch"], hq, hkv, D, c["kb"], c["vb"], g, g, 0, DTYPES[dt], s["table"].shape[1] * PAGE)
        cache = kvq.PagedCache(cfg, pages=s["pages"], block_table=s["table"], seq_len=s["seq_len"])
        rope = kvq.Rope(s["cos"], s["sin"], c["interleaved"]) if c["kind"] == "append" else None
        ws = torch.empty(kvq.kvq_paged_workspace_bytes(cfg, s["max_rows"]), dtype=torch.uint8, device="cuda") if c["kind"] == "attend" else None
        if c["kind"] == "append":
            s["q"], s["k"], s["v"] = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
        s["handle"] = (kvq, cfg, cache, rope, ws)
    return s["handle"]


def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"append": _append_plain, "restore": _restore_plain, "attend": _attend_plain}[c["kind"]](s)
    kvq, cfg, cache, rope, ws = _handle(s)
    if c["kind"] == "attend":
        kvq.kvq_paged_attention(cfg, cache, s["q"], s["cu"], s["out"], ws, s["max_rows"], c["window"], c["sinks"])
        return s["out"]
    if c["kind"] == "append":
        kvq.kvq_paged_append(cfg, cache, s["k"], s["v"], s["cu"], rope, s["q"], s["q_out"])
    kvq.kvq_paged_dequantize(cfg, cache, s["cu"], s["k_out"], s["v_out"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]} if c["kind"] == "append" else {"k": s["k_out"], "v": s["v_out"]}


# ------------------------------------------------------------------------------------------ the definition in 64 bits
def _code_places(bits, D, values):
    """Byte in its region and bit of the code of (token, channel), from the page's description."""
    t, d = torch.meshgrid(torch.arange(PAGE, device="cuda"), torch.arange(D, device="cuda"), indexing="ij")
    f = 8 // bits
    if values:
        tau = t % 32
        u, m = tau % 16, d // 16
        byte = (t // 32) * (4 * D * bits) + (m // f) * 512 + (4 * (d % 8) + (u % 8) // 2) * 16 + 4 * (2 * ((d % 16) // 8) + tau // 16) + 2 * (u % 2) + u // 8
        return byte, bits * (m % f)
    word, quad = d // 16 // f, min(4, D * bits // 128)
    byte = t * (D * bits // 8) + (word // 4) * (16 * quad) + ((d % 16) // 4) * (4 * quad) + (word % 4) * 4 + d % 4
    return byte, bits * (d // 16 % f)


def _exact_pages(c, pages):
    """Keys and values in 64 bits [page, token, channel] of one KV head's packed pages [page, page bytes]."""
    D, g = SHAPES[c["shape"]][2], SHAPES[c["shape"]][4]
    sides, start = [], 0
    for bits, values in ((c["kb"], False), (c["vb"], True)):
        byte, bit = _code_places(bits, D, values)
        code = (pages[:, start + byte].to(torch.int32) >> bit) & ((1 << bits) - 1)
        start += PAGE * D * bits // 8
        meta = pages[:, start:start + PAGE * (D // g) * 4].contiguous().view(torch.float16).double().view(len(pages), PAGE, D // g, 2)
        start += PAGE * (D // g) * 4
        sides.append(code.double() * meta[..., 0].repeat_interleave(g, 2) + meta[..., 1].repeat_interleave(g, 2))
    return sides


def _exact_codes(x, bits, g):
    """x rounded to its group's 2^bits values, in 64 bits.  The quantizer is defined with a reciprocal, a difference and a product of 32
    bits: 16-bit inputs often lie on the border between two codes, and these roundings say which side they belong to."""
    y = x.reshape(*x.shape[:-1], -1, g)
    lo, hi = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
    scale = ((hi - lo) / (2 ** bits - 1)).clamp(-65504, 65504).to(torch.float16).double()
    zero = lo.clamp(-65504, 65504).to(torch.float16).double()
    inverse = torch.where(scale > 0, 1.0 / torch.where(scale > 0, scale, 1.0), 0.0).float().double()
    code = ((y - zero).float().double() * inverse).float().double().round().clamp(0, 2 ** bits - 1)
    return (code * scale + zero).reshape(x.shape)


def exact(case, seed):
    c = case
    hq, hkv, D, dt, g, _ = SHAPES[c["shape"]]
    s = prepare(c, seed)
    lens, rows = _sizes(c)
    cu = s["cu"].tolist()
    if c["kind"] == "append":
        out = {"q": s["q_out"].double(), "k": s["k_out"].double(), "v": s["v_out"].double()}
        for b, (n, r) in enumerate(zip(lens, rows)):
            x, half = s["qkv"][cu[b]:cu[b + 1]].double(), c["rotary"] // 2
            cis = torch.complex(s["cos"][n - r:n].double(), s["sin"][n - r:n].double())[:, None]
            turned, rest = x[:, :hq + hkv, :2 * half], x[:, :hq + hkv, 2 * half:]
            pairs = turned.reshape(r, hq + hkv, half, 2) if c["interleaved"] else turned.reshape(r, hq + hkv, 2, half).transpose(2, 3)
            y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * cis)
            y = y if c["interleaved"] else y.transpose(2, 3)
            y = torch.cat([y.reshape(r, hq + hkv, 2 * half), rest], -1)
            out["q"][cu[b]:cu[b + 1]] = y[:, :hq]
            out["k"][cu[b]:cu[b + 1]] = _exact_codes(y[:, hq:], c["kb"], g)
            out["v"][cu[b]:cu[b + 1]] = _exact_codes(x[:, hq + hkv:], c["vb"], g)
        return out
    if c["kind"] == "restore":
        out = {"k": s["k_out"].double(), "v": s["v_out"].double()}
        for b, n in enumerate(lens):
            ids = s["table"][b, :-(-n // PAGE)].long()
            for h in range(hkv):
                for name, side in zip("kv", _exact_pages(c, s["pages"][ids, h])):
                    out[name][cu[b]:cu[b + 1], h] = side.reshape(-1, D)[:n]
        return out
    out = s["out"].double()
    for b, (n, r) in enumerate(zip(lens, rows)):
        held = torch.tensor(_visible_pages(c, n, r), device="cuda")
        ids = s["table"][b, held].long()
        token = (held[:, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)
        keep = token < n
        for h in range(hkv):
            k, v = (x.reshape(-1, D)[keep] for x in _exact_pages(c, s["pages"][ids, h]))
            t = token[keep]
            step = max(1, 100_000_000 // (len(t) * (hq // hkv)))
            for lo in range(0, r, step):
                hi = min(r, lo + step)
                p = torch.arange(n - r + lo, n - r + hi, device="cuda")[:, None, None]
                q = s["q"][cu[b] + lo:cu[b] + hi, h * (hq // hkv):(h + 1) * (hq // hkv)].double()
                logit = torch.einsum("rgd,td->rgt", q, k) / math.sqrt(D)
                hidden = (t > p) | ((t <= p - c["window"]) & (t >= c["sinks"]) if c["window"] else t < 0)
                weight = torch.softmax(logit.masked_fill(hidden, -math.inf), -1)
                out[cu[b] + lo:cu[b] + hi, h * (hq // hkv):(h + 1) * (hq // hkv)] = torch.einsum("rgt,td->rgd", weight, v)
    return out
