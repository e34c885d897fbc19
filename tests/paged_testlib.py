"""The paged cache's operators in NumPy (packing by the oracle's layout functions, attention in fp64) and a builder of ragged calls."""
from __future__ import annotations

import dataclasses
import math

import numpy as np
import torch

from oracle import layout as ol
from oracle import quantizer as oq

PAGE = 128


@dataclasses.dataclass(frozen=True)
class Shape:
    D: int = 128
    G: int = 4
    Hkv: int = 2
    kb: int = 4
    vb: int = 2
    gk: int = 128
    gv: int = 128
    dtype: str = "bf16"

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float16

    @property
    def layout(self):
        return ol.Layout(self.D, self.kb, self.vb, self.gk, self.gv, 0)


def bits_of(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def config(kvq, sh: Shape, batch, capacity):
    return kvq.make_config(batch, sh.G * sh.Hkv, sh.Hkv, sh.D, sh.kb, sh.vb, sh.gk, sh.gv, 0, sh.torch_dtype, capacity)


def tables(rotary, positions, base=10000.0):
    half = rotary // 2
    angle = np.arange(positions, dtype=np.float64)[:, None] * base ** (-np.arange(half) / half)
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def rotate(x, cos, sin, interleaved):
    """x float32 [rows, heads, D]; cos, sin float32 [rows, rotary / 2]: every product and sum rounded on its own."""
    half = cos.shape[1]
    y = x.copy()
    c, s = cos[:, None], sin[:, None]
    ia, ib = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def store(pages: np.ndarray, sh: Shape, page_of, k32, v32):
    """Quantize fp32 rows [n, Hkv, D] and put row i into token page_of[i] = (pool page, token of the page); in place."""
    L = sh.layout
    sides = []
    for x, bits, g in ((k32, sh.kb, sh.gk), (v32, sh.vb, sh.gv)):
        codes, s16, z16 = oq.quantize_groups(x.reshape(x.shape[:-1] + (sh.D // g, g)), bits)
        sides.append((codes.reshape(x.shape), s16, z16))
    by_page = {}
    for i, (p, t) in enumerate(page_of):
        by_page.setdefault(p, []).append((i, t))
    for p, where in by_page.items():
        rows, toks = [i for i, _ in where], [t for _, t in where]
        for h in range(sh.Hkv):
            pg = pages[p, h]
            (kc, ks, kz), (vc, vs, vz) = sides
            ol.put_k_codes(pg, L, toks, kc[rows, h])
            ol.put_k_meta_tokens(pg, L, toks, ks[rows, h], kz[rows, h])
            ol.put_v_codes(pg, L, toks, vc[rows, h])
            ol.put_v_meta_tokens(pg, L, toks, vs[rows, h], vz[rows, h])


def page_values(page: np.ndarray, sh: Shape):
    """(K^, V^) in fp64 [128, D] of one packed page, zeros where the metadata is not finite (tokens never written)."""
    L = sh.layout
    out = []
    for codes, (s, z), g in ((ol.get_k_codes(page, L), ol.get_k_meta(page, L), sh.gk), (ol.get_v_codes(page, L), ol.get_v_meta(page, L), sh.gv)):
        c = codes.reshape(PAGE, sh.D // g, g)
        with np.errstate(invalid="ignore"):
            x = oq.dequantize_groups_f64(c, s, z).reshape(PAGE, sh.D)
        out.append(np.where(np.isfinite(x), x, 0.0))
    return out


def gather(pages: np.ndarray, sh: Shape, table_row, n, h, needed=None):
    """K^, V^ in fp64 [n, D] of a sequence's KV head; only the tokens of `needed` (a mask) matter, other pages are not looked at."""
    K, V = np.zeros((n, sh.D)), np.zeros((n, sh.D))
    for i in range(-(-n // PAGE)):
        lo, hi = i * PAGE, min(n, i * PAGE + PAGE)
        if needed is not None and not needed[lo:hi].any():
            continue
        k, v = page_values(pages[int(table_row[i]), h], sh)
        K[lo:hi], V[lo:hi] = k[:hi - lo], v[:hi - lo]
    return K, V


def mask(n, rows, window, sinks):
    """[rows, n]: which tokens the last `rows` of n tokens see."""
    p = np.arange(n - rows, n)[:, None]
    t = np.arange(n)[None]
    sees = t <= p
    if window:
        sees &= (t > p - window) | (t < sinks)
    return sees


def attention(pages, sh: Shape, table, seq_len, cu, q64, window, sinks, out, scale=None):
    """q64 [rows, Hq, D] fp64; writes into a copy of out (fp64) and returns it."""
    out = out.copy()
    scale = scale if scale and scale > 0 else 1.0 / math.sqrt(sh.D)
    for b in range(len(seq_len)):
        n, r = int(seq_len[b]), int(cu[b + 1] - cu[b])
        if r == 0:
            continue
        sees = mask(n, r, window, sinks)
        for h in range(sh.Hkv):
            K, V = gather(pages, sh, table[b], n, h, sees.any(0))
            for j in range(sh.G):
                x = np.where(sees, scale * (q64[cu[b]:cu[b + 1], h * sh.G + j] @ K.T), -np.inf)
                w = np.exp(x - x.max(-1, keepdims=True))
                out[cu[b]:cu[b + 1], h * sh.G + j] = (w / w.sum(-1, keepdims=True)) @ V
    return out


class Call:
    """A ragged call on a pool whose pages lie in a random order: lens tokens per sequence (rows counted in), rows of the call.
    The tokens in front of the call's are in the pool already; tokens never written and pages out of reach are bytes of 255, and the
    table entries of pages that no row sees are -1."""

    def __init__(self, kvq, sh: Shape, lens, rows, window=0, sinks=0, pad=0, seed=0, capacity=None, fill=True, keys=1.0):
        rng = np.random.default_rng(seed)
        self.kvq, self.sh, self.window, self.sinks = kvq, sh, window, sinks
        self.lens, self.rows = list(lens), list(rows)
        B = len(lens)
        capacity = capacity or max(PAGE, -(-max(max(lens), 1) // PAGE) * PAGE)
        self.cfg = config(kvq, sh, B, capacity)
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n = int(self.cu[-1]) + pad
        held = []
        for b in range(B):
            sees = mask(lens[b], rows[b], window, sinks).any(0) if fill and rows[b] else np.ones(lens[b], bool)
            held.append([i for i in range(-(-lens[b] // PAGE)) if sees[i * PAGE:(i + 1) * PAGE].any()])
        count = sum(map(len, held))
        ids = rng.permutation(count + 3)
        self.table = np.full((B, capacity // PAGE), -1, np.int32)
        at = 0
        for b in range(B):
            for i in held[b]:
                self.table[b, i] = ids[at]
                at += 1
        self.pages = np.full((count + 3, sh.Hkv, sh.layout.page_bytes), 255, np.uint8)

        def draw(n, scale=1.0):
            x = torch.from_numpy(rng.standard_normal((n, sh.Hkv, sh.D)).astype(np.float32) * np.float32(scale))
            return x.to(sh.torch_dtype)
        self.k, self.v = draw(self.n, keys), draw(self.n)
        self.q = torch.from_numpy(rng.standard_normal((self.n, sh.G * sh.Hkv, sh.D)).astype(np.float32)).to(sh.torch_dtype)
        for b in range(B):
            old = lens[b] if fill else lens[b] - rows[b]
            k, v = draw(old, keys).float().numpy(), draw(old).float().numpy()
            where = [(int(self.table[b, t // PAGE]), t % PAGE) for t in range(old)]
            keep = [i for i, (p, _) in enumerate(where) if p >= 0]
            store(self.pages, sh, [where[i] for i in keep], k[keep], v[keep])

    def on_gpu(self, device="cuda"):
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
        cache = self.kvq.PagedCache(self.cfg, pages=d(self.pages), block_table=d(self.table),
                                    seq_len=d(np.asarray(self.lens, np.int32)))
        return cache, d(self.cu)

    def positions(self):
        return np.concatenate([np.arange(n - r, n) for n, r in zip(self.lens, self.rows)]).astype(np.int64)

    def places(self):
        return [(int(self.table[b, t // PAGE]), t % PAGE) for b, (n, r) in enumerate(zip(self.lens, self.rows)) for t in range(n - r, n)]

    def want_attention(self, out_fill=0.5, scale=None):
        q = self.q.double().numpy()
        return attention(self.pages, self.sh, self.table, self.lens, self.cu, q, self.window, self.sinks, np.full(q.shape, out_fill), scale)

    def got_attention(self, out_dtype=torch.float32, max_rows=None, out_fill=0.5, scale=0.0, cache=None, cu=None, workspace=None):
        kvq = self.kvq
        if cache is None:
            cache, cu = self.on_gpu()
        max_rows = max_rows or max(1, max(self.rows))
        if workspace is None:
            workspace = torch.full((kvq.kvq_paged_workspace_bytes(self.cfg, max_rows),), 171, dtype=torch.uint8, device=cu.device)
        out = torch.full(self.q.shape, out_fill, dtype=out_dtype, device=cu.device)
        kvq.kvq_paged_attention(self.cfg, cache, self.q.to(cu.device), cu, out, workspace, max_rows, self.window, self.sinks, scale)
        assert kvq.kvq_check_status(cache) == 0
        return out.double().cpu().numpy()
