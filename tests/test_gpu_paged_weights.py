"""Paged attention of many rows where 16-bit tiles and weights are at the end of their range: flat tails under peaks, values beside
much larger ones.  References: fp64 NumPy on the same packed bytes."""
import numpy as np
import pytest
import torch

import paged_testlib as pt

pytestmark = pytest.mark.gpu

S = pt.Shape


@pytest.fixture(scope="module")
def kvq():
    from paper_2502_15075_b200 import build
    build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


def refill(call, make):
    """Store rows make(sequence, tokens) -> (k, v) [tokens, Hkv, D] over all tokens of a call's sequences."""
    for b, n in enumerate(call.lens):
        where = [(int(call.table[b, t // 128]), t % 128) for t in range(n)]
        keep = [i for i, (p, _) in enumerate(where) if p >= 0]
        k, v = make(b, n)
        pt.store(call.pages, call.sh, [where[i] for i in keep], k[keep].astype(np.float32), v[keep].astype(np.float32))


@pytest.mark.parametrize("peaks", ["every page", "first token", "last tokens"])
@pytest.mark.parametrize("gap", [6.0, 13.4, 18.6, 20.6, 24.6, 28.3])
@pytest.mark.parametrize("D", [64, 128])
def test_flat_tail_under_peaks(kvq, D, gap, peaks):
    """Peaks whose values are zero over a tail `gap` bits below them: the output is the tail's share alone."""
    sh = S(D=D, kb=4, vb=4, gk=64, gv=64, G=1, Hkv=1, dtype="fp16")
    n, rows = 900, 300
    call = pt.Call(kvq, sh, [n], [rows], seed=1)
    call.q = torch.ones_like(call.q)
    t = np.arange(n)
    at = {"every page": t % 128 == 5, "first token": t == 0, "last tokens": t >= n - rows}[peaks]

    def make(_, n):
        k = np.zeros((n, 1, D)) + np.where(at, gap / (1.4426950408889634 * D ** 0.5), 0.0)[:, None, None]
        return k, np.ones((n, 1, D)) * ~at[:, None, None]
    refill(call, make)
    got, want = call.got_attention(), call.want_attention()
    # All weights of the tail are alike, so nothing averages out.  A weight is fp16 and held at least 2^11 times as large as it is relative to
    # the row's largest: off by 2^-11 of it, or by half of fp16's smallest step, 2^-25 2^-11 = 2^-36 of the largest weight, which is at most
    # the sum of all.  Values are exact; fp32 sums, exponents and logits of up to 30 bits in fp32 add less than 2^-14.
    bound = (2.0 ** -11 + 2.0 ** -14) * want + n * 2.0 ** -36
    assert np.all(np.abs(got - want) <= bound), f"off by {(np.abs(got - want) / bound).max():.2f} of what is allowed"


@pytest.mark.parametrize("side", ["keys", "values"])
@pytest.mark.parametrize("sh", [S(), S(kb=8, vb=8), S(kb=2, vb=4, gk=32, gv=64), S(D=64, kb=4, vb=8, gk=64, gv=32)], ids=str)
def test_small_values_beside_a_large_one(kvq, sh, side):
    """A token beyond half the fp16 range in a page of small ones: rows that do not see it (earlier ones, or behind the window) are served
    as exactly as without it."""
    rng = np.random.default_rng(2)
    for n, rows, window, at in ((300, 200, 0, 250), (700, 400, 100, 300)):
        call = pt.Call(kvq, sh, [n], [rows], window, 0, seed=3)
        small = 1e-3

        def make(_, n):
            k, v = (rng.standard_normal((n, sh.Hkv, sh.D)) for _ in range(2))
            x = k if side == "keys" else v
            x *= np.where(np.arange(n) == at, 4e4, small)[:, None, None]
            return k, v
        refill(call, make)
        if side == "keys":
            call.q = (call.q.float() / small).to(call.q.dtype)
        got, want = call.got_attention(), call.want_attention()
        assert np.all(np.isfinite(got))
        p = np.arange(n - rows, n)
        blind = (p < at) | ((p - window >= at) if window else False)
        # K^, V^ and the weights are off by 2^-11 of themselves; an error of K^ moves a logit of deviation one by 2^-11, a weight's ratio to
        # the others by sqrt(2) as much at most: (1 + 1 + sqrt 2) 2^-11 = 1.7e-3 where nothing averages out
        rel = np.linalg.norm(got - want, axis=-1) / np.linalg.norm(want, axis=-1)
        assert blind.sum() > 100 and rel[blind].max() <= 2e-3, f"rows that do not see the large token: {rel[blind].max():.2e}"
        if side == "keys":
            # Rows that see the large key have logits of up to 1e8 there, off by 2^-11 of the products' sum at most: which side of the others such a
            # logit lies on is only known beyond that.  (32: bits in fp32 beyond which a weight is nothing, twice the others' logits)
            K, _ = zip(*(pt.gather(call.pages, sh, call.table[0], n, h) for h in range(sh.Hkv)))
            k = np.repeat(np.stack([x[at] for x in K]), sh.G, axis=0)
            terms = call.q.double().numpy() * k / np.sqrt(sh.D)
            known = np.abs(terms.sum(-1)) > 2.0 ** -11 * np.abs(terms).sum(-1) + 32
            known[blind] = True
            assert known[~blind].mean() > 0.9 if (~blind).any() else True
            got, want = got[known], want[known]
        assert np.linalg.norm(got - want) / np.linalg.norm(want) <= 2e-3


@pytest.mark.parametrize("sh", [S(), S(kb=8, vb=8), S(kb=2, vb=2, dtype="bf16")], ids=str)
def test_the_largest_values_a_page_can_hold(kvq, sh):
    """Groups from -65504 on with the largest scale: up to 2^24, in several tokens of a page and in whole pages."""
    rng = np.random.default_rng(4)
    n, rows = 500, 150
    call = pt.Call(kvq, sh, [n], [rows], seed=5)
    t = np.arange(n)
    top = 65504.0 * 2 ** sh.vb

    def make(_, n):
        k, v = (rng.standard_normal((n, sh.Hkv, sh.D)) for _ in range(2))
        v *= np.where((t % 41 == 3) | (t // 128 == 1), top / 4, 1.0)[:, None, None]
        return k, np.clip(v, -6e4, top)
    refill(call, make)
    got, want = call.got_attention(), call.want_attention()
    assert np.all(np.isfinite(got))
    assert np.linalg.norm(got - want) / np.linalg.norm(want) <= 2e-3


@pytest.mark.parametrize("lens,rows,window,sinks", [([700, 333], [300, 90], 0, 0), ([900, 515], [400, 200], 150, 9), ([640], [640], 129, 130), ([130, 260], [60, 260], 1, 1)])
@pytest.mark.parametrize("sh", [S(), S(kb=8, vb=8, G=3), S(kb=2, vb=4, gk=32, gv=64, G=8, Hkv=1), S(D=64, kb=4, vb=8, gk=64, gv=32)], ids=str)
def test_large_keys_and_values_here_and_there(kvq, sh, lens, rows, window, sinks):
    """Tokens beyond the fp16 range on either side or both, at any place of a page, under masks and in tiles of several sequences; queries so
    small that such a key's logits are ordinary."""
    rng = np.random.default_rng(6)
    call = pt.Call(kvq, sh, lens, rows, window, sinks, seed=7)
    call.q = (call.q.float() * 2.0 ** -17).to(call.q.dtype)

    def make(_, n):
        k, v = (rng.standard_normal((n, sh.Hkv, sh.D)) for _ in range(2))
        k *= np.where(rng.random((n, sh.Hkv)) < 0.2, 2.0 ** 17, 1.0)[..., None]
        v *= np.where(rng.random((n, sh.Hkv)) < 0.1, 2.0 ** 17, 1.0)[..., None]
        return k, v
    refill(call, make)
    got, want = call.got_attention(), call.want_attention()
    assert np.all(np.isfinite(got))
    # (1 + 1 + sqrt 2) 2^-11 = 1.7e-3 as above, over a sequence's rows: single outputs may be differences of large values
    for b in range(len(lens)):
        s = slice(call.cu[b], call.cu[b + 1])
        assert np.linalg.norm(got[s] - want[s]) / np.linalg.norm(want[s]) <= 2e-3
    assert np.array_equal(got, call.got_attention())
