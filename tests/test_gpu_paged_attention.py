"""kvq_paged_attention against fp64 NumPy on the same packed bytes: window, first tokens, ragged rows, layouts, refusals."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paged_testlib as pt

pytestmark = pytest.mark.gpu

S = pt.Shape
REL, MABS = 2e-3, 1e-2            # the library's tolerance of attention in fp32 (see kvq_testlib)


@pytest.fixture(scope="module")
def kvq():
    from paper_2502_15075_b200 import build
    build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


def close(got, want, out_dtype=torch.float32):
    assert np.all(np.isfinite(got))
    half = torch.finfo(out_dtype).eps / 2
    rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
    assert rel <= REL + half, f"rel-L2 {rel:.3e}"
    over = np.abs(got - want) - (MABS + half * np.abs(want))
    assert over.max() <= 0, f"max-abs {np.abs(got - want).max():.3e}"


SHAPES = [S(), S(kb=2, vb=4, Hkv=1), S(kb=4, vb=4, dtype="fp16"), S(kb=8, vb=4), S(gk=32, gv=128), S(gk=64, gv=64), S(G=8, Hkv=1), S(kb=8, vb=8, gk=32, gv=32, dtype="fp16"),
          S(D=64, gk=64, gv=64, dtype="fp16"), S(D=64, gk=32, gv=32, G=1, Hkv=3, dtype="fp16"), S(kb=2, vb=2, G=1), S(D=64, kb=8, vb=2, gk=64, gv=32, G=6, Hkv=1)]
DECODE = [  # lens, window, sinks
    ([1, 2, 127, 128, 129], 0, 0), ([700, 1, 383], 0, 0), ([1000, 640], 1, 0), ([1000, 129, 17], 100, 4), ([900, 513], 128, 128), ([1100], 130, 200),
    ([777, 300], 2**31 - 1, 2**31 - 1), ([512, 385], 129, 1), ([600], 5, 1000), ([640, 640], 256, 33)]


@pytest.mark.parametrize("lens,window,sinks", DECODE)
@pytest.mark.parametrize("sh", SHAPES, ids=str)
def test_one_row_a_sequence(kvq, sh, lens, window, sinks):
    call = pt.Call(kvq, sh, lens, [1] * len(lens), window, sinks, seed=1, keys=2.0)
    close(call.got_attention(), call.want_attention())


ROWS = [  # lens, rows, window, sinks, pad
    ([300, 140], [2, 2], 0, 0, 0), ([300, 5, 0, 131], [2, 1, 0, 2], 60, 3, 2), ([130, 400], [130, 7], 0, 0, 1), ([700, 650], [70, 333], 100, 4, 0),
    ([64], [64], 10, 0, 0), ([260, 129, 257], [3, 129, 1], 1, 1, 0), ([1200], [520], 256, 130, 0), ([1, 128], [1, 128], 0, 0, 5)]


@pytest.mark.parametrize("lens,rows,window,sinks,pad", ROWS)
@pytest.mark.parametrize("sh", SHAPES, ids=str)
def test_several_rows_a_sequence(kvq, sh, lens, rows, window, sinks, pad):
    call = pt.Call(kvq, sh, lens, rows, window, sinks, pad, seed=2, keys=2.0)
    close(call.got_attention(), call.want_attention())


@pytest.mark.parametrize("out_dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 40])
def test_output_types_and_scale(kvq, out_dtype, rows):
    call = pt.Call(kvq, S(dtype="fp16"), [333, 200], [rows, rows], 150, 2, pad=1, seed=3)
    close(call.got_attention(out_dtype, scale=0.31), call.want_attention(scale=0.31), out_dtype)


@pytest.mark.parametrize("rows", [1, 2, 33])
def test_max_rows_may_be_larger_than_any_sequence_needs(kvq, rows):
    call = pt.Call(kvq, S(G=2), [333, 200, 64], [rows, max(0, rows - 1), 1], 0, 0, seed=4)
    for max_rows in (rows, rows + 1, 4 * rows, 500):
        close(call.got_attention(max_rows=max_rows), call.want_attention())


@pytest.mark.parametrize("rows", [1, 24])
def test_sequences_without_rows_and_padding_are_left_alone(kvq, rows):
    call = pt.Call(kvq, S(), [400, 300, 0, 200], [0, rows, 0, 1], 64, 1, pad=9, seed=5)
    got, want = call.got_attention(out_fill=0.25), call.want_attention(0.25)
    close(got, want)
    assert np.all(got[int(call.cu[-1]):] == 0.25)


@pytest.mark.parametrize("rows", [1, 2, 16])
def test_many_sequences(kvq, rows):
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(rows, 300, 70)]
    call = pt.Call(kvq, S(D=64, gk=64, gv=64, Hkv=1, G=4, dtype="fp16"), lens, [min(rows, n) for n in lens], 70, 4, seed=6)
    close(call.got_attention(), call.want_attention())


@pytest.mark.parametrize("rows", [1, 20])
def test_long_sequences_are_split_and_merged(kvq, rows):
    call = pt.Call(kvq, S(Hkv=1), [6000, 3000], [rows, 1], 0, 0, seed=7)
    close(call.got_attention(), call.want_attention())
    call = pt.Call(kvq, S(Hkv=1), [6000, 5000], [rows, rows], 4000, 200, seed=8)
    close(call.got_attention(), call.want_attention())


@pytest.mark.parametrize("rows", [1, 20])
@pytest.mark.parametrize("size", [1e-4, 60.0])
def test_small_and_large_values(kvq, rows, size):
    """Peaked and flat softmax, values far from one."""
    call = pt.Call(kvq, S(), [500, 260], [rows, rows], 0, 0, seed=9, keys=size)
    got, want = call.got_attention(), call.want_attention()
    # An element of K^ in a 16-bit tile is off by at most 2^-11 of it, 2^-11 / sqrt(3) in the mean square, so a logit of standard deviation
    # `size` by 60 * 2.8e-4 = 0.017 (16-bit fixed point of q: less); the difference of two logits by sqrt(2) as much, three standard
    # deviations 0.07, which is what a weight and so the output can be off by, relatively.
    rel = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert np.all(np.isfinite(got)) and rel <= (REL if size < 1 else 0.07)


@pytest.mark.parametrize("rows", [1, 30])
def test_values_beyond_the_fp16_range(kvq, rows):
    """A bf16 cache whose groups reach further than fp16 does: scale and zero-point are fp16, their reconstruction is not."""
    sh = S()
    call = pt.Call(kvq, sh, [300, 200], [rows, 1], 0, 0, seed=10)
    rng = np.random.default_rng(10)
    for b, n in enumerate(call.lens):
        where = [(int(call.table[b, t // 128]), t % 128) for t in range(n)]
        big = np.where(np.arange(n) % 50 == 7, 40.0, 1.0)[:, None, None]
        k = rng.standard_normal((n, sh.Hkv, sh.D)).astype(np.float32)
        v = (rng.standard_normal((n, sh.Hkv, sh.D)) * big * 1e3).astype(np.float32) + np.where(big > 1, 6e4, 0).astype(np.float32)
        pt.store(call.pages, sh, where, k, v.astype(np.float32))
    got, want = call.got_attention(), call.want_attention()
    assert np.all(np.isfinite(got))
    assert np.linalg.norm(got - want) / np.linalg.norm(want) <= REL


@pytest.mark.parametrize("rows", [1, 30])
def test_bad_device_inputs_set_the_status(kvq, rows):
    call = pt.Call(kvq, S(), [400, 300], [rows, 1], 0, 0, seed=11, capacity=512)
    want = call.want_attention()

    def attempt(change):
        cache, cu = call.on_gpu()
        change(cache, cu)
        ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, rows), dtype=torch.uint8, device="cuda")
        out = torch.full(call.q.shape, 0.5, dtype=torch.float32, device="cuda")
        kvq.kvq_paged_attention(call.cfg, cache, call.q.cuda(), cu, out, ws, rows)
        assert int(cache.status) == kvq.STATUS_BAD_INPUT and kvq.kvq_check_status(cache) == -9
        return out.double().cpu().numpy(), cache, ws

    def first(seq, value):
        return lambda c, cu: c.seq_len.__setitem__(seq, value)
    for value in (513, rows - 1 if rows > 1 else 0, -1, 2**31 - 1):
        got, _, _ = attempt(first(0, value))
        assert np.all(got[:rows] == 0.5)                  # passed over
        close(got[rows:], want[rows:])                    # the other sequence is served
    got, _, _ = attempt(lambda c, cu: cu.copy_(torch.tensor([0, 2**31 - 1, rows + 1], dtype=torch.int32)))
    assert np.all(got == 0.5)
    # a page outside the pool: that sequence is undefined, the other one served, and the next call on the same workspace too
    for bad in (-1, 10**9):
        got, cache, ws = attempt(lambda c, cu: c.block_table.__setitem__((0, 1), bad))
        close(got[rows:], want[rows:])
    cache, cu = call.on_gpu()
    close(call.got_attention(cache=cache, cu=cu, workspace=ws), want)


def test_more_rows_than_announced_are_passed_over(kvq):
    for G, rows, announced in ((4, 3, 2), (4, 40, 39), (1, 2, 1)):
        call = pt.Call(kvq, S(G=G), [400, 300], [rows, 1], 0, 0, seed=12)
        cache, cu = call.on_gpu()
        ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, announced), dtype=torch.uint8, device="cuda")
        out = torch.full(call.q.shape, 0.5, dtype=torch.float32, device="cuda")
        kvq.kvq_paged_attention(call.cfg, cache, call.q.cuda(), cu, out, ws, announced)
        assert int(cache.status) == kvq.STATUS_BAD_INPUT
        got = out.double().cpu().numpy()
        assert np.all(got[:rows] == 0.5)
        close(got[rows:], call.want_attention()[rows:])


@pytest.mark.parametrize("rows", [1, 2, 50])
def test_captured_call_is_replayed_for_other_lengths(kvq, rows):
    """One graph over a padded batch; lengths, offsets and the table change between replays, the workspace is shared with a second
    graph, and results equal the eager call's bit for bit."""
    sh = S(Hkv=2)
    calls = [pt.Call(kvq, sh, lens, r, 200, 5, pad=2 * rows - sum(r), seed=20 + i, capacity=1024)
             for i, (lens, r) in enumerate((([900, 300], [rows, rows]), ([1024, 64], [rows, 0]), ([rows, 777], [rows, 1])))]
    pool = max(c.pages.shape[0] for c in calls)
    cache = kvq.PagedCache(calls[0].cfg, n_pages=pool)
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    q = torch.zeros_like(calls[0].q, device="cuda")
    ws = torch.empty(kvq.kvq_paged_workspace_bytes(calls[0].cfg, rows), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros(q.shape, device="cuda") for _ in range(2)]

    def load(c):
        cache.pages.fill_(255)
        cache.pages[:c.pages.shape[0]] = torch.from_numpy(c.pages).cuda()
        cache.block_table.copy_(torch.from_numpy(c.table))
        cache.seq_len.copy_(torch.tensor(c.lens, dtype=torch.int32))
        cu.copy_(torch.from_numpy(c.cu))
        q.copy_(c.q)
    load(calls[0])
    graphs = []
    for out in outs:
        kvq.kvq_paged_attention(calls[0].cfg, cache, q, cu, out, ws, rows, 200, 5)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kvq.kvq_paged_attention(calls[0].cfg, cache, q, cu, out, ws, rows, 200, 5)
        graphs.append(g)
    for c in calls + calls[::-1]:
        load(c)
        for out in outs:
            out.fill_(0.5)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert kvq.kvq_check_status(cache) == 0
        assert torch.equal(outs[0], outs[1])
        got = outs[0].double().cpu().numpy()
        close(got, c.want_attention())
        assert np.array_equal(got, c.got_attention(max_rows=rows))


@pytest.mark.parametrize("rows", [1, 60])
def test_on_another_stream_and_repeated(kvq, rows):
    call = pt.Call(kvq, S(), [2000, 1500], [rows, rows], 900, 4, seed=13)
    cache, cu = call.on_gpu()
    q = call.q.cuda()
    ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, rows), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros(q.shape, device="cuda") for _ in range(5)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for out in outs:
        kvq.kvq_paged_attention(call.cfg, cache, q, cu, out, ws, rows, 900, 4, stream=s)
    s.synchronize()
    close(outs[0].double().cpu().numpy(), call.want_attention())
    assert all(torch.equal(outs[0], o) for o in outs[1:])      # the order in which partials arrive changes nothing


def test_prompt_chunks_and_decoding_in_turn(kvq):
    """As used: a prompt taken in by chunks (append with rotation, attention of the chunk), then single tokens, with a window; each
    call's output against fp64 on the bytes that the pool then holds."""
    sh = S(Hkv=2, G=4)
    hq, window, sinks = sh.G * sh.Hkv, 150, 4
    call = pt.Call(kvq, sh, [420, 390], [420, 390], seed=14, fill=False)
    cache, cu = call.on_gpu()
    cos, sin = pt.tables(sh.D, 512)
    rope = kvq.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    gen = torch.Generator(device="cuda").manual_seed(3)
    lens = [0, 0]
    for step in ([200, 3], [170, 300], [1, 1], [1, 0], [0, 2], [1, 1]):
        lens = [a + b for a, b in zip(lens, step)]
        n = sum(step)
        cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        cu.copy_(torch.tensor([0, step[0], n], dtype=torch.int32))
        qkv = torch.randn(n, hq + 2 * sh.Hkv, sh.D, generator=gen, device="cuda").to(sh.torch_dtype)
        q = torch.empty(n, hq, sh.D, dtype=sh.torch_dtype, device="cuda")
        kvq.kvq_paged_append(call.cfg, cache, qkv[:, hq:hq + sh.Hkv], qkv[:, hq + sh.Hkv:], cu, rope, qkv[:, :hq], q)
        out = torch.zeros(q.shape, device="cuda")
        ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, max(step)), dtype=torch.uint8, device="cuda")
        kvq.kvq_paged_attention(call.cfg, cache, q, cu, out, ws, max(step), window, sinks)
        assert kvq.kvq_check_status(cache) == 0
        want = pt.attention(cache.pages.cpu().numpy(), sh, call.table, lens, cu.cpu().numpy(), q.double().cpu().numpy(), window, sinks, np.zeros(q.shape))
        close(out.double().cpu().numpy(), want)


@pytest.mark.parametrize("rows,skip", [(1, 0), (1, 3), (1, 9), (40, 0), (300, 0), (600, 2)])
def test_a_page_that_never_arrives_ends_the_call(kvq, rows, skip):
    """The bounded waits run out, the call ends with a status, and the next call on the same workspace is right."""
    call = pt.Call(kvq, S(), [2600 if skip == 2 else 700, 500], [rows, 1], 0, 0, seed=15)
    cache, cu = call.on_gpu()
    q = call.q.cuda()
    ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, rows), dtype=torch.uint8, device="cuda")
    out = torch.zeros(q.shape, device="cuda")
    kvq.kvq_debug_paged_stall(call.cfg, cache, q, cu, out, ws, rows, skip, 2000)
    assert kvq.kvq_check_status(cache) == -7
    cache.status.zero_()
    close(call.got_attention(cache=cache, cu=cu, workspace=ws), call.want_attention())


def test_pools_beyond_four_gigabytes(kvq):
    """Pages whose offsets do not fit 32 bits, in all three operators (the rest of the pool is never touched)."""
    sh = S()
    for rows in (1, 50):
        call = pt.Call(kvq, sh, [300, 200], [rows, 1], 100, 3, seed=16)
        want, n, far = call.want_attention(), call.pages.shape[0], 200_000
        pages = torch.empty((far + n,) + call.pages.shape[1:], dtype=torch.uint8, device="cuda")
        assert pages.numel() > 2 ** 32
        pages[far:] = torch.from_numpy(call.pages).cuda()
        table = torch.where(torch.from_numpy(call.table) >= 0, torch.from_numpy(call.table) + far, -1).cuda()
        cache = kvq.PagedCache(call.cfg, pages=pages, block_table=table, seq_len=torch.tensor(call.lens, dtype=torch.int32, device="cuda"))
        cu = torch.from_numpy(call.cu).cuda()
        close(call.got_attention(cache=cache, cu=cu), want)
        near, _ = call.on_gpu()
        outs = []
        for c in (cache, near):
            kvq.kvq_paged_append(call.cfg, c, call.k.cuda(), call.v.cuda(), cu)
            kv = [torch.zeros(call.n, sh.Hkv, sh.D, dtype=sh.torch_dtype, device="cuda") for _ in range(2)]
            kvq.kvq_paged_dequantize(call.cfg, c, cu, *kv)
            assert kvq.kvq_check_status(c) == 0
            outs.append(kv)
        assert torch.equal(pages[far:], near.pages) and all(torch.equal(a, b) for a, b in zip(*outs))
        del pages, cache


@pytest.mark.parametrize("G", [3, 5, 7])
@pytest.mark.parametrize("rows", [1, 100])
def test_groups_of_heads_that_are_no_power_of_two(kvq, G, rows):
    call = pt.Call(kvq, S(G=G, Hkv=2), [400, 130], [rows, 7], 90, 3, seed=17)
    close(call.got_attention(), call.want_attention())


def test_table_with_wide_rows_and_more_sequences_than_fit_a_warp(kvq):
    """A block table whose rows lie apart, 200 sequences, and a decoding step next to a chunk in one call."""
    lens = [40 + 3 * i for i in range(200)]
    for rows in ([1] * 200, [1] * 199 + [60]):
        call = pt.Call(kvq, S(D=64, gk=64, gv=64, Hkv=1, G=2, dtype="fp16"), lens, rows, 0, 0, seed=18)
        cache, cu = call.on_gpu()
        wide = torch.full((200, 37), -7, dtype=torch.int32, device="cuda")
        wide[:, :call.table.shape[1]] = torch.from_numpy(call.table).cuda()
        cache = kvq.PagedCache(call.cfg, pages=cache.pages, block_table=wide, seq_len=cache.seq_len)
        close(call.got_attention(cache=cache, cu=cu), call.want_attention())


@pytest.mark.parametrize("pairs", [((1, 60), (2, 1)), ((300, 4), (1, 1)), ((40, 40), (3, 300))])
def test_two_streams_with_workspaces_of_their_own(kvq, pairs):
    """Calls of both kernels at once on one pool, each stream with its own workspace: as alone."""
    call = [[pt.Call(kvq, S(), [1900, 700], [r, 1], 0, 0, seed=30 + r) for r in rows] for rows in pairs]
    streams = [torch.cuda.Stream() for _ in pairs]
    jobs = []
    for i in range(2):
        for c in call[i]:
            cache, cu = c.on_gpu()
            ws = torch.empty(kvq.kvq_paged_workspace_bytes(c.cfg, max(c.rows)), dtype=torch.uint8, device="cuda")
            jobs.append((streams[i], c, cache, cu, c.q.cuda(), ws, [torch.zeros(c.q.shape, device="cuda") for _ in range(4)]))
    torch.cuda.synchronize()
    for k in range(4):
        for s, c, cache, cu, q, ws, outs in jobs:
            kvq.kvq_paged_attention(c.cfg, cache, q, cu, outs[k], ws, max(c.rows), stream=s)
    torch.cuda.synchronize()
    for s, c, cache, cu, q, ws, outs in jobs:
        assert kvq.kvq_check_status(cache) == 0
        want = c.got_attention(out_fill=0.0)
        for out in outs:
            assert np.array_equal(out.double().cpu().numpy(), want)


def test_one_workspace_for_calls_of_every_kind(kvq):
    """Decoding, chunks of several lengths and other windows in turn on one stream and one workspace, as a server that mixes them."""
    shared = None
    calls = [pt.Call(kvq, S(), [1500, 900], r, w, s, seed=40 + i)
             for i, (r, w, s) in enumerate((([1, 1], 0, 0), ([300, 7], 0, 0), ([2, 1], 200, 4), ([600, 600], 333, 1), ([1, 0], 0, 0)))]
    need = max(kvq.kvq_paged_workspace_bytes(c.cfg, max(c.rows)) for c in calls)
    shared = torch.full((need,), 171, dtype=torch.uint8, device="cuda")
    alone = [c.got_attention() for c in calls]
    for i in (0, 1, 2, 3, 4, 1, 0, 3, 2, 2, 1, 1, 4):
        assert np.array_equal(calls[i].got_attention(workspace=shared), alone[i])


def test_first_calls_of_a_process_may_be_captured(tmp_path):
    """No warm-up outside the capture: append, both attention kernels and the read-back recorded first of all, then replayed."""
    here = os.path.dirname(os.path.abspath(__file__))
    code = """
import sys; sys.path[:0] = [%r, %r]
import numpy as np, torch, paged_testlib as pt
from paper_2502_15075_b200 import kvq
calls = [pt.Call(kvq, pt.Shape(), [700, 200], [r, 1], seed=r) for r in (1, 40)]
jobs = []
for c in calls:
    cache, cu = c.on_gpu()
    ws = torch.empty(kvq.kvq_paged_workspace_bytes(c.cfg, max(c.rows)), dtype=torch.uint8, device="cuda")
    q = c.q.cuda(); kv = [x.cuda() for x in (c.k, c.v)]
    jobs.append((c, cache, cu, ws, q, torch.full(q.shape, 0.5, device="cuda"), kv, [torch.zeros_like(x) for x in kv]))
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    for c, cache, cu, ws, q, out, kv, back in jobs:
        kvq.kvq_paged_attention(c.cfg, cache, q, cu, out, ws, max(c.rows))
        kvq.kvq_paged_append(c.cfg, cache, kv[0], kv[1], cu)
        kvq.kvq_paged_dequantize(c.cfg, cache, cu, back[0], back[1])
g.replay()
torch.cuda.synchronize()
for c, cache, cu, ws, q, out, kv, back in jobs:
    assert kvq.kvq_check_status(cache) == 0
    assert np.array_equal(out.double().cpu().numpy(), c.got_attention())
    again = [torch.zeros_like(x) for x in back]
    kvq.kvq_paged_dequantize(c.cfg, cache, cu, again[0], again[1])
    assert torch.equal(back[0], again[0]) and torch.equal(back[1], again[1]) and bool(back[0].any())
""" % (os.path.dirname(here), here)
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-3000:]


@pytest.mark.parametrize("sh,rows,capacity", [
    (S(Hkv=8), [4, 1, 0, 3], 8192), (S(Hkv=8), [3, 3, 2, 1], 8192), (S(Hkv=8), [6, 5, 1, 2], 16384), (S(Hkv=8), [8, 3, 7, 0], 32768),
    (S(Hkv=8), [9, 10, 1, 0], 196608), (S(Hkv=8, G=8), [2, 1, 2, 0], 8192), (S(Hkv=4, G=3), [4, 3, 1, 1], 16384), (S(Hkv=8, G=1), [13, 9, 8, 1], 8192),
    (S(Hkv=8, gk=32, gv=128), [2, 1, 0, 2], 8192), (S(D=64, gk=64, gv=64, dtype="fp16", Hkv=8, G=2), [7, 5, 4, 1], 8192)], ids=str)
@pytest.mark.parametrize("window,sinks", [(0, 0), (7000, 5), (130, 4)])
def test_few_rows_over_large_capacities(kvq, sh, rows, capacity, window, sinks):
    """More pairs than one launch of the decode kernel takes, on capacities and windows where several serve the call and where they do
    not; a sequence's rows lie in all launches, in the first ones, in none."""
    call = pt.Call(kvq, sh, [500, 257, 130, 16], rows, window, sinks, pad=2, seed=50 + max(rows), capacity=capacity, keys=2.0)
    got = call.got_attention()
    close(got, call.want_attention())
    assert np.array_equal(got, call.got_attention())


def test_more_rows_than_announced_are_passed_over_by_every_launch(kvq):
    call = pt.Call(kvq, S(Hkv=8), [400, 300, 200], [5, 4, 1], 0, 0, seed=61, capacity=16384)
    cache, cu = call.on_gpu()
    ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, 4), dtype=torch.uint8, device="cuda")
    out = torch.full(call.q.shape, 0.5, dtype=torch.float32, device="cuda")
    kvq.kvq_paged_attention(call.cfg, cache, call.q.cuda(), cu, out, ws, 4)
    assert int(cache.status) == kvq.STATUS_BAD_INPUT
    got = out.double().cpu().numpy()
    assert np.all(got[:5] == 0.5)
    close(got[5:], call.want_attention()[5:])


@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("sh", [S(Hkv=1), S(Hkv=1, D=64, gk=64, gv=64)], ids=str)
def test_largest_batch(kvq, sh, rows):
    rng = np.random.default_rng(70)
    lens = [int(x) for x in rng.integers(0, 20, 1024)]
    call = pt.Call(kvq, sh, lens, [min(n, rows) for n in lens], 9, 1, pad=3, seed=71)
    close(call.got_attention(), call.want_attention())
