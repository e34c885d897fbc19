"""kvq_paged_append and kvq_paged_dequantize: every byte of the pool, the rotated queries and the values read back, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import quantizer as oq

import paged_testlib as pt

pytestmark = pytest.mark.gpu

S = pt.Shape
SHAPES = [S(), S(kb=2, vb=4), S(kb=4, vb=4, Hkv=1), S(kb=8, vb=4, dtype="fp16"), S(gk=32, gv=32, Hkv=3, G=1), S(gk=64, gv=128, kb=2, vb=8, dtype="fp16"),
          S(D=64, gk=64, gv=64, dtype="fp16"), S(D=64, gk=32, gv=32, G=1, Hkv=8), S(D=64, gk=64, gv=32, kb=8, vb=2, G=8, Hkv=1), S(G=8), S(kb=8, vb=8, gk=32, gv=64)]
# (lengths with the call's tokens counted in, tokens of the call)
CALLS = [([1], [1]), ([128, 129, 1], [1, 1, 1]), ([300, 5, 0, 131], [17, 5, 0, 4]), ([640, 200], [511, 73]), ([77, 256, 33], [0, 256, 32])]


@pytest.fixture(scope="module")
def kvq():
    from paper_2502_15075_b200 import build
    build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


def run_append(call, rotary, interleaved, seed=0, in_place=False, device="cuda", positions=None):
    """One append through the library and in NumPy; compares the pool, q and what is read back."""
    kvq, sh = call.kvq, call.sh
    cache, cu = call.on_gpu(device)
    n, real = call.n, int(call.cu[-1])
    pos = call.positions()
    want_pages = call.pages.copy()
    k32, v32, q32 = (x[:real].float().numpy() for x in (call.k, call.v, call.q))
    rope = None
    if rotary:
        cos, sin = pt.tables(rotary, positions or max(max(call.lens), 1))
        k32, q32 = (pt.rotate(x, cos[pos], sin[pos], interleaved) for x in (k32, q32))
        rope = kvq.Rope(torch.from_numpy(cos).to(device), torch.from_numpy(sin).to(device), interleaved)
    if real:
        pt.store(want_pages, sh, call.places(), k32, v32)
    # q, k and v of a token side by side, as a projection leaves them
    qkv = torch.cat([call.q, call.k, call.v], 1).to(device)
    hq = sh.G * sh.Hkv
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + sh.Hkv], qkv[:, hq + sh.Hkv:]
    q_out = torch.full((n, hq, sh.D), 7.0, dtype=sh.torch_dtype, device=device)
    if in_place:
        q = q_out.copy_(call.q)
    kvq.kvq_paged_append(call.cfg, cache, k, v, cu, rope, q if rotary else None, q_out if rotary else None)
    assert kvq.kvq_check_status(cache) == 0
    got = cache.pages.cpu().numpy()
    bad = np.argwhere(got != want_pages)
    assert len(bad) == 0, f"{len(bad)} bytes differ, first (page, head, byte) {bad[0].tolist()}"
    if rotary:
        want_q = pt.bits_of(call.q if in_place else torch.full((n, hq, sh.D), 7.0, dtype=sh.torch_dtype)).copy()
        want_q[:real] = oq.f32_to_bits(q32, sh.dtype)
        assert np.array_equal(pt.bits_of(q_out), want_q), "rotated queries differ"
    # the stored tokens in 16 bits
    outs = [torch.full((n, sh.Hkv, sh.D), 7.0, dtype=sh.torch_dtype, device=device) for _ in range(2)]
    kvq.kvq_paged_dequantize(call.cfg, cache, cu, outs[0], outs[1])
    assert kvq.kvq_check_status(cache) == 0
    for out, x, bits, g in ((outs[0], k32, sh.kb, sh.gk), (outs[1], v32, sh.vb, sh.gv)):
        want = pt.bits_of(torch.full((n, sh.Hkv, sh.D), 7.0, dtype=sh.torch_dtype)).copy()
        if real:
            codes, s16, z16 = oq.quantize_groups(x.reshape(real, sh.Hkv, sh.D // g, g), bits)
            want[:real] = oq.f32_to_bits(oq.dequantize_groups(codes, s16, z16).reshape(real, sh.Hkv, sh.D), sh.dtype)
        assert np.array_equal(pt.bits_of(out), want), "values read back differ"
    return cache


@pytest.mark.parametrize("lens,rows", CALLS)
@pytest.mark.parametrize("sh", SHAPES, ids=str)
def test_append_rotated_is_exact(kvq, sh, lens, rows):
    call = pt.Call(kvq, sh, lens, rows, pad=3, seed=len(lens), fill=False, keys=3.0)
    run_append(call, sh.D, False)


def long_call(sh):
    """Rows behind the last sequence that make a call as long as those whose values are stored by blocks of tokens."""
    return (3 << 19) // (sh.Hkv * sh.D) + 1


@pytest.mark.parametrize("lens,rows", CALLS)
@pytest.mark.parametrize("sh", SHAPES, ids=str)
def test_long_append_is_exact(kvq, sh, lens, rows):
    call = pt.Call(kvq, sh, lens, rows, pad=long_call(sh), seed=len(lens), fill=False, keys=3.0)
    run_append(call, sh.D, False)


@pytest.mark.parametrize("sh", [S(), S(D=64, gk=64, gv=32, vb=4, dtype="fp16")], ids=str)
def test_long_append_full_of_rows(kvq, sh):
    n = long_call(sh)
    lens = [n // 2 + 70, 300, 0, n // 2 + 1]
    run_append(pt.Call(kvq, sh, lens, [n // 2, 300, 0, n // 2 + 1], pad=0, seed=17, fill=False), 32, True)


@pytest.mark.parametrize("only", ["k", "v"])
def test_one_side_read_back(kvq, only):
    """Keys alone or values alone, into the middle of a buffer, twice: what both together give, and nothing beside it."""
    sh = S(Hkv=3, G=1)
    call = pt.Call(kvq, sh, [300, 131], [290, 131], seed=18, pad=4)
    cache, cu = call.on_gpu()
    both = [torch.zeros(call.n, sh.Hkv, sh.D, dtype=sh.torch_dtype, device="cuda") for _ in range(2)]
    kvq.kvq_paged_dequantize(call.cfg, cache, cu, *both)
    wide = torch.full((call.n + 2, sh.Hkv, sh.D), 7.0, dtype=sh.torch_dtype, device="cuda")
    part = wide[1:1 + call.n]
    for _ in range(2):
        kvq.kvq_paged_dequantize(call.cfg, cache, cu, part if only == "k" else None, part if only == "v" else None)
    assert kvq.kvq_check_status(cache) == 0
    real = int(call.cu[-1])
    assert torch.equal(part[:real], both[only == "v"][:real])
    assert bool((wide[0] == 7).all()) and bool((wide[1 + real:] == 7).all())


@pytest.mark.parametrize("rotary", [0, 16, 48, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_partial_and_interleaved_rotation(kvq, rotary, interleaved):
    call = pt.Call(kvq, S(Hkv=3, G=2), [200, 129], [150, 2], seed=5, fill=False)
    run_append(call, rotary, interleaved)
    if rotary <= 64:
        call = pt.Call(kvq, S(D=64, gk=32, gv=64, dtype="fp16"), [140], [39], seed=6, fill=False)
        run_append(call, rotary, interleaved)


def test_queries_rotated_in_place(kvq):
    run_append(pt.Call(kvq, S(), [300, 140], [200, 1], seed=7, fill=False, pad=2), 128, False, in_place=True)


def test_many_sequences_with_empty_ones(kvq):
    rng = np.random.default_rng(3)
    rows = [int(x) for x in rng.integers(0, 4, 150)]
    rows[0] = rows[-1] = 0
    lens = [r + int(x) for r, x in zip(rows, rng.integers(0, 140, 150))]
    run_append(pt.Call(kvq, S(D=64, gk=64, gv=64, Hkv=1, G=2, dtype="fp16"), lens, rows, seed=8, fill=False, pad=5), 64, False)


@pytest.mark.parametrize("scale", [0.0, 1e-7, 3e4])
def test_constant_tiny_and_large_rows(kvq, scale):
    call = pt.Call(kvq, S(), [150], [40], seed=9, fill=False)
    call.k = (call.k.float() * scale).to(call.k.dtype)
    call.v = (call.v.float() * scale).clamp(-6e4, 6e4).to(call.v.dtype)
    run_append(call, 128, False)


def test_appends_token_by_token_equal_one_append(kvq):
    """A sequence stored in one call, in uneven chunks and token by token: the same bytes."""
    sh = S(Hkv=2)
    n = 290
    whole = pt.Call(kvq, sh, [n], [n], seed=11, fill=False)
    want = run_append(whole, 128, False).pages
    cos, sin = pt.tables(128, n)
    rope = kvq.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    for chunks in ([100, 1, 27, 1, 130, 31], [1] * n):
        cache, cu = whole.on_gpu()
        t = 0
        for c in chunks:
            t += c
            cache.seq_len.fill_(t)
            cu[1] = c
            kvq.kvq_paged_append(whole.cfg, cache, whole.k[t - c:t].cuda(), whole.v[t - c:t].cuda(), cu, rope)
        assert kvq.kvq_check_status(cache) == 0
        assert torch.equal(cache.pages, want)


@pytest.mark.parametrize("pad", [0, long_call(S())])
def test_device_side_refusals_set_the_status_and_write_nothing(kvq, pad):
    sh = S()
    call = pt.Call(kvq, sh, [200, 130], [3, 2], pad=pad, seed=12, fill=False, capacity=256)
    BAD = kvq.STATUS_BAD_INPUT
    cos, sin = pt.tables(128, 256)
    rope = kvq.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())

    def attempt(change, rope=rope, untouched=True):
        cache, cu = call.on_gpu()
        change(cache, cu)
        kvq.kvq_paged_append(call.cfg, cache, call.k.cuda(), call.v.cuda(), cu, rope)
        assert int(cache.status) == BAD and kvq.kvq_check_status(cache) == -9
        same = torch.equal(cache.pages.cpu(), torch.from_numpy(call.pages))
        assert same == untouched
        out = torch.full((call.n, sh.Hkv, sh.D), 7.0, dtype=sh.torch_dtype, device="cuda")
        cache.status.zero_()
        kvq.kvq_paged_dequantize(call.cfg, cache, cu, out, None)
        if untouched and rope is not None and rope.cos.shape[0] >= 256:
            assert int(cache.status) == BAD and bool((out == 7.0).all())

    attempt(lambda c, cu: c.seq_len.copy_(torch.tensor([257, 257], dtype=torch.int32)))      # beyond the capacity
    attempt(lambda c, cu: c.seq_len.copy_(torch.tensor([2, 1], dtype=torch.int32)))          # more rows than tokens
    attempt(lambda c, cu: c.seq_len.copy_(torch.tensor([-5, -2**31], dtype=torch.int32)))
    attempt(lambda c, cu: c.block_table.fill_(10 ** 6))                                       # outside the pool
    attempt(lambda c, cu: c.block_table.fill_(-1))
    attempt(lambda c, cu: cu.copy_(torch.tensor([0, call.n + 4, 3], dtype=torch.int32)))               # not monotonic, beyond the rows
    attempt(lambda c, cu: cu.copy_(torch.tensor([-4, 2**31 - 1, 2**31 - 1], dtype=torch.int32)))
    short = kvq.Rope(rope.cos[:130].contiguous(), rope.sin[:130].contiguous())
    attempt(lambda c, cu: None, short, untouched=False)     # the second sequence fits the rotation's table, the first does not


def test_captured_append_is_replayed_for_other_lengths(kvq):
    """One graph, lengths and offsets changed between replays, padded rows: as eager calls."""
    sh = S(D=64, gk=64, gv=64, dtype="fp16")
    call = pt.Call(kvq, sh, [250, 180], [5, 3], seed=13, fill=False, capacity=384)
    cos, sin = pt.tables(64, 384)
    rope = kvq.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    cache, cu = call.on_gpu()
    cache.block_table.copy_(torch.arange(6, dtype=torch.int32).view(2, 3))
    eager, _ = call.on_gpu()
    for c in (cache, eager):
        c.pages = torch.full((6,) + tuple(call.pages.shape[1:]), 255, dtype=torch.uint8, device="cuda")
        c.c.pages, c.c.n_pages = c.pages.data_ptr(), 6
    eager.block_table.copy_(cache.block_table)
    k, v = call.k.cuda(), call.v.cuda()
    kvq.kvq_paged_append(call.cfg, cache, k, v, cu, rope)
    cache.pages.fill_(255)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvq.kvq_paged_append(call.cfg, cache, k, v, cu, rope)
    for lens, rows in (([250, 180], [5, 3]), ([8, 384], [8, 0]), ([131, 7], [1, 7])):
        for c in (cache, eager):
            c.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        cu.copy_(torch.tensor([0, rows[0], sum(rows)], dtype=torch.int32))
        graph.replay()
        kvq.kvq_paged_append(call.cfg, eager, k, v, cu, rope)
        torch.cuda.synchronize()
        assert torch.equal(cache.pages, eager.pages)
    assert kvq.kvq_check_status(cache) == 0
