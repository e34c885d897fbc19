"""Offsets of a ragged call that are out of order beside sequences that are in order, and sequences without rows."""
import pytest
import torch

import paged_testlib as pt

pytestmark = pytest.mark.gpu

S = pt.Shape
LONG = (3 << 19) // 256 + 1         # rows behind the last sequence that bring a call over the line of values stored by blocks


@pytest.fixture(scope="module")
def kvq():
    from paper_2502_15075_b200 import build
    build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


@pytest.mark.parametrize("pad", [0, LONG])
@pytest.mark.parametrize("offsets", [[0, 5, 3, 8], [0, 5, 5, 4], [0, -1, 5, 8], [0, 5, 10 ** 6, 8], [-2, 3, 5, 8], [0, 3, 5, 2 ** 31 - 1], [4, 3, 5, 8],
                                     [0, 8, 3, 3], [0, 0, -2 ** 31, 0]], ids=str)
def test_offsets_out_of_order_set_the_status_and_spare_older_tokens(kvq, offsets, pad):
    """Every call says so; no token in front of the call's and no page of nobody's changes, nor do the rows of padding."""
    sh = S()
    lens, most = [200, 130, 77], 8
    call = pt.Call(kvq, sh, lens, [3, 2, 3], pad=pad, seed=1, capacity=256)
    cache, cu = call.on_gpu()
    in_order = cu.clone()
    old = torch.tensor([n - most for n in lens], dtype=torch.int32, device="cuda")       # the tokens that no such call may touch
    starts = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), old.cumsum(0, dtype=torch.int32)])

    def older():
        before = cache.seq_len.clone()
        cache.seq_len.copy_(old)
        out = [torch.zeros((int(starts[-1]), sh.Hkv, sh.D), dtype=sh.torch_dtype, device="cuda") for _ in range(2)]
        kvq.kvq_paged_dequantize(call.cfg, cache, starts, *out)
        assert kvq.kvq_check_status(cache) == 0
        cache.seq_len.copy_(before)
        return out
    was, spare = older(), sorted(set(range(call.pages.shape[0])) - set(call.table.flatten().tolist()))
    cu.copy_(torch.tensor(offsets, dtype=torch.int32))
    cos, sin = (torch.from_numpy(x).cuda() for x in pt.tables(128, 256))
    rope = kvq.Rope(cos, sin)
    q_out = torch.full(call.q.shape, 7.0, dtype=sh.torch_dtype, device="cuda")
    kvq.kvq_paged_append(call.cfg, cache, call.k.cuda(), call.v.cuda(), cu, rope, call.q.cuda(), q_out)
    assert int(cache.status) == kvq.STATUS_BAD_INPUT and kvq.kvq_check_status(cache) == -9
    assert bool((q_out[max(most, max(x for x in offsets if x <= call.n)):] == 7.0).all())
    cache.status.zero_()
    out = [torch.full((call.n, sh.Hkv, sh.D), 7.0, dtype=sh.torch_dtype, device="cuda") for _ in range(2)]
    kvq.kvq_paged_dequantize(call.cfg, cache, cu, *out)
    assert int(cache.status) == kvq.STATUS_BAD_INPUT and all(bool((x[most:] == 7.0).all()) for x in out)
    cache.status.zero_()
    for max_rows in (8, 60):
        ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, max_rows), dtype=torch.uint8, device="cuda")
        o = torch.full(call.q.shape, 7.0, device="cuda")
        kvq.kvq_paged_attention(call.cfg, cache, call.q.cuda(), cu, o, ws, max_rows)
        assert int(cache.status) == kvq.STATUS_BAD_INPUT and bool((o[most:] == 7.0).all())
        cache.status.zero_()
    assert all(torch.equal(a, b) for a, b in zip(older(), was))
    assert torch.equal(cache.pages[spare].cpu(), torch.from_numpy(call.pages[spare]))
    # the same call in order makes good what was left
    kvq.kvq_paged_append(call.cfg, cache, call.k.cuda(), call.v.cuda(), in_order, rope, call.q.cuda(), q_out)
    fresh, _ = call.on_gpu()
    kvq.kvq_paged_append(call.cfg, fresh, call.k.cuda(), call.v.cuda(), in_order, rope, call.q.cuda(), torch.empty_like(q_out))
    back = [[torch.zeros((call.n, sh.Hkv, sh.D), dtype=sh.torch_dtype, device="cuda") for _ in range(2)] for _ in range(2)]
    for c, b in ((cache, back[0]), (fresh, back[1])):
        kvq.kvq_paged_dequantize(call.cfg, c, in_order, *b)
        assert kvq.kvq_check_status(c) == 0
    assert all(torch.equal(a, b) for a, b in zip(*back))


@pytest.mark.parametrize("pad", [0, LONG])
@pytest.mark.parametrize("batch", [3, 200, 1024])
def test_a_sequence_without_rows_and_a_bad_length_sets_the_status(kvq, batch, pad):
    """... in every call, and the others are served: the same bytes as without it."""
    sh = S(Hkv=1, D=64, gk=64, gv=64, G=2, dtype="fp16")
    rows = [1] * batch
    rows[batch // 2] = 0
    call = pt.Call(kvq, sh, [5] * batch, rows, pad=4 * pad, seed=2, fill=False, capacity=256)
    pools = []
    for length in (5, 257, -1):
        cache, cu = call.on_gpu()
        cache.seq_len[batch // 2] = length
        kvq.kvq_paged_append(call.cfg, cache, call.k.cuda(), call.v.cuda(), cu)
        want = 0 if length == 5 else kvq.STATUS_BAD_INPUT
        assert int(cache.status) == want
        pools.append(cache.pages.clone())
        cache.status.zero_()
        out = torch.zeros((call.n, 1, 64), dtype=sh.torch_dtype, device="cuda")
        kvq.kvq_paged_dequantize(call.cfg, cache, cu, out, None)
        assert int(cache.status) == want
        for max_rows in (1, 41):
            cache.status.zero_()
            ws = torch.empty(kvq.kvq_paged_workspace_bytes(call.cfg, max_rows), dtype=torch.uint8, device="cuda")
            kvq.kvq_paged_attention(call.cfg, cache, call.q.cuda(), cu, torch.zeros(call.q.shape, device="cuda"), ws, max_rows)
            assert int(cache.status) == want
    assert torch.equal(pools[0], pools[1]) and torch.equal(pools[0], pools[2])
