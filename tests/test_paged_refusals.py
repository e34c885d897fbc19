"""The paged cache's host side: what is refused before anything is launched, and the page arithmetic.  No GPU needed."""
import ctypes

import pytest

from paper_2502_15075_b200 import build as kvq_build


@pytest.fixture(scope="module")
def kvq():
    kvq_build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


A = 4096          # an aligned address that is never dereferenced


def cfg_of(kvq, **over):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, kb=4, vb=2, gk=128, gv=128, k_axis=0, in_dtype=1, capacity_tokens=256)
    base.update(over)
    return kvq.kvq_config(**base)


def cache_of(kvq, **over):
    base = dict(pages=A, n_pages=4, block_table=A, table_stride=2, seq_len=A, status=A)
    base.update(over)
    return kvq.kvq_paged_cache(**base)


def rope_of(kvq, **over):
    base = dict(cos=A, sin=A, n_positions=256, rotary_dim=128, interleaved=0)
    base.update(over)
    return kvq.kvq_rope(**base)


def append(kvq, cfg=None, cache=None, rope=None, k=A, v=A, row=1024, head=128, cu=A, n=3, q=None, q_row=0, q_head=0, q_out=None):
    r = None if rope is None else ctypes.byref(rope)
    return kvq._lib.kvq_paged_append(ctypes.byref(cfg or cfg_of(kvq)), ctypes.byref(cache or cache_of(kvq)), k, v, row, head, cu, n, r, q, q_row, q_head, q_out, None)


def attend(kvq, cfg=None, cache=None, q=A, cu=A, n=3, max_rows=1, window=0, sinks=0, out=A, dtype=2, ws=A, ws_bytes=1 << 40):
    return kvq._lib.kvq_paged_attention(ctypes.byref(cfg or cfg_of(kvq)), ctypes.byref(cache or cache_of(kvq)), q, cu, n, max_rows, window, sinks, out, dtype, 0.0, ws, ws_bytes, None)


UNSUPPORTED = [dict(kb=16), dict(vb=16), dict(kb=3), dict(vb=1), dict(kb=6), dict(k_axis=1), dict(residual_tokens=64), dict(head_dim=96), dict(batch=1025), dict(gk=16)]


@pytest.mark.parametrize("over", UNSUPPORTED, ids=str)
def test_configurations_outside_the_paged_ones(kvq, over):
    cfg = cfg_of(kvq, **over)
    out = ctypes.c_size_t()
    assert append(kvq, cfg) == -2 and attend(kvq, cfg) == -2
    assert kvq._lib.kvq_paged_dequantize(ctypes.byref(cfg), ctypes.byref(cache_of(kvq)), A, 1, A, A, None) == -2
    assert kvq._lib.kvq_paged_workspace_bytes(ctypes.byref(cfg), 1, ctypes.byref(out)) == -2


@pytest.mark.parametrize("over,code", [(dict(pages=None), -1), (dict(block_table=None), -1), (dict(seq_len=None), -1), (dict(status=None), -1), (dict(n_pages=0), -1),
                                       (dict(table_stride=1), -1), (dict(pages=A + 8), -3)], ids=str)
def test_caches(kvq, over, code):
    cache = cache_of(kvq, **over)
    assert append(kvq, cache=cache) == code and attend(kvq, cache=cache) == code
    assert kvq._lib.kvq_paged_dequantize(ctypes.byref(cfg_of(kvq)), ctypes.byref(cache), A, 1, A, A, None) == code


@pytest.mark.parametrize("over,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(cu=None), -1), (dict(n=-1), -1), (dict(k=A + 2), -3), (dict(v=A + 8), -3), (dict(row=127), -1), (dict(row=1028), -3),
    (dict(head=64), -1), (dict(head=132), -3), (dict(q=A), -1), (dict(q_out=A), -1), (dict(q=A, q_out=A + 4096), -1)], ids=str)
def test_append_arguments(kvq, over, code):
    assert append(kvq, **over) == code


def test_append_rotation_arguments(kvq):
    both = dict(q=A, q_out=2 * A, q_row=1024, q_head=128)
    for over, code in ((dict(cos=None), -1), (dict(sin=None), -1), (dict(n_positions=0), -1), (dict(rotary_dim=0), -1), (dict(rotary_dim=24), -1),
                       (dict(rotary_dim=144), -1), (dict(interleaved=2), -1), (dict(cos=A + 4), -3), (dict(sin=A + 8), -3)):
        assert append(kvq, rope=rope_of(kvq, **over), **both) == code
    for over, code in ((dict(q=A + 2), -3), (dict(q_out=A + 8), -3), (dict(q_row=100), -1), (dict(q_head=120), -1), (dict(q_row=1028), -3)):
        assert append(kvq, rope=rope_of(kvq), **{**both, **over}) == code
    # in place only where q is contiguous
    assert append(kvq, rope=rope_of(kvq), q=A, q_out=A, q_row=2048, q_head=128) == -1


@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(cu=None), -1), (dict(n=-1), -1), (dict(max_rows=0), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
    (dict(dtype=3), -1), (dict(q=A + 2), -3), (dict(out=A + 4), -3), (dict(ws=A + 8), -3), (dict(ws_bytes=0), -4)], ids=str)
def test_attention_arguments(kvq, over, code):
    assert attend(kvq, **over) == code


def test_nothing_to_do_is_success_without_tensors(kvq):
    assert append(kvq, n=0, k=None, v=None) == 0
    assert attend(kvq, n=0, q=None, out=None, ws=None, ws_bytes=0) == 0
    assert kvq._lib.kvq_paged_dequantize(ctypes.byref(cfg_of(kvq)), ctypes.byref(cache_of(kvq)), A, 3, None, None, None) == 0


def test_dequantize_arguments(kvq):
    def call(cu=A, n=3, k=A, v=A):
        return kvq._lib.kvq_paged_dequantize(ctypes.byref(cfg_of(kvq)), ctypes.byref(cache_of(kvq)), cu, n, k, v, None)
    assert call(cu=None) == -1 and call(n=-1) == -1 and call(k=A + 2) == -3 and call(v=A + 8) == -3


def test_workspace_bytes(kvq):
    with pytest.raises(kvq.KvqError):
        kvq.kvq_paged_workspace_bytes(cfg_of(kvq), 0)
    assert kvq.kvq_paged_workspace_bytes(cfg_of(kvq), 1) >= 16
    assert kvq.kvq_strerror(-9) != "unknown kvq error"
