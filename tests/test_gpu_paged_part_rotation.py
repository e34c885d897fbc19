"""Rotation of a part of the channels: those behind rotary_dim stay as they are, whatever they hold."""
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


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [16, 32, 48])
@pytest.mark.parametrize("sh,pad", [(S(), 0), (S(kb=8, dtype="fp16"), 0), (S(D=64, gk=32, gv=64, dtype="fp16"), 0), (S(kb=2, gk=32), (3 << 19) // 256)], ids=str)
def test_channels_that_are_not_rotated_keep_infinities(kvq, sh, pad, rotary, interleaved):
    """Infinities behind rotary_dim in queries and keys, in short and long calls: queries leave with them, keys are stored as without a
    rotation (the angles here are zero, so the other channels are too)."""
    call = pt.Call(kvq, sh, [140], [39], pad=pad, seed=1, fill=False)
    for x in (call.q, call.k):
        x[3::5, :, rotary + 1] = float("inf")
        x[4::7, 0, sh.D - 1] = float("-inf")
    cos, sin = torch.ones(140, rotary // 2, device="cuda"), torch.zeros(140, rotary // 2, device="cuda")
    pools = []
    q = call.q.cuda()
    for rope in (None, kvq.Rope(cos, sin, interleaved)):
        cache, cu = call.on_gpu()
        q_out = None if rope is None else torch.zeros_like(q)
        kvq.kvq_paged_append(call.cfg, cache, call.k.cuda(), call.v.cuda(), cu, rope, None if rope is None else q, q_out)
        assert kvq.kvq_check_status(cache) == 0
        pools.append(cache.pages.cpu().numpy())
    assert np.array_equal(pools[0], pools[1])
    assert torch.equal(q_out[:39], q[:39])             # (equal takes -0 for +0, no NaN for anything)
