"""The chunk kernel's axis of (tile, page) pairs may be longer than 31 bits (a prompt of two million tokens, pages shared by many sequences)."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvq():
    from paper_2502_15075_b200 import build
    build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


def test_divisions_of_its_split_are_exact(kvq):
    """Start of share c of N pairs, c N / 148, and the share of a pair, ((x + 1) 148 - 1) / N, for N up to 2^40."""
    rng = random.Random(1)
    n, d = [], []
    for _ in range(4000):
        N = max(148, int(2 ** rng.uniform(8, 40)) + rng.randint(-2, 2))
        c = rng.randint(0, 148)
        start = c * N // 148
        for x in (start - 1, start, rng.randrange(N)):
            x = min(max(x, 0), N - 1)
            n += [c * N, (x + 1) * 148 - 1]
            d += [148, N]
    q = kvq.kvq_debug_divide(*(torch.tensor(v, dtype=torch.int64, device="cuda") for v in (n, d)))
    assert q.tolist() == [a // b for a, b in zip(n, d)]
