"""Which kernel serves a call of the paged attention, worked out on the host.  No GPU needed."""
import pytest

from paper_2502_15075_b200 import build as kvq_build

LAST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def kvq():
    kvq_build.build()
    from paper_2502_15075_b200 import kvq as mod
    return mod


def cfg_of(kvq, **over):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, kb=4, vb=2, gk=128, gv=128, k_axis=0, in_dtype=1, capacity_tokens=32768)
    base.update(over)
    return kvq.kvq_config(**base)


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("capacity", [128, 4096, 32768, 2 ** 31 - 128])
def test_any_announced_number_of_rows_takes_few_launches(kvq, heads, capacity):
    """max_rows up to "no bound at all": at most five launches of the decode kernel, or the other kernel, and no more workspace than as
    many rows as a sequence can have tokens."""
    cfg = cfg_of(kvq, n_q_heads=2 * heads, capacity_tokens=capacity)
    sizes = []
    for rows in [*range(1, 60), capacity, 2 ** 20, 2 ** 30, LAST - 9, LAST - 1, LAST]:
        for window, sinks in ((0, 0), (100, 4), (LAST, LAST)):
            launches = kvq.kvq_debug_paged_launches(cfg, rows, window, sinks)
            assert 0 <= launches <= 5
            if launches:
                assert launches * (8 // heads) >= min(rows, capacity)
        sizes.append(kvq.kvq_paged_workspace_bytes(cfg, rows))
    assert max(sizes) == kvq.kvq_paged_workspace_bytes(cfg, capacity) < 1 << 30


def test_single_tokens_and_prompts(kvq):
    cfg = cfg_of(kvq)
    assert kvq.kvq_debug_paged_launches(cfg, 1) == 1
    assert kvq.kvq_debug_paged_launches(cfg, 2) == 1
    assert kvq.kvq_debug_paged_launches(cfg, 8192) == 0


@pytest.mark.parametrize("batch,kv_heads,capacity,few", [
    (1024, 8, 131072, True), (1024, 63, 4 << 20, True), (1024, 63, 8 << 20, False), (1024, 8, 2 ** 31 - 128, False), (1, 8, 2 ** 31 - 128, True)])
def test_pages_that_pass_31_bits_go_to_the_kernel_that_counts_in_64(kvq, batch, kv_heads, capacity, few):
    """Pool pages may be shared by sequences, so the pages that a batch sees are not bounded by memory: the decode kernel's prefixes are
    32-bit numbers of pages (and up to 18 more per stream), the other kernel's 64-bit ones."""
    cfg = cfg_of(kvq, batch=batch, n_q_heads=kv_heads, n_kv_heads=kv_heads, capacity_tokens=capacity)
    assert few == (batch * kv_heads * (capacity // 128 + 18) < 2 ** 31)
    for rows in (1, 8):
        for window in (0, LAST):
            assert (kvq.kvq_debug_paged_launches(cfg, rows, window) > 0) == few
    assert kvq.kvq_debug_paged_launches(cfg, 1, 1000, 4) > 0          # a window's pages are few
