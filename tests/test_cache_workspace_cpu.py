"""The workspace query of the 8-bit cache's attention, which looks at sizes alone."""
import itertools
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # stands for a device pointer: nothing here reaches the device


@pytest.fixture(scope="module")
def abi():
    if not os.path.exists(os.path.join(ROOT, "paper_2510_22641_amd", "libssd.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2510_22641_amd import ssd
    return ssd


def _query(abi, B, rows, max_rows, max_len, heads=32, kv_heads=32, d_head=128, page_size=16, **kw):
    return abi.ssd_cache_attention_workspace(
        abi.ssd_cache(n_pages=4, n_heads=kv_heads, page_size=page_size, d_head=d_head),
        abi.ssd_cache_attn(B=B, rows=rows, max_rows=max_rows, max_len=max_len, n_q_heads=heads, max_pages=1 << 10, **kw))


def test_pointers_and_strides_are_not_looked_at(abi):
    full = dict(q=P, out=P, row_start=P, seq_len=P, page_table=P, status=P, ldq=1 << 20, ldo=1 << 20)
    for B, rows, max_rows in ((4, 5, 3), (4, 12, 3), (1, 1, 1), (3, 1000, 999)):
        size = _query(abi, B, rows, max_rows, 32768)
        assert size > 0 and size == _query(abi, B, rows, max_rows, 32768, **full)


def test_the_largest_calls_workspace_serves_the_smaller_ones(abi):
    """One request alone, a batch of them, chunks, ragged prompts and padded rows, at any lengths."""
    shapes = [(1, 1, 1), (2, 2, 1), (8, 8, 1), (32, 32, 1), (1, 9, 9), (3, 20, 9), (1, 64, 64), (2, 64, 33), (4, 64, 50),
              (1, 60, 1)]
    for heads, kv, dh in ((32, 32, 128), (32, 8, 128), (12, 12, 64), (40, 5, 64)):
        for (B, rows, most), length in itertools.product(shapes, (1, 100, 129, 500, 513, 3000, 32768, 1 << 20)):
            for n, longer in ((64, length), (200, length), (64, 2 * length), (5000, 1 << 22)):
                assert _query(abi, B, rows, most, length, heads, kv, dh) <= _query(abi, 1, n, n, longer, heads, kv, dh)
    assert _query(abi, 1, 1 << 20, 1 << 20, 1 << 20) == (1 << 16) * 130 * 4


def test_sizes_that_the_call_refuses_and_short_caches_need_none(abi):
    assert _query(abi, 0, 1, 1, 5000) == _query(abi, 1, -1, 1, 5000) == _query(abi, 1, 1, 1, 0) == 0
    assert _query(abi, 1, 1, 1, 5000, heads=33) == 0
    assert _query(abi, 1, 1, 1, 128) == 0
