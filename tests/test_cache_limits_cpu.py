"""Sizes past what the 8-bit cache's launches can index are refused on the host."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # stands for a device pointer: the calls below return before they use one


@pytest.fixture(scope="module")
def abi():
    if not os.path.exists(os.path.join(ROOT, "paper_2510_22641_amd", "libssd.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2510_22641_amd import ssd
    return ssd


def _code(fn, *args):
    from paper_2510_22641_amd import ssd
    with pytest.raises(ssd.SSDError) as e:
        fn(*args)
    return e.value.code


@pytest.mark.parametrize("bad", [dict(max_rows=(1 << 30) + 1), dict(max_rows=(1 << 31) - 1),
                                 dict(n_free=(1 << 30) + 1), dict(n_free=(1 << 31) - 1)])
def test_slot_maps(abi, bad):
    ok = dict(B=2, page_size=16, n_pages=4, max_pages=4, d_seq_len=P, d_new=P, d_free=P, n_free=4,
              d_page_table=P, d_row_start=P, d_slot=P, max_rows=8, d_taken=P, d_status=P, stream=None)
    assert _code(abi.ssd_page_map, *dict(ok, **bad).values()) == abi.SSD_ERR_SHAPE


@pytest.mark.parametrize("name", ["ssd_cache_store", "ssd_cache_load"])
@pytest.mark.parametrize("rows,heads,d_head", [(1 << 24, 4096, 128), (1 << 24, 64, 64), (1 << 23, 128, 64)])
def test_rows(abi, name, rows, heads, d_head):
    cache = abi.ssd_cache(P, P, P, P, n_pages=4, n_heads=heads, page_size=16, d_head=d_head)
    assert _code(getattr(abi, name), cache, rows, P, P, P, heads * d_head, abi.SSD_BF16, P, None) == abi.SSD_ERR_SHAPE


@pytest.mark.parametrize("B,max_rows,heads,kv_heads", [(64, 1 << 22, 32, 32), (4096, 1 << 16, 32, 8), (4096, 1, 4096, 4096),
                                                       (1, 1 << 24, 4096, 1024)])
def test_attention(abi, B, max_rows, heads, kv_heads):
    cache = abi.ssd_cache(P, P, P, P, n_pages=4, n_heads=kv_heads, page_size=16, d_head=64)
    at = abi.ssd_cache_attn(B=B, rows=1 << 20, max_rows=max_rows, max_len=50, n_q_heads=heads, dtype=abi.SSD_F32, q=P,
                            ldq=heads * 64, out=P, ldo=heads * 64, row_start=P, seq_len=P, max_pages=4, page_table=P,
                            scale=1.0, status=P)
    assert abi.ssd_cache_attention_workspace(cache, at) == 0
    assert _code(abi.ssd_cache_attention, cache, at, P, 1 << 40, None) == abi.SSD_ERR_SHAPE


def test_a_bias_without_distances_is_no_bias_to_leave_out():
    import torch
    from paper_2510_22641_amd import runtime
    c = runtime.PagedCache(1, 2, 64, 2, 64, 5, device="cpu")
    q, rs = torch.zeros(3, 2, 64), torch.tensor([0, 1, 3], dtype=torch.int32)
    with pytest.raises(ValueError):
        c.attend(0, q, rs, 2, 1.0, torch.zeros(2, 0))
