"""Pages of the 8-bit cache that are filled over several stores: what earlier rows keep."""
import math

import pytest
import torch

from tests.test_gpu_cache import BF16, F32, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_the_largest_numbers_stay_as_their_page_is_filled(dtype):
    """A value near the type's largest number gets code 64 of scale 2^122: 2^128, which float32 does not
    hold.  Further rows leave it, and it is read back within half a code, 2^121."""
    top = torch.finfo(dtype).max
    c, g = make_cache([0], heads=2, d_head=64, max_seq=64)
    _, slot = c.grow([9])
    x = torch.randn(9, 2, 64, generator=g)
    x[0, 0, :4] = torch.tensor([top, -top, top / 2, top * (1 - 2.0 ** -6)])
    x[0, 1, 7] = -top
    x = x.to(dtype)
    for first, last in ((0, 1), (1, 4), (4, 5), (5, 9)):
        k = x[first:last].cuda()
        c.append(0, k, k, slot[first:last])
        assert bool((c.k_scale[0, int(slot[0]) // 16] == 2.0 ** 122).all())
        for y in c.rows(0, slot[:last], dtype):
            assert bool(((y.double().cpu() - x[:last].double()).abs() <= 2.0 ** 121).all())
    assert int(c.status) == 0
