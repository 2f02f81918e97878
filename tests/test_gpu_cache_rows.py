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


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("step", [1, 3])
@pytest.mark.parametrize("factor", [1.0, 1.3, 1.9, 2.0, 3.7])
def test_rows_stored_bit_by_bit_are_off_by_less_than_the_largest_scales_code(factor, step, dtype):
    """A page filled over several stores, the magnitudes rising, with rows of 50 and 2 times that given up
    on the way.  Storing rounds by half a code; each rise of the scale (to 2, 4, ... times) rounds again
    by half a code of the new one, in all less than one code of the largest; a value on that scale's
    steps is on those of all smaller ones, so nothing is lost after."""
    c, g = make_cache([0, 0], heads=2, d_head=64, max_seq=96)
    _, slot = c.grow([48, 0])
    x = (torch.randn(48, 2, 64, generator=g) * factor ** torch.arange(48)[:, None, None]).to(dtype)
    most = torch.zeros(48, 2)  # the largest scale that each row's block has had since the row came
    for first in range(0, 48, step):
        for times in {1: (50.0, 1.0), 4: (2.0, 1.0)}.get(first // step % 7, (1.0,)):  # the last of them stays
            k = (x[first:first + step].float() * times).to(dtype).cuda()
            c.append(0, k, k, slot[first:first + step])
            now = c.k_scale[0, (slot // 16).long()].cpu()[:first + step]
            if times == 1.0:
                most[first:first + step] = 0
            most[:first + step] = torch.maximum(most[:first + step], now)
    for y in c.rows(0, slot):
        err = (y.double().cpu() - x.double()).abs()
        assert bool((err < most[..., None].double()).all()), float((err / most[..., None].double()).max())
    assert int(c.status) == 0
    # one store of the same rows: half a code each
    c, _ = make_cache([0, 0], heads=2, d_head=64, max_seq=96)
    _, slot = c.grow([48, 0])
    c.append(0, x.cuda(), x.cuda(), slot)
    once = c.k_scale[0, (slot // 16).long()].double().cpu()[..., None]
    assert bool(((c.rows(0, slot)[0].double().cpu() - x.double()).abs() <= once / 2).all())
