"""Attention over the 8-bit cache where the scales of its blocks lie far apart or near their ends,
against the definition in 64 bits and a bound that follows each key's own weight."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_cache import BF16, F32, make_cache

pytestmark = pytest.mark.gpu

NEAR = 4  # powers of two that the value scales of 64 keys may differ by while one exponent serves them


def _blocks(c, layer, b, n):
    """Codes [heads, n, d_head] and scales [heads, n] of sequence b's first n positions, keys and values."""
    ps = c.page_size
    pages = c.page_table[b, :-(-n // ps)].long()
    out = []
    for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)):
        x = codes[layer, pages].double().transpose(0, 1).reshape(c.n_heads, -1, c.d_head)[:, :n]
        s = scale[layer, pages].double().t().repeat_interleave(ps, 1)[:, :n]
        out += [x.cpu(), s.cpu()]
    return out


def reference(c, q, starts, counts, scale, bias=None, layer=0):
    """(output, bound of the error) in float64.

    Score of a key: products of whole codes with a query held to 2^-22 of itself (float32, two f16
    planes; bf16 elements are exact) and to 2^-39 of its row's largest (an f16 step against 2^14),
    summed in float32 over d_head of them, two factors and the bias: off by (d_head + 10) 2^-24 + 2^-22
    (float32) of sum |q k| scale + |bias|.  The exponential's argument and result add (gap + 6) 2^-24.
    So each weight is off by its own key's error, whatever other keys hold.  Sums over n keys in
    float32: n 2^-24 each, twice for the rescaling.  Weights times their value scale are f16 planes:
    within 2^-22 (two planes) or 2^-11 (one) of themselves, or 2^-25 where they lie under f16's normal
    numbers: they count 2^7 for the largest product of weight and value scale, or for up to 2^(NEAR +
    1) of it where one exponent serves keys of several scales: 2^(NEAR + 1 - 32) of it times the codes.
    Weights under 2^-126 of the largest are zero in float32."""
    G = q.shape[1] // c.n_heads
    q64 = q.double().cpu()
    out, tol = torch.zeros_like(q64), torch.zeros_like(q64)
    u, r = 2.0 ** -24, 0
    for b, (s0, n) in enumerate(zip(starts, counts)):
        if not n:
            continue
        kc, ks, vc, vs = _blocks(c, layer, b, s0 + n)
        N = kc.shape[1]
        d = torch.arange(s0, s0 + n)[:, None] - torch.arange(N)
        for h in range(q.shape[1]):
            qh, g = q64[r:r + n, h], h // G
            v = vc[g] * vs[g][:, None]
            x = qh @ kc[g].t() * ks[g] * scale
            mag = qh.abs() @ kc[g].abs().t() * ks[g] * abs(scale)
            lost = qh.abs().amax(1, keepdim=True) * 2.0 ** -39 * kc[g].abs().sum(1) * ks[g] * abs(scale)
            if bias is not None:
                bh = bias[h].double().cpu()[d.clamp(0, bias.shape[1] - 1)]
                x, mag = x + bh, mag + torch.where(bh.isinf(), 0.0, bh.abs())
            x = x.masked_fill(d < 0, -math.inf)
            top = x.amax(1, keepdim=True)
            top = torch.where(top > -math.inf, top, 0.0)
            gap = torch.where(x > -math.inf, top - x, 0.0)
            w = torch.exp(x - top)
            e = mag * ((c.d_head + 10) * u + (2.0 ** -22 if q.dtype == F32 else 0.0)) + lost + (gap + 6) * u
            dw = torch.exp(x - top + e) - w
            L = w.sum(1, keepdim=True)
            inv = torch.where(L > 0, 1 / L, 0.0)
            out[r:r + n, h] = w @ v * inv
            near = w @ v.abs() * inv
            low = 2.0 ** (NEAR + 1 - 32) * (w * vs[g]).amax(1, keepdim=True) * ((d >= 0).double() @ vc[g].abs())
            gone = torch.where(w < 2.0 ** -125, w, 0.0) @ v.abs()
            tol[r:r + n, h] = (dw @ v.abs() + low + gone) * inv + near * \
                (dw.sum(1, keepdim=True) * inv + 2 * (N + 8) * u + 2.0 ** (-22 if q.dtype == F32 else -11)) + 2.0 ** -148
        r += n
    if q.dtype == BF16:
        tol = tol + (out.abs() + tol) * 2.0 ** -8
    return out, tol


def check(c, q, new, scale, bias=None):
    rs = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    got = c.attend(0, q, rs, max(new), scale, bias).double().cpu()
    ref, tol = reference(c, q, [l - n for l, n in zip(c.lens, new)], new, scale, bias)
    assert bool((tol < math.inf).all()) and int(c.status) == 0
    err = (got - ref).abs()
    assert bool((err <= tol).all()), (float((err / tol).max()), float((err - tol).max()))
    return ref, tol


def pages_of(c, b, first, last):
    """Pages that hold positions first .. last - 1 of sequence b."""
    return c.page_table[b, first // c.page_size:-(-last // c.page_size)].long()


SHAPES = [(1, 16), (1, 3), (9, 16), (20, 5), (40, 16), (140, 16), (140, 5)]
IDS = ["f32", "bf16"]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", SHAPES)
@pytest.mark.parametrize("apart", [10, 18, 26, 34, 90])
def test_values_of_large_scale_and_no_weight(rows, page, apart, dtype):
    """Blocks of large values in front that a bias of -60 or of -inf leaves without weight: the output
    is made of the others, and as exact."""
    c, g = make_cache([400], 2, 64, page, max_seq=800)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** -6)
    c.k_scale.fill_(2.0 ** -6)
    c.v_scale[0, pages_of(c, 0, 0, 32)] = 2.0 ** (apart - 6)
    q = (torch.randn(rows, 4, 64, generator=g) / 8).to(dtype).cuda()
    bias = torch.randn(4, 800, generator=g).cuda()
    # positions under 40 lie 360 and more behind every row, those past 40 + rows nearer
    bias[:2, 360:] -= 60
    bias[2:, 360:] = -math.inf
    ref, tol = check(c, q, [rows], 1.0, bias)
    if dtype == F32 and apart == 34:
        assert float((tol / ref.abs().amax(2, keepdim=True))[:, 2:].max()) < 1e-3  # (the bound says something)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", SHAPES)
def test_values_of_scales_anywhere(rows, page, dtype):
    """Every block its own value scale, low scores on the large ones and high ones on the small."""
    c, g = make_cache([333, 50], 2, 128, page, max_seq=600)
    c.grow([rows, rows])
    e = torch.randint(-60, 60, c.v_scale.shape, generator=g)
    c.v_scale.copy_(torch.exp2(e.float()))
    c.k_scale.fill_(2.0 ** -7)
    q = torch.randn(2 * rows, 4, 128, generator=g).to(dtype).cuda()
    check(c, q, [rows, rows], 0.25)
    # keys against the queries' common direction where values are large
    q = (q.float() / 4 + 1).to(dtype)
    c.k_codes[0].copy_(torch.where(e[0] > 0, -1, 1)[:, :, None, None].cuda() * c.k_codes[0].abs())
    check(c, q, [rows, rows], 0.25)
    check(c, q, [rows, rows], 0.25, torch.randn(4, 77, generator=g).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", [(2, 1), (9, 2), (20, 5), (40, 16), (140, 5), (260, 16)])
def test_later_rows_values_leave_earlier_rows_alone(rows, page, dtype):
    """Value scales that grow from row to row of the call: a row does not see those behind it."""
    c, g = make_cache([45], 4, 64, page, max_seq=600)
    c.grow([rows])
    c.k_scale.fill_(2.0 ** -6)
    for i, p in enumerate(c.page_table[0, :-(-c.lens[0] // page)].tolist()):
        c.v_scale[0, p] = 2.0 ** min(-20 + 9 * i, 110)
    q = torch.randn(rows, 4, 64, generator=g).to(dtype).cuda()
    check(c, q, [rows], 0.125)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("lens,rows,heads,group,d_head", [(700, 1, 32, 1, 64), (5000, 1, 1, 4, 128), (600, 9, 2, 1, 64),
                                                          (900, 20, 2, 3, 64), (3000, 17, 1, 2, 128), (40, 200, 2, 1, 64)])
def test_means_of_values_near_the_largest_number(lens, rows, heads, group, d_head, dtype):
    """Equal weights over hundreds of values of up to 2^127: their sum is no float32 number, their mean
    is, whole and in ranges of keys."""
    c, g = make_cache([lens], heads, d_head, 16, max_seq=lens + rows + 1)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** 121)
    c.v_codes.copy_(c.v_codes.abs().clamp(max=63))
    q = torch.zeros(rows, heads * group, d_head, dtype=dtype, device="cuda")
    check(c, q, [rows], 1.0)
    check(c, q, [rows], 1.0, torch.randn(heads * group, 200, generator=g).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", [(1, 16), (1, 3), (9, 16), (40, 16), (140, 5)])
@pytest.mark.parametrize("query,keys,scale", [(-115, 115, 1.0), (-124, 121, 1.0), (-90, 110, 2.0 ** -30),
                                              (100, -98, 2.0 ** -9), (-30, -60, 2.0 ** 85), (60, 60, 2.0 ** -127)])
def test_queries_and_keys_of_extreme_magnitudes(query, keys, scale, rows, page, dtype):
    """Tiny queries over huge keys and the like: the factor between their products and the scores is
    formed from exponents, and neither part of it has to be a normal number."""
    c, g = make_cache([130], 2, 64, page, max_seq=400)
    c.grow([rows])
    c.v_scale.fill_(0.125)
    c.k_scale.fill_(2.0 ** keys)
    q = torch.randn(rows, 4, 64, generator=g).double() * 2.0 ** (query - 7)
    q = (torch.where(q.abs() < 2.0 ** -126, 0.0, q)).to(dtype).cuda()
    check(c, q, [rows], scale)
    check(c, q, [rows], -scale, torch.randn(4, 90, generator=g).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", SHAPES + [(260, 16)])
@pytest.mark.parametrize("scale", [2.0 ** 17 * 0.7, -2.0 ** 24 * 0.9, 2.0 ** 40 * 0.7, -2.0 ** 100 * 0.6])
def test_scores_of_any_magnitude(rows, page, scale, dtype):
    """Two keys share every row's largest score, far over the others': the output is the mean of their
    values, however coarse the scores' own type is there."""
    c, g = make_cache([290], 2, 64, page, max_seq=600)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** -6)
    c.k_scale.fill_(1.0)
    c.k_codes.clamp_(min=-100, max=100)
    q = torch.randint(1, 4, (rows, 4, 64), generator=g).to(dtype).cuda()  # products are exact
    want = 0.0
    for p in (3, 260):
        page_id, o = int(c.page_table[0, p // page]), p % page
        c.k_codes[0, page_id, :, o] = 101 if scale > 0 else -101  # 64 and more over the others
        want = want + c.v_codes[0, page_id, :, o].double().cpu() * 2.0 ** -7
    rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    got = c.attend(0, q, rs, rows, scale).double().cpu()
    want = want.repeat_interleave(2, 0)[None].expand_as(got)
    # equal weights: planes of 2^-22 (bf16: 2^-11) of values of at most 127 2^-6 each, a division, a rounding
    lim = 2.0 ** (-22 if dtype == F32 else -11) * 2 + want.abs() * (2.0 ** -22 if dtype == F32 else 2.0 ** -8)
    assert bool(((got - want).abs() <= lim).all()) and int(c.status) == 0


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", SHAPES + [(260, 16)])
@pytest.mark.parametrize("magnitude", [2.0 ** 22, 2.0 ** 31, 2.0 ** 90])
def test_scores_far_below_zero_give_means_of_the_values(rows, page, magnitude, dtype):
    """A score's step is past any difference that a weight resolves: still each row is some mean."""
    c, g = make_cache([290], 2, 64, page, max_seq=600)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** -6)
    c.k_scale.fill_(magnitude)
    c.k_codes.copy_(-torch.randint(1, 100, c.k_codes.shape, generator=g).to(torch.int8))
    q = (torch.rand(rows, 4, 64, generator=g) + 0.5).to(dtype).cuda()
    rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    got = c.attend(0, q, rs, rows, 0.125).float()
    at = torch.arange(c.lens[0], device="cuda")
    v = c.v_codes[0, c.page_table[0, at // page].long(), :, at % page].float() * 2.0 ** -6  # [n, heads, d_head]
    hi, lo = (t.repeat_interleave(2, 0) for t in (v.amax(0), v.amin(0)))
    slack = 2.0 ** -7 * float(v.abs().max())
    assert bool(((got <= hi + slack) & (got >= lo - slack)).all()) and int(c.status) == 0
    assert bool((got.abs().amax(-1) > 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", SHAPES)
def test_keys_of_large_scale_and_no_weight(rows, page, dtype):
    """Keys of a scale 2^30 and more over the others', against the queries: their scores are far below,
    and the others' as exact as without them."""
    c, g = make_cache([300], 2, 64, page, max_seq=600)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** -6)
    c.k_scale.fill_(2.0 ** -6)
    q = (torch.randn(rows, 4, 64, generator=g) / 4 + 1).to(dtype).cuda()
    for at, e in ((8, 24), (100, 30), (102, 90), (250, 28)):
        p = pages_of(c, 0, at, at + 1)
        c.k_scale[0, p] = 2.0 ** e
        c.k_codes[0, p] = -c.k_codes[0, p].abs() - 1
        c.k_codes[0, p] = c.k_codes[0, p].clamp(min=-127)
    check(c, q, [rows], 0.125)
    check(c, q, [rows], 0.125, torch.randn(4, 90, generator=g).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", [(2, 1), (9, 2), (20, 5), (40, 16), (140, 5), (260, 16)])
def test_later_rows_keys_leave_earlier_rows_alone(rows, page, dtype):
    """A row's scores do not depend on the key scales of the rows behind it."""
    c, g = make_cache([45], 4, 64, page, max_seq=600)
    c.grow([rows])
    pages = c.page_table[0, :-(-c.lens[0] // page)].tolist()
    q = torch.randn(rows, 4, 64, generator=g).to(dtype).cuda()
    for first in (1, rows // 2):  # the rows from `first` on are masked for those before it
        c.k_scale.fill_(2.0 ** -6)
        for p in pages[(45 + first) // page + 1:]:
            c.k_scale[0, p] = 2.0 ** 40
        n = min((45 + first) // page * page + page - 45, rows)  # rows before those pages
        rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        got = c.attend(0, q, rs, rows, 0.125).double().cpu()[:n]
        ref, tol = reference(c, q[:n], [45], [n], 0.125)
        assert bool(((got - ref).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows,page", SHAPES)
def test_blocks_that_were_never_written(rows, page, dtype):
    """A scale of 0 makes keys and values of zeros, whatever the codes are: among others, and alone."""
    c, g = make_cache([290], 2, 64, page, max_seq=600)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** -6)
    c.k_scale.fill_(2.0 ** -6)
    q = torch.randn(rows, 4, 64, generator=g).to(dtype).cuda()
    for first, last in ((0, 1), (37, 120), (280, 290 + rows)):
        c.v_scale[0, pages_of(c, 0, first, last)] = 0
        c.k_scale[0, pages_of(c, 0, first, last)] = 0
    check(c, q, [rows], 0.125)
    check(c, q, [rows], 0.125, torch.randn(4, 300, generator=g).cuda())
    c.v_scale.fill_(0)
    check(c, q, [rows], 0.125)
    c.k_scale.fill_(0)
    rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    assert not bool(c.attend(0, q, rs, rows, 0.125).any())
    # a factor that is no number is in every row that has a key
    assert bool(c.attend(0, q, rs, rows, math.nan).isnan().all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=IDS)
@pytest.mark.parametrize("rows", [1, 9, 40, 140])
def test_unwritten_blocks_beside_masked_large_ones(rows, dtype):
    """The 64 keys in front are a masked block of values of 2^56 and blocks without any: their scores
    stand for no value at all."""
    c, g = make_cache([290], 2, 64, 16, max_seq=600)
    c.grow([rows])
    c.v_scale.fill_(2.0 ** -6)
    c.k_scale.fill_(2.0 ** -6)
    c.v_scale[0, pages_of(c, 0, 0, 16)] = 2.0 ** 56
    c.v_scale[0, pages_of(c, 0, 16, 64)] = 0
    q = (torch.randn(rows, 4, 64, generator=g) / 8).to(dtype).cuda()
    bias = torch.randn(4, 300, generator=g).cuda()
    bias[:, 275:] = -math.inf
    check(c, q, [rows], 1.0, bias)
