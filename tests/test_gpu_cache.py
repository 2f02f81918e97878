"""The 8-bit paged cache against its definition in 64 bits: slot maps, stored rows, attention."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _mods():
    from paper_2510_22641_amd import runtime, ssd
    return runtime, ssd


def make_cache(lens, heads=2, d_head=64, page=16, spare=2, seed=0, layers=1, max_seq=None, batch=None):
    """A cache whose sequences hold ``lens`` positions of random rows (codes and scales at random)."""
    runtime, _ = _mods()
    max_seq = max_seq or max(max(lens), 1) + 64
    pages = sum(-(-max_seq // page) for _ in lens) + spare
    c = runtime.PagedCache(layers, heads, d_head, batch or len(lens), max_seq, pages, page, page_seed=seed)
    g = torch.Generator().manual_seed(seed)
    for t in (c.k_codes, c.v_codes):
        t.copy_((torch.randn(t.shape, generator=g) * 40).round().clamp(-127, 127).to(torch.int8))
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.exp2(torch.randint(-7, -3, t.shape, generator=g).float()))
    if sum(lens):
        c.grow(lens)
    return c, g


def cached(c, layer, b, n):
    """Keys and values [heads, n, d_head] of sequence b's first n positions, in float64."""
    ps = c.page_size
    pages = c.page_table[b, :-(-n // ps)].long()
    out = []
    for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)):
        x = codes[layer, pages].double() * scale[layer, pages].double()[:, :, None, None]
        out.append(x.transpose(0, 1).reshape(c.n_heads, -1, c.d_head)[:, :n].cpu())
    return out


def attend_reference(c, layer, q, starts, counts, scale, bias=None, apart=False):
    """(output, bound of the error) in float64 from the cache's own values.

    Bound.  A score is a sum of d_head products in float32 (the planes of a float32 query hold its
    24 bits, a bf16 query is exact), times two factors, plus the bias: off by at most
    (d_head + 6) 2^-24 times sum |q k| scale + |bias|.  The exponential's argument is a difference of
    two scores times log2 e, its result one more rounding or two: in all e = 2 ds + (|d| + 6) 2^-24
    relative, d the difference, in the weights and again in their sum.  Sums over n keys in float32
    add n 2^-24 each.  Float32 queries and weights enter the products as two f16 planes, each within
    2^-11 of what it rounds: 2^-22 in all, of sum |q k| scale and of the weights.  bf16 queries are
    exact in one plane (8 bits in 11); their weights are one plane, within 2^-11, and the output is
    rounded once (2^-8).

    apart: blocks of scales more than 2^24 apart among 64 keys.  A code times its scale's ratio to
    the largest is held in f16, whose step below 2^-14 is 2^-24: it is off by at most 2^-25 of the
    largest scale, which moves a score by at most sum |q| scale 2^-25 times that of the keys, and
    an output by 2^-25 times that of the values.  A weight, 2^7 times its value, meets the same step:
    it is off by at most 2^-32 of the row's largest whatever its own size, so a key by 2^-32 times
    its value, at most 127 times the largest scale: 2^-25 of it for each of the keys, where the
    values that carry the weight may be far smaller."""
    H, G = c.n_heads, q.shape[1] // c.n_heads
    q64 = q.double().cpu()
    out, tol = torch.zeros_like(q64), torch.zeros_like(q64)
    u, r = 2.0 ** -24, 0
    for b, (s0, n) in enumerate(zip(starts, counts)):
        if n == 0:
            continue
        k, v = cached(c, layer, b, max(s0 + n, 0))
        N = k.shape[1]
        d = torch.arange(s0, s0 + n)[:, None] - torch.arange(N)
        for h in range(q.shape[1]):
            qh, kh, vh = q64[r:r + n, h], k[h // G], v[h // G]
            x = qh @ kh.t() * scale
            mag = qh.abs() @ kh.abs().t() * abs(scale)
            if bias is not None:
                bh = bias[h].double().cpu()[d.clamp(0, bias.shape[1] - 1)]
                x, mag = x + bh, mag + torch.where(bh.isinf(), 0.0, bh.abs())
            x = x.masked_fill(d < 0, -math.inf)
            some = (x > -math.inf).any(1)
            top = torch.where(some, x.amax(1) if N else torch.zeros(n), 0.0)
            w = torch.exp(x - top[:, None])
            ds = torch.where(x > -math.inf, (c.d_head + 6 + 4) * u * mag, 0.0).amax(1) if N else torch.zeros(n)
            if apart:
                pages = c.page_table[b, :-(-N // c.page_size)].long()
                kt, vt = (float(t[layer, pages, h // G].max()) for t in (c.k_scale, c.v_scale))
                ds = ds + qh.abs().sum(1) * abs(scale) * 2.0 ** -25 * kt
            gap = torch.where(w > 1e-8, top[:, None] - x, 0.0).amax(1) if N else torch.zeros(n)
            L = w.sum(1)
            inv = torch.where(some, 1 / L, 0.0)[:, None]
            out[r:r + n, h] = w @ vh * inv
            e = 2 * ds + (gap + 6) * u
            near = (w @ vh.abs()) * inv
            extra = 2.0 ** (-22 if q.dtype == F32 else -11)
            tol[r:r + n, h] = near * (2 * e + 2 * (N + 8) * u + extra)[:, None] + ((N + 1) * 2.0 ** -25 * vt if apart else 0.0) + 1e-30
        r += n
    if q.dtype == BF16:
        tol = tol + (out.abs() + tol) * 2.0 ** -8
    return out, tol


def check_attend(c, q, new, scale, bias=None, layer=0, row_start=None, out=None, apart=False):
    """The call on the last new[b] rows of each sequence against the reference."""
    if row_start is None:
        row_start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    starts = [l - n for l, n in zip(c.lens, new)]
    got = c.attend(layer, q, row_start, max(max(new), 1), scale, bias, out)
    ref, tol = attend_reference(c, layer, q, starts, new, scale, bias, apart)
    err = (got.double().cpu() - ref).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float((err / tol).max()))
    assert int(c.status) == 0
    return got


# ---- slot maps ----------------------------------------------------------------------------------


def map_reference(table, lens, new, free, ps):
    table, free, slots, starts = [list(r) for r in table], list(free), [], [0]
    for b, (l, n) in enumerate(zip(lens, new)):
        for p in range(l, l + n):
            if p % ps == 0:
                table[b][p // ps] = free.pop(0)
            slots.append(table[b][p // ps] * ps + p % ps)
        starts.append(starts[-1] + n)
    return table, starts, slots


@pytest.mark.parametrize("B,page,most,length", [(1, 16, 1, 0), (1, 1, 5, 3), (3, 5, 9, 40), (64, 16, 1, 300),
                                               (257, 7, 33, 100), (1000, 16, 3, 50), (4096, 16, 2, 20),
                                               (2, 256, 3000, 700)])
def test_page_map_matches_its_definition(B, page, most, length):
    runtime, abi = _mods()
    r = np.random.default_rng(B + page)
    lens = r.integers(0, length + 1, B).tolist()
    new = r.integers(0, most + 1, B).tolist()
    new[0] = most
    P = max(-(-(l + n) // page) for l, n in zip(lens, new)) + 1
    n_pages = sum(-(-(l + n) // page) for l, n in zip(lens, new)) + 3
    ids = r.permutation(n_pages).astype(np.int32)
    table = np.full((B, P), -7, np.int32)
    at = 0
    for b, l in enumerate(lens):
        k = -(-l // page)
        table[b, :k] = ids[at:at + k]
        at += k
    free = ids[at:]
    dev = lambda x, t: torch.tensor(np.asarray(x), dtype=t, device="cuda")  # noqa: E731
    tab, rows = dev(table, torch.int32), sum(new)
    rs = torch.full((B + 1,), -9, dtype=torch.int32, device="cuda")
    slot = torch.full((rows + 5,), -9, dtype=torch.int64, device="cuda")
    taken, status = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(2):  # the lengths unchanged, a second call is the same
        abi.ssd_page_map(B, page, n_pages, P, dev(lens, torch.int32), dev(new, torch.int32), dev(free, torch.int32),
                         len(free), tab, rs, slot, rows + 5, taken, status, torch.cuda.current_stream().cuda_stream)
        want, starts, slots = map_reference(table, lens, new, free, page)
        assert tab.cpu().numpy().tolist() == want
        assert rs.tolist() == starts and slot.tolist() == slots + [-1] * 5
        assert int(status) == 0
        assert int(taken) == sum(-(-(l + n) // page) - -(-l // page) for l, n in zip(lens, new))
    # with the pages in the table, a call without a free list reads them
    slot.fill_(-9)
    abi.ssd_page_map(B, page, n_pages, P, dev(lens, torch.int32), dev(new, torch.int32), None, 0, tab, rs, slot,
                     rows + 5, taken, status, torch.cuda.current_stream().cuda_stream)
    assert slot.tolist() == slots + [-1] * 5 and int(status) == 0 and int(taken) == 0
    assert tab.cpu().numpy().tolist() == want


def _map(abi, lens, new, free, table, page, n_pages, max_rows):
    dev = lambda x, t: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    tab = dev(table, torch.int32)
    rs = torch.zeros(len(lens) + 1, dtype=torch.int32, device="cuda")
    slot = torch.full((max_rows,), -9, dtype=torch.int64, device="cuda")
    taken, status = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    abi.ssd_page_map(len(lens), page, n_pages, len(table[0]), dev(lens, torch.int32), dev(new, torch.int32),
                     None if free is None else dev(free, torch.int32), 0 if free is None else len(free), tab, rs, slot,
                     max_rows, taken, status, torch.cuda.current_stream().cuda_stream)
    return tab.tolist(), rs.tolist(), slot.tolist(), int(taken), int(status)


def test_page_map_reports_what_does_not_fit():
    _, abi = _mods()
    e = [[-1, -1], [-1, -1], [-1, -1]]
    # rows past max_rows are cut, the pages they would need stay free
    t, rs, slot, taken, st = _map(abi, [0, 0, 0], [3, 3, 3], [4, 5, 6, 7, 8, 9], e, 2, 10, 4)
    assert (t, rs, slot, taken) == ([[4, 5], [6, -1], [-1, -1]], [0, 3, 4, 4], [8, 9, 10, 12], 3)
    assert st == abi.SSD_DEV_CAPACITY
    # too few free pages
    t, rs, slot, taken, st = _map(abi, [0, 0, 0], [3, 3, 3], [4, 5, 6], e, 2, 10, 9)
    assert (t, rs, taken) == ([[4, 5], [6, -1], [-1, -1]], [0, 3, 6, 9], 3)
    assert slot == [8, 9, 10, 12, 13, -1, -1, -1, -1] and st == abi.SSD_DEV_CAPACITY
    # a length past the table, negative lengths and counts
    t, rs, slot, taken, st = _map(abi, [3, -1, 0], [3, 2, -4], [4, 5], [[1, 2], [-1, -1], [-1, -1]], 2, 10, 6)
    assert (rs, slot, taken, st) == ([0, 3, 5, 5], [5, -1, -1, -1, -1, -1], 0, abi.SSD_DEV_CAPACITY)
    # pages outside the pools, in the table and in the free list
    t, rs, slot, taken, st = _map(abi, [1, 0], [2, 1], [99], [[-5, -1], [3, -1]], 2, 10, 3)
    assert slot[0] == -1 and slot[1] == -1 and st & abi.SSD_DEV_BAD_PAGE


@pytest.mark.parametrize("free", [-1, -5, 10, 2 ** 31 - 1])
def test_page_map_reports_pages_outside_in_the_free_list(free):
    _, abi = _mods()
    t, rs, slot, taken, st = _map(abi, [1, 0], [1, 3], [4, free], [[2, -1], [-1, -1]], 2, 10, 4)
    assert (t, rs, taken) == ([[2, -1], [4, free]], [0, 1, 4], 2)
    assert slot == [5, 8, 9, -1] and st == abi.SSD_DEV_BAD_PAGE


# ---- stored rows --------------------------------------------------------------------------------


def scale_for(top):
    """The smallest 2^e, e >= -100, with top <= 127 2^e."""
    e = torch.full(top.shape, -100.0, dtype=torch.float64)
    m, x = torch.frexp(top)
    e = torch.where(top > 0, torch.maximum(e, x.double() - 7 + (m > 127 / 128).double()), e)
    return torch.exp2(e)


def store_reference(codes, scale, x, slots, ps):
    """codes [pages, heads, ps, d] and scale [pages, heads] (float64, on the host) after a store."""
    r = 0
    while r < len(slots):
        if slots[r] < 0:
            r += 1
            continue
        page, o = divmod(slots[r], ps)
        n = 1
        while o + n < ps and r + n < len(slots) and slots[r + n] == slots[r] + n:
            n += 1
        got = x[r:r + n].transpose(0, 1)
        held = codes[page, :, :o] * scale[page][:, None, None] if o else codes[page, :, :0]
        top = torch.cat([held, torch.where(got.isfinite(), got, 0.0)], 1).abs().amax((1, 2))
        s = scale_for(top)
        scale[page] = s
        if o:
            codes[page, :, :o] = torch.round(held / s[:, None, None])
        c = torch.round(got / s[:, None, None]).clamp(-127, 127)
        codes[page, :, o:o + n] = torch.where(c.isnan(), 0.0, c)
        r += n


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens,new,heads,d_head,page", [
    ([0], [1], 1, 64, 16), ([7], [1], 3, 128, 16), ([15, 16, 31, 0], [1, 1, 2, 0], 2, 64, 16),
    ([3, 0, 12], [9, 6, 17], 5, 64, 5), ([0, 100], [300, 2], 2, 128, 16), ([2, 250], [500, 290], 1, 128, 256),
    ([1], [70], 2, 64, 1), ([11], [333], 2, 64, 48)])
def test_stored_rows_match_their_definition(lens, new, heads, d_head, page, dtype):
    c, g = make_cache(lens, heads, d_head, page, max_seq=1024, layers=2)
    before = {n: getattr(c, n).clone() for n in ("k_codes", "v_codes", "k_scale", "v_scale")}
    rs, slot = c.grow(new)
    rows = sum(new)
    # magnitudes from row to row far apart, so that scales rise and fall
    k, v = ((torch.randn(rows, heads, d_head, generator=g) * torch.exp2(torch.randint(-8, 8, (rows, heads, 1), generator=g).float()))
            .to(dtype).cuda() for _ in range(2))
    for again in range(2):  # a second store of the same rows changes nothing
        c.append(1, k, v, slot)
        assert int(c.status) == 0
        for n, x in (("k", k), ("v", v)):
            want, ws = before[n + "_codes"][1].cpu().double(), before[n + "_scale"][1].cpu().double()
            store_reference(want, ws, x.cpu().double(), slot.tolist(), page)
            assert torch.equal(getattr(c, n + "_scale")[1].cpu().double(), ws)
            got = getattr(c, n + "_codes")[1].cpu().double()
            live = torch.zeros(c.n_pages, page, dtype=torch.bool)
            for b in range(len(lens)):
                for p in range(c.lens[b]):
                    live[int(c.page_table[b, p // page]), p % page] = True
            live = live[:, None, :, None].expand_as(got)
            assert torch.equal(got[live], want[live])
            # nothing else moves: other layers, and blocks without a new row
            assert torch.equal(getattr(c, n + "_codes")[0], before[n + "_codes"][0])
            assert torch.equal(got[~live], before[n + "_codes"][1].cpu().double()[~live])
    kr, vr = c.rows(1, slot, dtype)
    for n, x in (("k", kr), ("v", vr)):
        pages, off = slot // page, slot % page
        want = getattr(c, n + "_codes")[1][pages, :, off].float() * getattr(c, n + "_scale")[1][pages][..., None]
        assert torch.equal(x, want.to(dtype))
        assert torch.equal(want.to(dtype).float(), want)  # 8 bits and a power of two: exact in either type


def test_a_value_is_off_by_at_most_half_a_code():
    c, g = make_cache([0], heads=4, d_head=128, max_seq=512)
    _, slot = c.grow([200])
    k, v = (torch.randn(200, 4, 128, generator=g).cuda() for _ in range(2))
    c.append(0, k, v, slot)
    kr, _ = c.rows(0, slot)
    for p0 in range(0, 200, 16):
        x, y = k[p0:p0 + 16], kr[p0:p0 + 16]
        top = x.abs().amax((0, 2), keepdim=True)
        # half a code of the smallest power of two over top / 127: at most top / 127
        assert bool(((x - y).abs() <= top / 127).all())


def test_token_by_token_ends_as_one_definition_says():
    """Rows appended one at a time, and after a rollback: the scale follows the rows that are live."""
    c, g = make_cache([0], heads=2, d_head=64, max_seq=64)
    x = torch.randn(3, 2, 64, generator=g)
    x[1] *= 100
    codes, scale = torch.zeros(c.n_pages, 2, 16, 64).double(), torch.zeros(c.n_pages, 2).double()
    _, slot = c.grow([3])
    for i, r in enumerate((0, 1, 1, 2)):  # the large row is rolled back: row 2 takes its place
        at = slot[min(i, 1 if i == 3 else i):][:1] if i != 2 else slot[1:2]
        row = x[r:r + 1].cuda()
        c.append(0, row, row, at)
        store_reference(codes, scale, x[r:r + 1].double(), at.tolist(), 16)
    page = int(c.page_table[0, 0])
    assert torch.equal(c.k_scale[0, page].cpu().double(), scale[page])
    assert torch.equal(c.k_codes[0, page, :, :2].cpu().double(), codes[page, :, :2])
    assert float(scale[page].max()) <= float(x[[0, 2]].abs().max()) / 63.5 * 2


def test_values_at_the_borders_of_codes_and_scales():
    c, _ = make_cache([0], heads=1, d_head=64, max_seq=64)
    tiny = 2.0 ** -140
    rows = [[127.0, 0.5, 1.5, 2.5, -126.5, 0.0], [128.0, 1.0, 3.0, -127.0, 0.0, 0.0], [0.0] * 6,
            [tiny, -tiny, 0.0, 0.0, 0.0, 0.0], [3.4028234663852886e38, 1.0, -3.4e38, 0.0, 0.0, 0.0],
            [127.0 * 2.0 ** -100, 2.0 ** -101, 0.0, 0.0, 0.0, 0.0]]
    for r in rows:
        c, _ = make_cache([0], heads=1, d_head=64, max_seq=64)
        x = torch.zeros(1, 1, 64)
        x[0, 0, :len(r)] = torch.tensor(r)
        _, slot = c.grow([1])
        c.append(0, x.cuda(), x.cuda(), slot)
        page = int(slot[0]) // 16
        s = scale_for(x.double().abs().amax().reshape(1))
        assert float(c.k_scale[0, page, 0]) == float(s)
        assert torch.equal(c.v_codes[0, page, 0, 0].cpu().double(), torch.round(x[0, 0].double() / s))
        assert int(c.status) == 0


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_what_is_not_finite_is_reported_and_stays_alone(dtype):
    _, abi = _mods()
    c, g = make_cache([0, 0], heads=2, d_head=64, max_seq=64)
    _, slot = c.grow([3, 1])
    x = torch.randn(4, 2, 64, generator=g)
    x[1, 0, 3], x[1, 0, 4], x[1, 0, 5] = math.inf, -math.inf, math.nan
    c.append(0, x.to(dtype).cuda(), x.to(dtype).cuda(), slot)
    assert int(c.status) == abi.SSD_DEV_NOT_FINITE
    k, _ = c.rows(0, slot)
    clean = torch.where(x.isfinite(), x, 0.0).to(dtype).float()
    top = clean[:3].abs().amax((0, 2))
    s = scale_for(top.double()).float()
    assert float(k[1, 0, 3]) == 127 * float(s[0]) == -float(k[1, 0, 4]) and float(k[1, 0, 5]) == 0
    fine = x.isfinite()
    assert bool(((k.cpu() - clean).abs() <= torch.cat([s[None].expand(3, 2), scale_for(clean[3:].abs().amax(2).double()).float()])[..., None] / 2)[fine].all())


def test_rows_without_a_slot_strided_rows_and_bad_slots():
    _, abi = _mods()
    g = torch.Generator().manual_seed(3)
    wide = torch.randn(6, 3, 2, 64, generator=g).cuda()
    odd = torch.randn(6 * 129 + 1, generator=g).cuda()[1:].view(6, 129)[:, :128].view(6, 2, 64)  # unaligned rows
    for k, v in ((wide[:, 1], wide[:, 2]), (odd, odd)):
        c, _ = make_cache([4], heads=2, d_head=64, max_seq=64)
        codes, scale = c.k_codes[0].cpu().double(), c.k_scale[0].cpu().double()
        _, slot = c.grow([6])
        some = slot.clone()
        some[2] = -1
        c.append(0, k, v, some)
        store_reference(codes, scale, k.cpu().double(), some.tolist(), 16)
        page = int(c.page_table[0, 0])
        assert torch.equal(c.k_codes[0, page, :, :10].cpu().double(), codes[page, :, :10])
        assert torch.equal(c.k_scale[0].cpu().double(), scale) and int(c.status) == 0
    bad = slot.clone()
    bad[0], bad[1], bad[2] = c.n_pages * 16, -2, 1 << 40
    codes = c.k_codes.clone()
    c.append(0, wide[:3, 0], wide[:3, 0], bad[:3])
    assert int(c.status) == abi.SSD_DEV_BAD_PAGE and torch.equal(c.k_codes, codes)
    c.status.zero_()
    k = c.rows(0, bad[:3])[0]
    assert int(c.status) == abi.SSD_DEV_BAD_PAGE and not bool(k.any())


def test_rows_are_read_back_into_strided_and_unaligned_rows():
    _, abi = _mods()
    c, g = make_cache([20], heads=3, d_head=64, max_seq=64)
    slot = torch.tensor([5, -1, 0, 5], device="cuda") + int(c.page_table[0, 0]) * 16
    slot[1] = -1
    for dt in (F32, BF16):
        want = c.rows(0, slot, dt)[0]
        buf = torch.full((4 * 201 + 1,), 7.0, dtype=dt, device="cuda")
        o, ov = buf[1:].view(4, 201), torch.zeros(4 * 201 + 1, dtype=dt, device="cuda")[1:]
        abi.ssd_cache_load(c._layer(0), 4, slot, o, ov, 201, c._dtype(o), c.status, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(o[[0, 2, 3], :192].reshape(3, 3, 64), want[[0, 2, 3]])
        assert bool((o[1] == 7).all()) and bool((o[:, 192:] == 7).all()) and int(c.status) == 0


# ---- attention ----------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens,new,heads,group,d_head,page", [
    ([0], [1], 1, 1, 64, 16), ([1], [1], 2, 1, 128, 16), ([31, 32, 33], [1, 1, 1], 2, 1, 64, 16),
    ([700], [1], 2, 1, 128, 16), ([300, 0, 5], [1, 1, 0], 2, 4, 64, 7), ([90, 250], [9, 5], 3, 1, 64, 5),
    ([17, 129, 0], [17, 33, 40], 2, 3, 128, 16), ([40], [130], 2, 1, 64, 32), ([5, 64], [100, 257], 1, 5, 128, 24),
    ([2000], [3], 1, 8, 64, 1), ([100, 3], [64, 64], 2, 1, 128, 16), ([1000], [300], 1, 4, 128, 64),
    ([3], [20], 1, 1, 64, 256)])
def test_attention_matches_its_definition(lens, new, heads, group, d_head, page, dtype):
    c, g = make_cache(lens, heads, d_head, page, max_seq=max(l + n for l, n in zip(lens, new)) + 1)
    c.grow(new)
    q = torch.randn(sum(new), heads * group, d_head, generator=g).to(dtype).cuda()
    check_attend(c, q, new, d_head ** -0.5)
    bias = torch.randn(heads * group, 40, generator=g).cuda()  # shorter than the distances
    check_attend(c, (q.float() / 8).to(dtype), new, 1.0, bias)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 40, 200])
def test_attention_masks(rows, dtype):
    """Biases of -inf and of the type's lowest value; rows they leave without a key are zeros."""
    c, g = make_cache([70], 2, 64, 16, max_seq=512)
    c.grow([rows])
    q = torch.randn(rows, 2, 64, generator=g).to(dtype).cuda()
    bias = torch.randn(2, 300, generator=g).cuda()
    bias[0, 50:] = -math.inf   # a window of 50
    bias[1] = -math.inf
    out = check_attend(c, q, [rows], 0.125, bias)
    assert not bool(out[:, 1].any())
    low = torch.finfo(F32).min
    bias = torch.zeros(2, 300, device="cuda")
    bias[0, :20] = low  # the nearest 20 positions as good as masked
    bias[1] = low       # every score the same: the mean
    out = c.attend(0, q, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), rows, 0.0, bias)
    k, v = cached(c, 0, 0, 70 + rows)
    for j in (0, rows - 1):
        p = 70 + j
        for h, part in ((0, v[0, :p - 19]), (1, v[1, :p + 1])):
            ref = part.mean(0)
            lim = part.abs().mean(0) * (2 * (p + 8) * 2.0 ** -24 + 2.0 ** -20 + (0 if dtype == F32 else 2.0 ** -8)) + 1e-9
            assert bool(((out[j, h].double().cpu() - ref).abs() <= lim).all())


@pytest.mark.parametrize("rows", [1, 9, 100])
def test_attention_leaves_other_rows_and_sequences_alone(rows):
    """Rows behind the last sequence, rows without a position, stale codes and scales behind a
    sequence, and NaN queries in their own rows."""
    _, abi = _mods()
    c, g = make_cache([30, 8], 2, 128, 16, max_seq=300, batch=3)
    c.grow([rows, rows, 0])
    n = 2 * rows
    q = torch.randn(n + 4, 4, 128, generator=g).cuda()
    rs = torch.tensor([0, rows, n, n], dtype=torch.int32, device="cuda")
    # pages no sequence reads hold scales of NaN
    used = {int(p) for b in range(2) for p in c.page_table[b, :-(-c.lens[b] // 16)]}
    for p in set(range(c.n_pages)) - used:
        c.k_scale[0, p] = c.v_scale[0, p] = math.nan
    out = torch.full((n + 4, 4, 128), 7.0, device="cuda")
    got = c.attend(0, q, rs, rows, 0.1, None, out)
    ref, tol = attend_reference(c, 0, q[:n], [30, 8], [rows, rows], 0.1)
    assert bool(((got[:n].double().cpu() - ref).abs() <= tol).all())
    assert bool((got[n:] == 7).all())
    bad = q.clone()
    bad[0, 1, 5] = math.nan
    out2 = c.attend(0, bad, rs, rows, 0.1)
    assert bool(out2[0, 1].isnan().all())
    rest = torch.ones(n, 4, dtype=torch.bool)
    rest[0, 1] = False
    assert torch.equal(out2[:n][rest.cuda()], got[:n][rest.cuda()])
    # every row before position 0: no key
    a = dict(B=1, rows=rows, max_rows=rows, max_len=1, n_q_heads=4, dtype=abi.SSD_F32, q=q, ldq=512, out=out, ldo=512,
             seq_len=torch.tensor([-rows - 3], dtype=torch.int32, device="cuda"), max_pages=c.max_pages,
             page_table=c.page_table, scale=1.0, status=c.status)
    at = abi.ssd_cache_attn(**a)
    ws = torch.empty(abi.ssd_cache_attention_workspace(c._layer(0), at) + 256, dtype=torch.uint8, device="cuda")
    abi.ssd_cache_attention(c._layer(0), at, ws, ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert not bool(out[:rows].any()) and bool((out[n:] == 7).all()) and int(c.status) == 0


@pytest.mark.parametrize("rows", [1, 12, 150])
def test_attention_of_strided_and_unaligned_rows(rows):
    c, g = make_cache([44], 2, 64, 16, max_seq=400)
    c.grow([rows])
    for dt in (F32, BF16):
        base = torch.randn(rows * 403 + 1, generator=g).to(dt).cuda()
        q = base[1:].view(rows, 403)[:, :256].view(rows, 4, 64)
        buf = torch.full((rows * 259 + 1,), 7.0, dtype=dt, device="cuda")
        out = buf[1:].view(rows, 259)[:, :256].view(rows, 4, 64)
        check_attend(c, q, [rows], 0.125, out=out)
        assert bool((buf[1:].view(rows, 259)[:, 256:] == 7).all())


@pytest.mark.parametrize("rows", [1, 70])
def test_attention_reports_pages_and_positions_outside(rows):
    _, abi = _mods()
    rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    for page, bit in ((-1, abi.SSD_DEV_BAD_PAGE), (1 << 20, abi.SSD_DEV_BAD_PAGE), (None, abi.SSD_DEV_CAPACITY)):
        c, g = make_cache([100], 2, 64, 16, max_seq=100 + rows)
        c.grow([rows])
        q = torch.randn(rows, 2, 64, generator=g).cuda()
        if page is None:
            c.seq_len += 40  # the last rows sit behind the table
            c.attend(0, q, rs, rows, 0.125)
        else:
            c.page_table[0, 2] = page
            got = c.attend(0, q, rs, rows, 0.125)
            assert bool(got.isfinite().all())
        assert int(c.status) == bit


def test_many_sequences_and_one_long_one():
    lens = [1 + (37 * i) % 200 for i in range(120)]
    c, g = make_cache(lens, 2, 64, 16)
    c.grow([1] * 120)
    check_attend(c, torch.randn(120, 4, 64, generator=g).cuda(), [1] * 120, 0.125)
    c, g = make_cache([20000], 1, 128, 16)
    c.grow([5])
    for dt in (F32, BF16):
        check_attend(c, torch.randn(5, 4, 128, generator=g).to(dt).cuda(), [5], 0.09)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens,new,heads,group,d_head,page", [
    # eight waves a block, whole and split; even and odd pages
    ([600 + i for i in range(70)], [1] * 70, 4, 1, 64, 16), ([650 - i for i in range(33)], [2] * 33, 8, 3, 128, 7),
    ([40000], [1], 1, 4, 128, 16), ([40000], [3], 1, 1, 64, 5),
    # four waves, in ranges
    ([900], [1], 2, 1, 128, 16), ([1023], [7], 2, 2, 64, 9),
    # blocks of 64 pairs with ranges, of 128, of 256 with and without rows left over
    ([2000, 5], [17, 21], 2, 3, 128, 16), ([70, 0], [65, 128], 4, 1, 128, 16), ([30], [129], 1, 1, 64, 3),
    ([10, 77], [300, 257], 64, 1, 64, 16), ([33], [260], 128, 1, 128, 5)])
def test_attention_of_every_launch_shape(lens, new, heads, group, d_head, page, dtype):
    c, g = make_cache(lens, heads, d_head, page, max_seq=max(l + n for l, n in zip(lens, new)) + 1)
    c.grow(new)
    q = torch.randn(sum(new), heads * group, d_head, generator=g).to(dtype).cuda()
    check_attend(c, q, new, -(d_head ** -0.5))  # (a negative factor is a factor)
    bias = torch.randn(heads * group, 300, generator=g).cuda()
    check_attend(c, (q.float() / 8).to(dtype), new, 1.0, bias)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,page", [(1, 16), (1, 3), (9, 16), (40, 16), (140, 5)])
def test_attention_over_blocks_of_scales_far_apart(rows, page, dtype):
    c, g = make_cache([210, 15], 2, 128, page, max_seq=400)
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.exp2(torch.randint(-45, -3, t.shape, generator=g).float()))
    c.grow([rows, rows])
    q = torch.randn(2 * rows, 4, 128, generator=g).to(dtype).cuda()
    check_attend(c, q, [rows, rows], 0.5, apart=True)
    # one range of magnitudes for all, however small or large
    for e in (-99, 90):
        c.k_scale.fill_(2.0 ** -e)
        c.v_scale.fill_(2.0 ** e)
        check_attend(c, (q.float() * 2.0 ** (e - 9)).to(dtype), [rows, rows], 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 30, 200])
def test_attention_of_queries_of_zeros_infinities_and_no_factor(rows, dtype):
    c, g = make_cache([50], 2, 64, 16, max_seq=400)
    c.grow([rows])
    q = torch.randn(rows, 2, 64, generator=g).to(dtype).cuda()
    q[0, 0] = 0                                     # equal scores: the mean of the values
    check_attend(c, q, [rows], 0.125)
    check_attend(c, q, [rows], 0.0)
    rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    out = c.attend(0, q, rs, rows, 0.125)
    bad = q.clone()
    bad[rows - 1, 1, 3] = math.inf
    got = c.attend(0, bad, rs, rows, 0.125)
    assert bool(got[rows - 1, 1].isnan().all())
    got[rows - 1, 1] = out[rows - 1, 1]
    assert torch.equal(got, out)


def test_pools_past_32_bits():
    """A page table that reaches the last pages of pools over 4 GiB."""
    runtime, _ = _mods()
    n_pages = (1 << 32) // (16 * 32 * 128) + 64
    c = runtime.PagedCache(1, 32, 128, 1, 64, n_pages)
    c.free = c.free.flip(0).contiguous()
    _, slot = c.grow([40])
    assert int(slot.min()) >= (n_pages - 3) * 16
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(40, 32, 128, generator=g).cuda() for _ in range(2))
    c.append(0, k, v, slot)
    check_attend(c, torch.randn(40, 32, 128, generator=g).cuda(), [40], 0.09)
    assert bool(((c.rows(0, slot)[0] - k).abs() <= k.abs().max() / 127).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_prompt_then_tokens_together(dtype):
    """As a server uses them: prompts of ragged lengths, then steps of one token and of a chunk, over
    two layers."""
    runtime, _ = _mods()
    c = runtime.PagedCache(2, 2, 64, 3, 256, 60, 16, page_seed=4)
    g = torch.Generator().manual_seed(1)
    for new in ([37, 1, 100], [1, 1, 1], [5, 0, 9], [1, 1, 0]):
        rs, slot = c.grow(new)
        for layer in range(2):
            k, v = (torch.randn(sum(new), 2, 64, generator=g).to(dtype).cuda() for _ in range(2))
            c.append(layer, k, v, slot)
            check_attend(c, torch.randn(sum(new), 4, 64, generator=g).to(dtype).cuda(), new, 0.125, layer=layer, row_start=rs)
    assert int(c.status) == 0


def test_a_captured_step_replays():
    runtime, abi = _mods()
    c = runtime.PagedCache(1, 2, 64, 2, 1200, 200, 16, page_seed=4)
    g = torch.Generator().manual_seed(2)
    rs, slot = c.grow([600, 30])
    c.append(0, *(torch.randn(630, 2, 64, generator=g).cuda() for _ in range(2)), slot)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, new = c.seq_len.clone(), torch.ones(2, dtype=torch.int32, device="cuda")
    k, v, q = (torch.randn(2, h, 64, generator=g).cuda() for h in (2, 2, 4))
    out, slots = torch.zeros_like(q), torch.zeros(2, dtype=torch.int64, device="cuda")
    taken = torch.zeros(1, dtype=torch.int32, device="cuda")
    row_start = torch.zeros(3, dtype=torch.int32, device="cuda")
    c.grow([64, 64])  # pages for the steps to come
    kv = c._layer(0)
    a = abi.ssd_cache_attn(B=2, rows=2, max_rows=1, max_len=1200, n_q_heads=4, dtype=abi.SSD_F32, q=q, ldq=256, out=out,
                           ldo=256, row_start=row_start, seq_len=lens, max_pages=c.max_pages, page_table=c.page_table,
                           scale=0.125, status=st)
    ws = torch.empty(abi.ssd_cache_attention_workspace(kv, a), dtype=torch.uint8, device="cuda")

    def step(stream):
        abi.ssd_page_map(2, 16, c.n_pages, c.max_pages, lens, new, None, 0, c.page_table, row_start, slots, 2, taken, st, stream)
        abi.ssd_cache_store(kv, 2, slots, k, v, 128, abi.SSD_F32, st, stream)
        abi.ssd_cache_attention(kv, a, ws, ws.numel(), stream)

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream().cuda_stream)
    for i in range(5):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got, codes, scales = out.clone(), c.k_codes.clone(), c.k_scale.clone()
        out.zero_()
        step(torch.cuda.current_stream().cuda_stream)  # the same step again changes nothing
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(codes, c.k_codes) and torch.equal(scales, c.k_scale)
        n = [600 + i + 1, 30 + i + 1]
        c.lens = n
        ref, tol = attend_reference(c, 0, q, [n[0] - 1, n[1] - 1], [1, 1], 0.125)
        assert bool(((got.double().cpu() - ref).abs() <= tol).all()) and int(st) == 0
        lens += 1


def test_a_captured_call_keeps_its_workspace():
    """A captured call and the calls after it, larger ones and others' tensors among them, do not write
    each other's memory."""
    runtime, _ = _mods()
    c, g = make_cache([2000, 900], heads=2, max_seq=2048)
    assert c.device.index is not None
    q = torch.randn(2, 4, 64, generator=g).cuda()
    first, _ = c.grow([1, 1])
    c.attend(0, q, first, 1, 0.125)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = c.attend(0, q, first, 1, 0.125)
    rs, _ = c.grow([9, 30])
    more = torch.randn(39, 4, 64, generator=g).cuda()
    late = c.attend(0, more, rs, 30, 0.125)
    ones = [torch.ones(1 << n, device="cuda") for n in range(8, 19) for _ in range(3)]
    # (a row sits at its sequence's end, which has moved)
    ref, tol = attend_reference(c, 0, q, [n - 1 for n in c.lens], [1, 1], 0.125)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert bool(((out.double().cpu() - ref).abs() <= tol).all())
        assert all(bool((t == 1).all()) for t in ones)
        assert torch.equal(late, c.attend(0, more, rs, 30, 0.125)) and int(c.status) == 0
