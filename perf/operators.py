"""Measured cases of the 8-bit paged cache: slot maps, storing and reading rows, and attention.

Each case is one call (or, for the cache's rows, the store and the read that follows it) on one
layer's cache: int8 codes in pages of ``page`` positions with one power-of-two scale for each page
and head.  Shapes are the decoders' that the repository serves (12 or 32 heads of 64 with a position
bias, 32 heads of 128 scaled) and grouped heads over the same caches; lengths run from one token to
long contexts.
"""
from __future__ import annotations

import math
import random

import torch

own = False  # true: the library's calls; false: the same arithmetic in elementary torch operations

MAX_E, MIN_E = 122, -100  # exponents of the scales


def _case(name, kind, B, rows, length, heads, kv_heads, d_head, page, dtype, ragged, bias, shape):
    c = dict(kind=kind, B=B, rows=rows, length=length, heads=heads, kv_heads=kv_heads,
             d_head=d_head, page=page, dtype=dtype, ragged=ragged, bias=bias, shape=shape)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token for each of eight running requests: nothing but launch latency
        _case("map-decode-8", "map", 8, 1, 600, 32, 32, 64, 16, "f32", True, False, 1),
        # a server's full batch, prompts and single tokens mixed, pages of five positions
        _case("map-mixed-1024", "map", 1024, 160, 2000, 32, 32, 64, 5, "f32", True, False, 2),
        # one layer's new rows of a 32-request step
        _case("store-decode-32", "store", 32, 1, 900, 32, 32, 64, 16, "f32", True, False, 3),
        # verify chunks that begin and end inside pages of odd size
        _case("store-verify-odd", "store", 8, 9, 333, 12, 12, 64, 5, "bf16", True, False, 4),
        # a long prompt's keys and values
        _case("store-prefill-8k", "store", 1, 8192, 0, 32, 32, 128, 16, "bf16", False, False, 5),
        # the headline decoder's single token: 32 heads of 64 with the position bias, short context
        _case("attend-token-short", "attend", 1, 1, 70, 32, 32, 64, 16, "f32", False, True, 6),
        # a chat request's next token at a long context
        _case("attend-token-32k", "attend", 1, 1, 32768, 32, 32, 128, 16, "bf16", False, False, 7),
        # a batch's next tokens, grouped heads, ragged lengths
        _case("attend-batch-32", "attend", 32, 1, 4096, 32, 8, 128, 16, "f32", True, False, 8),
        # the verify pass of eight requests: nine rows each, with the position bias
        _case("attend-verify-8x9", "attend", 8, 9, 1000, 32, 32, 64, 16, "f32", True, True, 9),
        # verify chunks of ragged sizes over pages of odd size at middle lengths
        _case("attend-verify-odd", "attend", 5, 17, 2777, 24, 8, 128, 7, "bf16", True, False, 10),
        # one image and question of a chat decoder (608 rows), three requests at odd lengths
        _case("attend-prefill-608", "attend", 3, 608, 45, 32, 32, 128, 16, "f32", True, False, 11),
        # a chunk of a long prompt over what was cached before it
        _case("attend-prefill-4k", "attend", 1, 4096, 4096, 32, 8, 128, 16, "bf16", False, False, 12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["map", "store", "store", "attend", "attend", "attend", "attend"])
    kv_heads, group = rng.choice([(4, 1), (12, 1), (32, 1), (32, 1), (8, 3), (8, 4), (4, 8), (1, 5)])
    d_head = rng.choice([64, 128])
    page = rng.choice([16, 16, 16, 32, 64, 5, 7, 1, 24])
    dtype = rng.choice(["f32", "bf16"])
    bias = rng.random() < 0.4
    top = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        if kind == "map":
            B, rows, length = _log_int(rng, 1, 1024), _log_int(rng, 1, 2048), _log_int(rng, 1, 8192)
        elif kind == "store":
            B, rows, length = _log_int(rng, 1, 256), _log_int(rng, 1, 8192), _log_int(rng, 1, 2048)
        else:
            form = rng.choice(["token", "verify", "prefill"])
            B = _log_int(rng, 1, 8 if form == "prefill" else 64)
            rows = {"token": 1, "verify": rng.randint(2, 33), "prefill": _log_int(rng, 34, 4096)}[form]
            length = _log_int(rng, 1, 32768)
        c = _case(None, kind, B, rows, length, kv_heads * group, kv_heads, d_head, page, dtype,
                  rng.random() < 0.7, bias, rng.randrange(1 << 20))
        w = work(c)
        # what a plain form holds at once stays small against the card too
        if _cost(c) <= top and w["bytes"] <= 1 << 30 and _scores(c) <= 1 << 31:
            return c


# ---- sizes -------------------------------------------------------------------------------------


def _sizes(case):
    """Per sequence: cached positions before the call, and the call's new rows."""
    r = random.Random(case["shape"])
    lens, new = [], []
    for b in range(case["B"]):
        if case["ragged"]:
            lens.append(r.randint(case["length"] // 3, case["length"]) if b else case["length"])
            # some sequences have one row, a few none
            new.append(case["rows"] if b == 0 else r.choice([case["rows"], 1, r.randint(0, case["rows"])]))
        else:
            lens.append(case["length"])
            new.append(case["rows"])
    return lens, new


def _scores(case):
    lens, _ = _sizes(case)
    return case["B"] * case["heads"] * case["rows"] * (max(lens) + case["rows"]) if case["kind"] == "attend" else 0


def _up(a, b):
    return -(-a // b)


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 1e15


def work(case):
    lens, new = _sizes(case)
    ps, hk, dh = case["page"], case["kv_heads"], case["d_head"]
    e = 4 if case["dtype"] == "f32" else 2
    rows = sum(new)
    if case["kind"] == "map":
        taken = sum(_up(l + n, ps) - _up(l, ps) for l, n in zip(lens, new))
        return {"bytes": 8 * case["B"] + 8 * taken + 4 * (case["B"] + 1) + 8 * rows, "flops": 0}
    if case["kind"] == "store":
        held = sum(l % ps for l, n in zip(lens, new) if n)  # rows held by blocks that are filled up
        pages = sum(_up(l + n, ps) - l // ps for l, n in zip(lens, new) if n)
        # rows in, codes out; then codes in, rows out
        return {"bytes": 2 * hk * (rows * dh * (e + 1) + held * dh + (rows + held) * dh * (1 + e) + 12 * pages)
                + 16 * rows + 8 * held, "flops": 0}
    keys = sum(l + n for l, n in zip(lens, new) if n)
    pages = sum(_up(l + n, ps) for l, n in zip(lens, new) if n)
    pairs = sum(n * l + n * (n + 1) // 2 for l, n in zip(lens, new))
    bias = 4 * case["heads"] * max(l + n for l, n in zip(lens, new)) if case["bias"] else 0
    return {"bytes": 2 * hk * (keys * dh + 4 * pages) + 4 * pages + 2 * e * rows * case["heads"] * dh + bias,
            "flops": 4 * dh * case["heads"] * pairs}


# ---- inputs ------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 7)
    dev = "cuda"
    lens, new = _sizes(case)
    B, ps, hq, hk, dh = case["B"], case["page"], case["heads"], case["kv_heads"], case["d_head"]
    ft = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = dict(case=case, kind=case["kind"], B=B, ps=ps, hq=hq, hk=hk, dh=dh, ft=ft, rows=sum(new),
             max_new=max(new), max_len=max(l + n for l, n in zip(lens, new)))
    before = [_up(l, ps) for l in lens]
    after = [_up(l + n, ps) for l, n in zip(lens, new)]
    n_pages = sum(after) + 8
    s["n_pages"], s["max_pages"] = n_pages, max(after) + 1
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["new"] = torch.tensor(new, dtype=torch.int32, device=dev)
    # pages in any order; the cached positions' pages are in the table, the others free
    pages = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    held = before if case["kind"] == "map" else after
    first = torch.tensor([0] + held, device=dev).cumsum(0)
    col = torch.arange(s["max_pages"], device=dev)
    at = first[:-1, None] + col
    s["page_table"] = torch.where(col < torch.tensor(held, device=dev)[:, None],
                                  pages[at.clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    s["free"] = pages[sum(held):].contiguous()
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    s["row_start"] = torch.zeros(B + 1, dtype=torch.int32, device=dev)
    if case["kind"] == "map":
        s["slot"] = torch.zeros(s["rows"], dtype=torch.int64, device=dev)
        s["taken"] = torch.zeros(1, dtype=torch.int32, device=dev)
        return s
    s["row_start"][1:] = s["new"].cumsum(0)
    if case["kind"] == "store":
        # slots of the new rows, and of every row the touched blocks then hold
        s["slot"] = _slots(s, s["seq_len"].long(), s["new"].long(), s["rows"])
        back = [l % ps if n else 0 for l, n in zip(lens, new)]
        bt = torch.tensor(back, device=dev)
        s["read"] = _slots(s, s["seq_len"].long() - bt, s["new"].long() + bt, s["rows"] + sum(back))
        s["k"], s["v"] = (_rows(g, (s["rows"], hk, dh), ft) for _ in range(2))
        s["k_out"], s["v_out"] = (torch.zeros(s["read"].numel(), hk, dh, dtype=ft, device=dev) for _ in range(2))
    else:
        # unscaled scores with a position bias (T5), or scaled ones
        s["scale"] = 1.0 if case["bias"] else dh ** -0.5
        s["q"] = (torch.randn(s["rows"], hq, dh, generator=g, device=dev) * (dh ** -0.5 if case["bias"] else 1.0)).to(ft)
        s["bias"] = torch.randn(hq, s["max_len"], generator=g, device=dev) if case["bias"] else None
        s["out"] = torch.zeros(s["rows"], hq, dh, dtype=ft, device=dev)
        s["workspace"] = None
    # the cache: codes of normal values whose largest fills the range (one page more than the
    # table names, where the plain form drops what belongs nowhere)
    for n in ("k", "v"):
        c = torch.empty(n_pages + 1, hk, ps, dh, dtype=torch.int8, device=dev)
        for p in range(0, n_pages + 1, 4096):  # in pieces: the float values are four times the codes
            part = c[p:p + 4096]
            part.copy_((torch.randn(part.shape, generator=g, device=dev) * 32).round_().clamp_(-127, 127))
        s[n + "_codes"] = c
        e = torch.randint(-6, -3, (n_pages + 1, hk), generator=g, device=dev)
        s[n + "_scale"] = torch.exp2(e.float())
    return s


def _rows(g, shape, ft):
    """Rows of keys or values: normal, with a few large channels in each head."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = torch.rand(shape[1:], generator=g, device="cuda") < 0.03
    return (x * torch.where(big, 6.0, 1.0)).to(ft)


def _slots(s, start, count, total):
    """Slots of positions start .. start + count of every sequence, one after the other."""
    end = count.cumsum(0)
    r = torch.arange(total, device=end.device)
    b = torch.searchsorted(end, r, right=True)
    p = start[b] + r - (end - count)[b]
    return s["page_table"][b, p // s["ps"]].long() * s["ps"] + p % s["ps"]


# ---- one pass ----------------------------------------------------------------------------------


def run(s):
    return _OWN[s["kind"]](s) if own else _PLAIN[s["kind"]](s)


def _plain_map(s):
    ps, dev = s["ps"], s["seq_len"].device
    start, count = s["seq_len"].long(), s["new"].long()
    before = (start + ps - 1) // ps
    need = (start + count + ps - 1) // ps - before
    base = need.cumsum(0) - need
    col = torch.arange(s["max_pages"], device=dev)
    j = col - before[:, None]
    fresh = (j >= 0) & (j < need[:, None])
    at = (base[:, None] + j).clamp(0, s["free"].numel() - 1)
    table = torch.where(fresh, s["free"][at], s["page_table"])
    end = count.cumsum(0)
    r = torch.arange(s["rows"], device=dev)
    b = torch.searchsorted(end, r, right=True)
    p = start[b] + r - (end - count)[b]
    slot = table[b, p // ps].long() * ps + p % ps
    row_start = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), end]).to(torch.int32)
    return {"page_table": table, "row_start": row_start, "slot": slot, "taken": need.sum().to(torch.int32).reshape(1)}


def _pow2(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _plain_blocks(s, x, codes, scale):
    """Stores rows x into the blocks they touch, [B][blocks] of them (the spare last page where a
    sequence touches fewer)."""
    ps, dev, n_pages = s["ps"], x.device, s["n_pages"]
    start, count = s["seq_len"].long(), s["new"].long()
    nb = (s["max_new"] + ps - 2) // ps + 1
    page_no = (start // ps)[:, None] + torch.arange(nb, device=dev)
    used = (page_no * ps < (start + count)[:, None]) & (count > 0)[:, None]
    page = torch.where(used, s["page_table"].gather(1, page_no.clamp(max=s["max_pages"] - 1)).long(), n_pages)
    pos = page_no[:, :, None] * ps + torch.arange(ps, device=dev)
    held = (pos < start[:, None, None])[:, :, None, :, None]
    j = pos - start[:, None, None]
    fresh = ((j >= 0) & (j < count[:, None, None]) & used[:, :, None])[:, :, None, :, None]
    row = (s["row_start"][:-1].long()[:, None, None] + j).clamp(0, s["rows"] - 1)
    xr = x.float()[row].transpose(2, 3)  # [B][blocks][heads][offset][d_head]
    old, so = codes[page].float(), scale[page]
    top = torch.maximum(torch.where(fresh, xr, 0.0).abs().amax((3, 4)),
                        torch.where(held, old, 0.0).abs().amax((3, 4)) * so)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e.long() - 7 + (m > 127 / 128).long(), MIN_E).clamp(min=MIN_E)
    inv = _pow2(-e)[..., None, None]
    c = torch.where(fresh, torch.round(xr * inv),
                    torch.where(held, torch.round(old * so[..., None, None] * inv), old))
    codes[page] = c.to(torch.int8)
    scale[page] = _pow2(e)


def _plain_read(s, codes, scale):
    page, off = s["read"] // s["ps"], s["read"] % s["ps"]
    return (codes[page, :, off].float() * scale[page][..., None]).to(s["ft"])


def _plain_store(s):
    _plain_blocks(s, s["k"], s["k_codes"], s["k_scale"])
    _plain_blocks(s, s["v"], s["v_codes"], s["v_scale"])
    n = s["n_pages"]
    return {"k": _plain_read(s, s["k_codes"], s["k_scale"]), "v": _plain_read(s, s["v_codes"], s["v_scale"]),
            "k_scale": s["k_scale"][:n], "v_scale": s["v_scale"][:n]}


def _plain_attend(s):
    dev, B, ps, hk, dh = s["q"].device, s["B"], s["ps"], s["hk"], s["dh"]
    group, M = s["hq"] // hk, s["max_new"]
    n_blocks = (s["max_len"] + ps - 1) // ps
    table = s["page_table"][:, :n_blocks].long().clamp(min=0)
    N = n_blocks * ps

    def values(codes, scale):  # [B][kv heads][N][d_head]
        x = codes[table].float() * scale[table][..., None, None]
        return x.transpose(1, 2).reshape(B, hk, N, dh)

    start, count = s["seq_len"].long(), s["new"].long()
    j = torch.arange(M, device=dev)
    row = (s["row_start"][:-1].long()[:, None] + j).clamp(max=s["rows"] - 1)  # [B][M]
    q = s["q"].float()[row].reshape(B, M, hk, group, dh).permute(0, 2, 3, 1, 4)
    q = q.reshape(B, hk, group * M, dh).contiguous()
    k = values(s["k_codes"], s["k_scale"])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    del k
    x = x.view(B, s["hq"], M, N)
    d = (start[:, None] + j)[:, :, None] - torch.arange(N, device=dev)  # [B][M][N] distances
    if s["bias"] is not None:
        x = x + s["bias"][:, d.clamp(0, s["max_len"] - 1)].transpose(0, 1)
    x = x.masked_fill((d < 0)[:, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hk, group * M, N), values(s["v_codes"], s["v_scale"]))
    o = o.view(B, s["hq"], M, dh).transpose(1, 2).reshape(B * M, s["hq"], dh)
    # back to the rows in order
    end = count.cumsum(0)
    r = torch.arange(s["rows"], device=dev)
    b = torch.searchsorted(end, r, right=True)
    return o[b * M + r - (end - count)[b]].to(s["ft"])


def _dtype(s, abi):
    return abi.SSD_F32 if s["ft"] == torch.float32 else abi.SSD_BF16


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_map(s):
    from paper_2510_22641_amd import ssd as abi
    abi.ssd_page_map(s["B"], s["ps"], s["n_pages"], s["max_pages"], s["seq_len"], s["new"], s["free"],
                     s["free"].numel(), s["page_table"], s["row_start"], s["slot"], s["rows"],
                     s["taken"], s["status"], _stream())
    return {n: s[n] for n in ("page_table", "row_start", "slot", "taken")}


def _cache(s, abi):
    return abi.ssd_cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["n_pages"], s["hk"],
                       s["ps"], s["dh"])


def _own_store(s):
    from paper_2510_22641_amd import ssd as abi
    kv, st, dt, ld, n = _cache(s, abi), _stream(), _dtype(s, abi), s["hk"] * s["dh"], s["n_pages"]
    abi.ssd_cache_store(kv, s["rows"], s["slot"], s["k"], s["v"], ld, dt, s["status"], st)
    abi.ssd_cache_load(kv, s["read"].numel(), s["read"], s["k_out"], s["v_out"], ld, dt, s["status"], st)
    return {"k": s["k_out"], "v": s["v_out"], "k_scale": s["k_scale"][:n], "v_scale": s["v_scale"][:n]}


def _own_attend(s):
    from paper_2510_22641_amd import ssd as abi
    kv, ld = _cache(s, abi), s["hq"] * s["dh"]
    a = abi.ssd_cache_attn(B=s["B"], rows=s["rows"], max_rows=s["max_new"], max_len=s["max_len"],
                         n_q_heads=s["hq"], dtype=_dtype(s, abi), q=s["q"], ldq=ld, out=s["out"], ldo=ld,
                         row_start=s["row_start"], seq_len=s["seq_len"], page_table=s["page_table"],
                         max_pages=s["max_pages"], bias=s["bias"],
                         n_bias=s["max_len"] if s["bias"] is not None else 0, scale=s["scale"],
                         status=s["status"])
    if s["workspace"] is None:  # a program sizes its workspace once
        s["workspace"] = torch.empty(abi.ssd_cache_attention_workspace(kv, a), dtype=torch.uint8, device="cuda")
    abi.ssd_cache_attention(kv, a, s["workspace"], s["workspace"].numel(), _stream())
    return s["out"]


_PLAIN = {"map": _plain_map, "store": _plain_store, "attend": _plain_attend}
_OWN = {"map": _own_map, "store": _own_store, "attend": _own_attend}


# ---- the definition in 64 bits -----------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _sizes(case)
    return {"map": _exact_map, "store": _exact_store, "attend": _exact_attend}[case["kind"]](s, lens, new)


def _exact_map(s, lens, new):
    table, free, ps = s["page_table"].tolist(), iter(s["free"].tolist()), s["ps"]
    slots, starts, taken = [], [0], 0
    for b, (l, n) in enumerate(zip(lens, new)):
        for p in range(l, l + n):
            if p % ps == 0:
                table[b][p // ps] = next(free)
                taken += 1
            slots.append(table[b][p // ps] * ps + p % ps)
        starts.append(starts[-1] + n)
    dev = s["seq_len"].device
    i32 = dict(dtype=torch.int32, device=dev)
    return {"page_table": torch.tensor(table, **i32), "row_start": torch.tensor(starts, **i32),
            "slot": torch.tensor(slots, dtype=torch.int64, device=dev), "taken": torch.tensor([taken], **i32)}


def _exact_store(s, lens, new):
    ps, table = s["ps"], s["page_table"].tolist()
    out = {}
    for name in ("k", "v"):
        x, vals, scales = s[name].double(), [], s[name + "_scale"].double()
        row = 0
        for b, (l, n) in enumerate(zip(lens, new)):
            p = l
            while p < l + n:
                page, o = table[b][p // ps], p % ps
                m = min(ps - o, l + n - p)
                got = x[row:row + m].transpose(0, 1)  # [heads][rows][d_head]
                held = s[name + "_codes"][page, :, :o].double() * scales[page][:, None, None]
                top = torch.cat([held, got], 1).abs().amax((1, 2))
                e = torch.ceil(torch.log2(top.clamp(min=2.0 ** (MIN_E - 20)) / 127))
                # the logarithm's own rounding, one way and the other
                e = torch.where(top <= 127 * torch.exp2(e - 1), e - 1, e)
                e = torch.where(top > 127 * torch.exp2(e), e + 1, e).clamp(min=MIN_E)
                sc = torch.exp2(e)
                scales[page] = sc
                held = torch.round(held / sc[:, None, None])
                vals.append((torch.cat([held, torch.round(got / sc[:, None, None])], 1) * sc[:, None, None]).transpose(0, 1))
                p, row = p + m, row + m
        out[name] = torch.cat(vals) if vals else x[:0]
        out[name + "_scale"] = scales[:s["n_pages"]]
    return out


def _exact_attend(s, lens, new):
    ps, hk, dh = s["ps"], s["hk"], s["dh"]
    group = s["hq"] // hk
    out = torch.zeros(s["rows"], s["hq"], dh, dtype=torch.float64, device="cuda")
    row = 0
    for b, (l, n) in enumerate(zip(lens, new)):
        if not n:
            continue
        pages = s["page_table"][b, :_up(l + n, ps)].long()
        dist = torch.arange(l, l + n, device="cuda")[:, None] - torch.arange(l + n, device="cuda")
        for h in range(hk):
            k, v = ((s[c + "_codes"][pages, h].double() * s[c + "_scale"][pages, h].double()[:, None, None]).reshape(-1, dh)[:l + n]
                    for c in ("k", "v"))
            for g in range(group):
                x = s["q"][row:row + n, h * group + g].double() @ k.t().contiguous() * s["scale"]
                if s["bias"] is not None:
                    x = x + s["bias"][h * group + g].double()[dist.clamp(min=0)]
                x = x.masked_fill(dist < 0, -math.inf)
                out[row:row + n, h * group + g] = torch.softmax(x, -1) @ v
        row += n
    return out
