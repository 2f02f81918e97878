"""The decode loop over the 8-bit cache against the oracle.

The codes a device holds depend on the order in which its rows came, so the oracle is given the
device's own cached values and computes everything else: a step's logits from those values within the
usual tolerances (tests/parity.py), and the step's keys and values, which the device's cache must hold
to half a code.
"""
import numpy as np
import pytest
import torch

import synth
from oracle.model import Decoder
from tests import parity

pytestmark = pytest.mark.gpu

SMALL = [synth.S1, synth.S_T5, synth.S_LLAMA, synth.S_LLAMA_F32]


class Given(np.ndarray):
    """Cached values that stay as they are; what the oracle would store is kept beside them."""

    def __setitem__(self, at, value):
        self.seen[at] = value


def _given(a):
    a = a.view(Given)
    a.seen = {}
    return a


def _cache(dd, b, n):
    """Device values and code widths of sequence b's first n positions: [L, n, H, dh], [L, n, H]."""
    c, ps = dd.cache, dd.cap.page_size
    pages = dd.page_table[b, :-(-n // ps)].long()
    out = []
    for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)):
        s = scale[:, pages].double()  # [L, pages, H]
        x = codes[:, pages].double() * s[..., None, None]
        x = x.permute(0, 1, 3, 2, 4).reshape(x.shape[0], -1, dd.shape.n_heads, dd.shape.d_head)
        out.append((x[:, :n].cpu().numpy(), s.repeat_interleave(ps, 1)[:, :n].cpu().numpy()))
    return out


def _state(dd, dec, b, n, z):
    st = dec.new_state(n)
    dec.set_visual(st, z)
    (k, ks), (v, vs) = _cache(dd, b, n)
    st.K, st.V = _given(k), _given(v)
    st.widths = (ks, vs)
    return st


def _check_stored(st, layers, positions, what):
    for given, width in ((st.K, st.widths[0]), (st.V, st.widths[1])):
        for l in layers:
            for p in positions:
                want, got = np.asarray(given.seen[l, p]), np.asarray(given)[l, p]
                slack = 2e-2 * float(np.std(want)) + 1e-6
                assert np.all(np.abs(got - want) <= width[l, p][:, None] / 2 + slack), (what, l, p)


def _setup(wl, batch=1, **kw):
    from paper_2510_22641_amd import runtime
    w, z, pr = parity.workload_inputs(wl, 0, batch)
    dd = runtime.from_workload(wl, 0, weights=w, max_batch=batch, kv_dtype="i8", page_seed=7, **kw)
    pt, vt = dd.upload_inputs(pr, z)
    return dd, Decoder(wl.shape, w, wl.draft_layers), pr, z, pt, vt


def _rounds(dd, dec, wl, pr, z, pt, vt, rounds):
    sh, g, L = wl.shape, wl.gamma, wl.shape.n_layers
    B = pt.shape[0]
    pending, lg = dd.prefill(pt, vt, logits=True)
    lg = lg.cpu().numpy()
    n = sh.prefix_len() + pr.shape[1]
    for b in range(B):
        st = _state(dd, dec, b, n, z[b])
        x = dec.embed(pr[b]) if dec.t5 else np.concatenate([np.asarray(z[b], np.float64), dec.embed(pr[b])])
        x = dec.run_layers(x, list(range(n)), st, 0, L)
        parity.check_logits(lg[b], dec.head(x[-1:])[0], sh, f"seq {b} prefill")
        _check_stored(st, range(L), range(n), f"seq {b} prefill")
    for r in range(rounds):
        lens = dd.seq_len.cpu().numpy()
        # one draft step: layers 1..k, the imitation network and the head
        d, dl = dd.draft(pending, 1, logits=True)
        dl = dl.cpu().numpy()
        for b in range(B):
            st = _state(dd, dec, b, int(lens[b]) + 1, z[b])
            ref, _ = dec.draft_step(st, int(pending[b]), int(lens[b]))
            parity.check_logits(dl[b, 0], ref, sh, f"seq {b} round {r} draft")
            _check_stored(st, range(dec.k), [int(lens[b])], f"seq {b} round {r} draft")
        # the whole round, every layer recomputed in the verify
        d, _ = dd.draft(pending, g)
        u = np.concatenate([pending.cpu().numpy()[:, None], d.cpu().numpy()], 1)
        t, tl = dd.verify(pending, d, g, reuse=False, logits=True)
        tl = tl.cpu().numpy()
        for b in range(B):
            st = _state(dd, dec, b, int(lens[b]) + g + 1, z[b])
            at = [int(lens[b]) + j for j in range(g + 1)]
            for j, p in enumerate(at):
                parity.check_logits(tl[b, j], dec.full_step(st, int(u[b, j]), p)[0], sh, f"seq {b} round {r} verify {j}")
            _check_stored(st, range(L), at, f"seq {b} round {r} verify")
        dd.accept(d, t, pending, g)
    assert dd.sync_status() == (0, 0)


@pytest.mark.parametrize("wl", SMALL, ids=lambda w: w.name)
def test_rounds_over_the_8bit_cache(wl):
    _rounds(*[x for x in (lambda s: (s[0], s[1], wl, *s[2:]))(_setup(wl))], rounds=4)


@pytest.mark.parametrize("wl", [synth.S_T5, synth.S_LLAMA], ids=lambda w: w.name)
def test_ragged_batch_over_the_8bit_cache(wl):
    dd, dec, pr, z, pt, vt = _setup(wl, batch=3, extra_seq=8)
    _rounds(dd, dec, wl, pr, z, pt, vt, rounds=3)


@pytest.mark.parametrize("wl", [synth.S1, synth.S_LLAMA], ids=lambda w: w.name)
def test_long_verify_chunks_over_the_8bit_cache(wl):
    """25 rows in ranges of a cache that single rows attend whole."""
    wl = wl.with_(gamma=24, prompt_len=150)
    dd, dec, pr, z, pt, vt = _setup(wl, extra_seq=150)
    _rounds(dd, dec, wl, pr, z, pt, vt, rounds=2)


@pytest.mark.parametrize("wl", [synth.S_T5, synth.S_LLAMA], ids=lambda w: w.name)
def test_contexts_past_1024_positions(wl):
    wl = wl.with_(prompt_len=1100)
    dd, dec, pr, z, pt, vt = _setup(wl)
    _rounds(dd, dec, wl, pr, z, pt, vt, rounds=1)


@pytest.mark.parametrize("wl", SMALL, ids=lambda w: w.name)
def test_generate_equals_the_stepwise_calls_over_the_8bit_cache(wl):
    """Graphs on, verify reusing the drafts' states: the same calls in the same order, token for token;
    without graphs, and in a context that allocates nothing, the same tokens again."""
    from paper_2510_22641_amd import runtime
    dd, dec, pr, z, pt, vt = _setup(wl, batch=2, extra_seq=2 * wl.gamma)
    step = parity.device_run(dd, pt, vt, wl.new_tokens, wl.gamma, reuse=True, logits=False)
    toks, stats = dd.generate(pt, vt, wl.new_tokens, wl.gamma)
    assert toks.cpu().numpy().tolist() == step.tokens and stats["rounds"] == len(step.rounds)
    dd.set_graphs(False)
    again, _ = dd.generate(pt, vt, wl.new_tokens, wl.gamma)
    assert torch.equal(again, toks) and dd.sync_status() == (0, 0)
    w, _, _ = parity.workload_inputs(wl, 0, 2)
    st = runtime.from_workload(wl, 0, weights=w, max_batch=2, kv_dtype="i8", page_seed=7,
                               extra_seq=2 * wl.gamma, static=True)
    toks2, _ = st.generate(pt, vt, wl.new_tokens, wl.gamma)
    st.close()
    assert torch.equal(toks2, toks)


def test_the_tokens_are_those_of_the_float32_cache_up_to_near_ties():
    """Where the two caches' streams first part, the oracle's logits of the two tokens are close, within
    a quarter of the logits' spread (what half a code everywhere does to these decoders was not
    derived: the bound tells a cache that works from one that does not)."""
    from paper_2510_22641_amd import runtime
    for wl in (synth.S_T5, synth.S_LLAMA):
        dd, dec, pr, z, pt, vt = _setup(wl)
        a = dd.generate(pt, vt, wl.new_tokens, wl.gamma)[0].cpu().numpy()[0].tolist()
        w, _, _ = parity.workload_inputs(wl, 0, 1)
        f = runtime.from_workload(wl, 0, weights=w)
        b = f.generate(pt, vt, wl.new_tokens, wl.gamma)[0].cpu().numpy()[0].tolist()
        first = next((i for i, (x, y) in enumerate(zip(a, b)) if x != y), None)
        if first is not None:
            lg = parity.oracle_full_logits_along(dec, pr[0], z[0], a, first)
            assert abs(lg[a[first]] - lg[b[first]]) <= 0.25 * float(np.std(lg))


def test_rows_that_are_not_finite_end_the_call():
    from paper_2510_22641_amd import ssd as abi
    wl = synth.S_LLAMA
    dd, dec, pr, z, pt, vt = _setup(wl)
    vt[0, 3] = float("inf")
    with pytest.raises(abi.SSDError) as e:
        dd.generate(pt, vt, wl.new_tokens, wl.gamma)
    assert e.value.code == abi.SSD_ERR_DEVICE
    assert dd.sync_status() == (abi.SSD_ERR_DEVICE, abi.SSD_DEV_NOT_FINITE)


def test_a_full_8bit_cache_reports_its_capacity():
    from paper_2510_22641_amd import ssd as abi
    wl = synth.S_LLAMA
    dd, dec, pr, z, pt, vt = _setup(wl)
    pending, _ = dd.prefill(pt, vt)
    dd.seq_len.fill_(dd._dims.max_seq - 1)
    before = dd.cache.k_codes.clone()
    dd.draft(pending, 2)
    rc, st = dd.sync_status()
    assert rc == abi.SSD_ERR_DEVICE and st & abi.SSD_DEV_CAPACITY
    page = int(dd.page_table[0, (dd._dims.max_seq - 1) // 16])
    rest = [p for p in range(before.shape[1]) if p != page]
    assert torch.equal(dd.cache.k_codes[:, rest], before[:, rest])
