"""8-bit contexts at the far end of their longest caches: the rotary and bias tables, the pages and the
passes there against the oracle (tests/test_gpu_cache_decoder.py, whose cached values are the device's)."""
import numpy as np
import pytest
import torch

import synth
from tests import parity
from tests.test_gpu_cache_decoder import _check_stored, _setup, _state

pytestmark = pytest.mark.gpu

LONGEST = 65536


@pytest.mark.parametrize("wl", [synth.S1, synth.S_T5, synth.S_LLAMA, synth.S_LLAMA_F32], ids=lambda w: w.name)
def test_draft_and_verify_at_the_longest_contexts_end(wl):
    base = wl.shape.prefix_len() + wl.prompt_len + wl.new_tokens + wl.gamma + 1
    dd, dec, pr, z, pt, vt = _setup(wl, extra_seq=LONGEST - base)
    assert dd._dims.max_seq == LONGEST
    pending, _ = dd.prefill(pt, vt)  # (the visual keys and values of T5)
    g = torch.Generator().manual_seed(3)
    for codes, scale in ((dd.cache.k_codes, dd.cache.k_scale), (dd.cache.v_codes, dd.cache.v_scale)):
        for l in range(codes.shape[0]):
            codes[l].copy_((torch.randn(codes.shape[1:], generator=g) * 32).round().clamp(-127, 127).to(torch.int8))
        scale.copy_(torch.exp2(torch.randint(-8, -4, scale.shape, generator=g).float()))
    gamma, L = wl.gamma, wl.shape.n_layers
    # the last rows are the cache's last; and a place where one page is half full
    for n in (LONGEST - gamma - 1, 40007):
        dd.seq_len.fill_(n)
        torch.cuda.synchronize()
        d, dl = dd.draft(pending, 1, logits=True)
        dl = dl.cpu().numpy()
        st = _state(dd, dec, 0, n + 1, z[0])
        ref, _ = dec.draft_step(st, int(pending[0]), n)
        parity.check_logits(dl[0, 0], ref, wl.shape, f"draft at {n}")
        _check_stored(st, range(dec.k), [n], f"draft at {n}")
        d, _ = dd.draft(pending, gamma)
        u = np.concatenate([pending.cpu().numpy()[:, None], d.cpu().numpy()], 1)
        t, tl = dd.verify(pending, d, gamma, reuse=False, logits=True)
        tl = tl.cpu().numpy()
        st = _state(dd, dec, 0, n + gamma + 1, z[0])
        for j in range(gamma + 1):
            ref = dec.full_step(st, int(u[0, j]), n + j)[0]
            parity.check_logits(tl[0, j], ref, wl.shape, f"verify at {n + j}")
        _check_stored(st, range(L), range(n, n + gamma + 1), f"verify at {n}")
    assert dd.sync_status() == (0, 0)


@pytest.mark.parametrize("wl", [synth.S_T5, synth.S_LLAMA], ids=lambda w: w.name)
@pytest.mark.parametrize("prompt,batch", [(5000, 1), (40000, 2), (65000, 1)])
def test_prompts_of_many_positions(wl, prompt, batch):
    """The last row's logits and some cached rows of long prefills (the oracle attends the device's rows)."""
    wl = wl.with_(prompt_len=prompt)
    dd, dec, pr, z, pt, vt = _setup(wl, batch=batch)
    pending, lg = dd.prefill(pt, vt, logits=True)
    n = wl.shape.prefix_len() + wl.prompt_len
    # a row's own path through the layers needs the cached rows alone: a few stand for all
    at = [0, 1, 777, 2500, 4095, 4096, n - 2, n - 1]
    for b in range(batch):
        st = _state(dd, dec, b, n, z[b])
        x = dec.embed(pr[b]) if dec.t5 else np.concatenate([np.asarray(z[b], np.float64), dec.embed(pr[b])])
        x = dec.run_layers(x[at], at, st, 0, wl.shape.n_layers)
        parity.check_logits(lg.cpu().numpy()[b], dec.head(x[-1:])[0], wl.shape, "prefill")
        _check_stored(st, range(wl.shape.n_layers), at, "prefill")
    assert dd.sync_status() == (0, 0)
