"""Streams whose reference cache is in 8 bits (DV_FLAG_CACHE8): frames that meet it only where a call was cut."""
import dataclasses

import numpy as np
import pytest

import synth

from .gpu_util import dev, encoder, host, require_gpu
from .test_gpu_encoder_options import MID, frames

gpu = pytest.mark.gpu


def stream(m, blob, fr, batch, group, cut, masks=None, tau=0.9):
    """Embeddings, masks and tokens of a stream, flushed at its end."""
    torch = require_gpu()
    enc = encoder(m, blob, batch)
    outs, k = [], 0
    for c in cut:
        kw = dict(masks_in=dev(masks[k:k + c])) if masks is not None else {}
        outs.append(enc.stream_encode(dev(fr[k:k + c]), group, tau, want_tokens=True, **kw))
        k += c
    if m.reorder:
        outs.append(enc.stream_flush(want_tokens=True))
    torch.cuda.synchronize()
    return [np.concatenate([host(o[j]) for o in outs if o is not None and o[j] is not None]) for j in range(3)]


@gpu
@pytest.mark.parametrize("injected", [False, True])
@pytest.mark.parametrize("batch", [9, 11, 18])
@pytest.mark.parametrize("kw", [dict(), dict(restore=True), dict(decision=True), dict(rotary=True)],
                         ids=["plain", "restore", "decision", "rotary"])
def test_reordered_calls_of_many_batches(kw, batch, injected):
    """A call longer than max_batch_frames is encoded in several batches; its frames find their references in
    the call and are not affected by the cache's rounding: to the bit those of a plain cache.  Of a stream cut inside a
    group only the rest of that group is affected, and results do not depend on max_batch_frames."""
    m = dataclasses.replace(MID, reorder=True, **kw)
    m8 = dataclasses.replace(m, cache8=True)
    blob = synth.make_blob(m, 76, perturb_ln=True)
    n, group = 30, 8
    fr = frames(m, n)
    tau = 0.0 if m.decision else 0.9
    masks = None
    if injected:
        masks = (np.random.default_rng(7).random((n, m.depth, m.n_tokens)) < 0.7).astype(np.uint8)
    want = stream(m, blob, fr, 32, group, (n,), masks, tau)
    got = stream(m8, blob, fr, batch, group, (n,), masks, tau)
    assert all(len(x) == n for x in (*want, *got))
    # (a flush completes the last frames from the cached anchor 28: another call)
    for a, b in zip(want, got):
        assert np.array_equal(a[:29], b[:29])
    cut = (7, 23)       # the first call ends on anchor 4: frames 5 to 7 attend to it
    whole = stream(m8, blob, fr, 32, group, cut, masks, tau)
    got = stream(m8, blob, fr, batch, group, cut, masks, tau)
    for a, b, c in zip(want, whole, got):
        assert np.array_equal(b, c)
        assert np.array_equal(a[np.r_[:5, 8:29]], c[np.r_[:5, 8:29]])
    assert not np.array_equal(want[2][5:8], got[2][5:8])
