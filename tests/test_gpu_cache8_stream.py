"""Streams whose reference cache is in 8 bits (DV_FLAG_CACHE8): frames that meet it only where a call was cut."""
import dataclasses

import numpy as np
import pytest

import oracle
import synth
from oracle import reusevit

from .gpu_util import check_close, dev, encoder, host, require_gpu
from .test_gpu_encoder_options import CARRIED, CUT, H80, MID, SMALL_F32, frames

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


@gpu
@pytest.mark.parametrize("cut", [(30,), (7, 23), (2, 1, 27), (17, 13)])
@pytest.mark.parametrize("batch", [9, 10, 16])
def test_reordered_calls_without_reuse_and_with_all(batch, cut):
    """Reuse off: no frame meets the cache, wherever calls are cut and batches end.  All reused: as at any threshold."""
    m = dataclasses.replace(MID, reorder=True)
    m8 = dataclasses.replace(m, cache8=True)
    blob = synth.make_blob(m, 78, perturb_ln=True)
    fr = frames(m, 30)
    want = stream(m, blob, fr, 32, 8, (30,), None, float("-inf"))
    got = stream(m8, blob, fr, batch, 8, cut, None, float("-inf"))
    assert all(np.array_equal(a, b) for a, b in zip(want, got))
    want, whole = [stream(x, blob, fr, 32, 8, c, None, float("inf")) for x, c in ((m, (30,)), (m8, cut))]
    got = stream(m8, blob, fr, batch, 8, cut, None, float("inf"))
    own = np.ones(30, bool)                     # frames behind a call's last anchor, to the end of their group
    for end in np.cumsum(cut):
        anchor = (end - 1) // 4 * 4
        own[anchor + 1:anchor // 8 * 8 + 8] = False
    for a, b, c in zip(want, whole, got):
        assert np.array_equal(b, c) and np.array_equal(a[own], c[own])


# ---- what frames that meet the cache take from it ---------------------------------------------------
# frames, group, calls and which frames reference one of an earlier call; reordered: the first call ends on anchor
# 4, the past reference of frames 5, 6 and 8
STAR = (11, 4, CUT, CARRIED)
REORDERED = (17, 16, (7, 10), np.isin(np.arange(17), (5, 6, 8)))
# fp32 cases, with a seed whose cached keys and values keep clear of the 8-bit format's ties
F32 = {"rotary": (dict(rotary=True), STAR, 94), "restore": (dict(restore=True), STAR, 92),
       "all": (dict(restore=True, decision=True, rotary=True), STAR, 108), "reorder": (dict(reorder=True), REORDERED, 87),
       "reorder-restore-rotary": (dict(reorder=True, restore=True, rotary=True), REORDERED, 86)}


def case(kw, form, seed, model):
    m = dataclasses.replace(model, cache8=True, **kw)
    blob = synth.make_blob(m, seed, perturb_ln=True)
    n = form[0]
    masks = (np.random.default_rng(seed).random((n, m.depth, m.n_tokens)) < 0.7).astype(np.uint8)
    return m, blob, frames(m, n, seed), masks


@pytest.mark.parametrize("name", F32)
def test_seeds_keep_clear_of_ties(name):
    """No cached value is within 2^-20 of its size and 2^-22 of its row's largest of a border between codes or
    scales (an fp32 row's error: sums of 64 products and a turn, each 2^-24 of their terms)."""
    kw, form, seed = F32[name]
    m, blob, fr, masks = case(kw, form, seed, SMALL_F32)
    seen, keep = [], reusevit.eight_bits

    def watch(rows, heads):
        out = keep(rows, heads)
        far = 2.0 ** -20 * np.abs(rows) + 2.0 ** -22 * np.abs(rows).max(1, keepdims=True)
        seen.append(np.array_equal(keep(rows + far, heads), out) and np.array_equal(keep(rows - far, heads), out))
        return out

    reusevit.eight_bits = watch
    try:
        oracle.encode(fr, blob, m.as_dict(), form[1], masks=masks, cached8=form[3])
    finally:
        reusevit.eight_bits = keep
    assert seen and all(seen)


@gpu
@pytest.mark.parametrize("name", F32)
def test_cached_values_against_the_oracle_f32(name):
    """Injected maps, fp32: every frame within the parity bar of the oracle that quantises what it carries over, and
    the frames that meet it outside the bar of the one that does not."""
    require_gpu()
    kw, form, seed = F32[name]
    m, blob, fr, masks = case(kw, form, seed, SMALL_F32)
    n, group, cut, carried = form
    emb, out, toks = stream(m, blob, fr, 17, group, cut, masks)
    assert len(emb) == n
    sources = out == 2 if m.reorder else None
    r = oracle.encode(fr, blob, m.as_dict(), group, masks=masks, sources=sources, cached8=carried)
    assert np.array_equal(out, r["masks"])
    check_close(emb, r["emb"], "f32", "embeddings")
    check_close(toks, r["tokens"], "f32", "tokens")
    plain = oracle.encode(fr, blob, m.as_dict(), group, masks=masks, sources=sources)
    for f in np.flatnonzero(carried):
        with pytest.raises(AssertionError):
            check_close(toks[f:f + 1], plain["tokens"][f:f + 1], "f32", "unquantised")


@gpu
@pytest.mark.parametrize("kw", [dict(), dict(restore=True), dict(decision=True), dict(reorder=True),
                                dict(reorder=True, restore=True, decision=True, rotary=True)],
                         ids=["plain", "restore", "decision", "reorder", "all"])
@pytest.mark.parametrize("model", [MID, H80], ids=["bf16", "dh80"])
def test_cached_values_against_the_oracle_bf16(model, kw):
    """Gate mode, bf16: with the decisions that were made, every frame within the parity bar of the quantising
    oracle (a key of bf16 may fall on the other side of a code's border; the bar holds all the same)."""
    require_gpu()
    form = REORDERED if kw.get("reorder") else STAR
    m, blob, fr, _ = case(kw, form, 77, model)
    n, group, cut, carried = form
    emb, out, toks = stream(m, blob, fr, 17, group, cut, None, 0.0 if m.decision else 0.9)
    assert len(emb) == n and (out[carried] != 0).any()
    r = oracle.encode(fr, blob, m.as_dict(), group, masks=out, sources=out == 2 if m.reorder else None, cached8=carried)
    check_close(emb, r["emb"], "bf16", "embeddings")
    check_close(toks, r["tokens"], "bf16", "tokens")
