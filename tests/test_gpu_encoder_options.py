"""The encoder with rotary positions (DV_FLAG_ROTARY) and with a stream's reference cache in 8 bits
(DV_FLAG_CACHE8), against the CPU oracle and against itself."""
import dataclasses

import numpy as np
import pytest

import oracle
import synth
from oracle import reusevit
from synth.configs import ModelConfig

from .gpu_util import check_close, dev, encoder, host, mask_parity, require_gpu
from .test_gpu_parity import _video

gpu = pytest.mark.gpu

SMALL_F32 = ModelConfig(144, 16, 2, 64, 2, 128, "f32")      # 82 tokens: two pages of the cache
MID = ModelConfig(112, 16, 3, 256, 4, 512, "bf16")
H80 = ModelConfig(144, 16, 2, 640, 8, 640, "bf16")          # head dim 80, two pages


def frames(m, n, seed=61):
    return _video(m, n, seed=seed, sigma=0.02, pan=1.0)


# ---- rotary positions ----------------------------------------------------------------------------
def test_rotary_is_a_turn_of_relative_places():
    """The oracle's turn: scores depend on differences of rows and columns, the class token is
    unchanged."""
    rng = np.random.default_rng(0)
    rows = np.tile(rng.standard_normal((2, 64)), (41, 1))          # 82 tokens of a 9 x 9 grid, two contents
    t = reusevit.turn_rows(rows, np.arange(82), 2, 9)
    assert np.allclose(t[0], rows[0])
    assert np.allclose(np.linalg.norm(t, axis=1), np.linalg.norm(rows, axis=1))
    q, k = t[1:, :32], t[1:, :32]
    s = q @ k.T
    assert np.isclose(s[0, 20], s[36, 56]) and not np.isclose(s[0, 20], s[0, 22])   # (0,0)-(2,2), (4,0)-(6,2)


@gpu
@pytest.mark.parametrize("m,kw", [
    (SMALL_F32, dict()), (MID, dict()), (H80, dict()), (MID, dict(restore=True)), (MID, dict(decision=True)),
    (MID, dict(reorder=True))], ids=["f32", "bf16", "dh80", "restore", "decision", "reorder"])
def test_rotary_encoder_against_oracle(m, kw):
    """Gate mode, teacher-forced: decisions outside the threshold's band are the oracle's, outputs
    within the parity bar; the same frames without the turn are far from them."""
    torch = require_gpu()
    m = dataclasses.replace(m, rotary=True, **kw)
    blob = synth.make_blob(m, 71, perturb_ln=True)
    fr = frames(m, 9)
    tau = 0.0 if m.decision else float(np.float32(0.9))
    enc = encoder(m, blob, 8)
    emb, masks, toks = enc.encode(dev(fr), 4, tau, want_tokens=True)
    torch.cuda.synchronize()
    masks = host(masks)
    sources = masks == 2 if m.reorder else None
    r = oracle.encode(fr, blob, m.as_dict(), 4, masks=masks, sources=sources)
    if not m.decision:
        bad, _ = mask_parity(masks, r["cos"], tau)
        assert bad == 0
    check_close(host(emb), r["emb"], m.dtype, "embeddings")
    check_close(host(toks), r["tokens"], m.dtype, "tokens")
    plain = oracle.encode(fr, blob, dict(m.as_dict(), rotary=False), 4, masks=masks, sources=sources)
    with pytest.raises(AssertionError):
        check_close(host(emb), plain["emb"], m.dtype, "without the turn")


@gpu
@pytest.mark.parametrize("m", [SMALL_F32, MID], ids=["f32", "bf16"])
def test_rotary_stream_equals_one_shot_bitwise(m):
    torch = require_gpu()
    m = dataclasses.replace(m, rotary=True)
    blob = synth.make_blob(m, 72, perturb_ln=True)
    fr = frames(m, 14)
    want = encoder(m, blob, 8).encode(dev(fr), 4, 0.9, want_tokens=True)
    enc = encoder(m, blob, 8)
    outs, k = [], 0
    for c in (3, 5, 1, 5):
        outs.append(enc.stream_encode(dev(fr[k:k + c]), 4, 0.9, want_tokens=True))
        k += c
    for j in range(3):
        assert torch.equal(torch.cat([o[j] for o in outs]), want[j])
    off = torch.empty_like(want[0])
    encoder(m, blob, 8).encode_noalloc(dev(fr), 4, 0.9, off)
    assert torch.equal(off, want[0])
    dense = encoder(m, blob, 8).encode(dev(fr), 4, float("-inf"))
    none = encoder(m, blob, 8).encode_masked(dev(fr), 4, torch.zeros_like(want[1]))
    assert torch.equal(dense[0], none[0])


# ---- the 8-bit reference cache -------------------------------------------------------------------
CUT = (5, 2, 1, 3)    # calls of a stream in groups of 4: frames 5, 6, 7 and 9 .. 10 continue a group
CARRIED = np.array([False] * 5 + [True] * 3 + [False] + [False] * 2)
SEED = 73


def cached_case(m, seed):
    blob = synth.make_blob(m, seed, perturb_ln=True)
    fr = frames(m, 11, seed)
    masks = (np.random.default_rng(seed).random((11, m.depth, m.n_tokens)) < 0.7).astype(np.uint8)
    return blob, fr, masks


def test_oracle_holds_the_reference_in_eight_bits():
    """The oracle's quantiser against a search of the format's values; and the inputs of the fp32
    comparison below keep clear of its ties, where fp32 and fp64 could part: no value of a cached
    reference is within 2^-20 of its size of one (fp32 sums of 64 products are off by 2^-24 a few
    times over)."""
    m = SMALL_F32
    rng = np.random.default_rng(1)
    x = rng.standard_normal((82, 64)) * np.exp(rng.standard_normal((82, 64)))
    got = reusevit.eight_bits(x, 2)
    c = np.arange(127)
    grid = np.where(c < 8, c * 2.0 ** -9, (8 + c % 8) * 2.0 ** (c // 8 - 10.0))
    for a in (0, 64):
        for h in (0, 32):
            y, z = x[a:a + 64, h:h + 32], got[a:a + 64, h:h + 32]
            s = 2.0 ** -60
            while np.abs(y).max() > 448 * s:
                s *= 2
            near = grid[np.abs(np.abs(y)[..., None] / s - grid).argmin(-1)] * s
            assert np.array_equal(np.abs(z), near) and np.array_equal(np.sign(z), np.sign(near * np.sign(y)))
    blob, fr, masks = cached_case(m, SEED)
    seen = []
    keep = reusevit.eight_bits

    def watch(rows, heads):
        out = keep(rows, heads)
        up, down = keep(rows * (1 + 2.0 ** -20), heads), keep(rows * (1 - 2.0 ** -20), heads)
        seen.append(np.array_equal(up, out) and np.array_equal(down, out))
        return out

    reusevit.eight_bits = watch
    try:
        oracle.encode(fr, blob, m.as_dict(), 4, masks=masks, cached8=CARRIED)
    finally:
        reusevit.eight_bits = keep
    assert seen and all(seen)


def streamed(m, blob, fr, masks, batch=8, cut=CUT):
    enc = encoder(m, blob, batch)
    outs, k = [], 0
    for c in cut:
        outs.append(enc.stream_encode(dev(fr[k:k + c]), 4, masks_in=dev(masks[k:k + c]), want_tokens=True))
        k += c
    require_gpu().cuda.synchronize()
    return [np.concatenate([host(o[j]) for o in outs]) for j in range(3)]


@gpu
@pytest.mark.parametrize("rotary", [False, True])
@pytest.mark.parametrize("m", [SMALL_F32, MID, H80], ids=["f32", "bf16", "dh80"])
def test_cached_reference_in_eight_bits(m, rotary):
    """Injected maps; frames that continue a group of an earlier call attend to the quantised keys and
    values.  fp32: within the parity bar of the oracle that quantises too, and outside it of the
    one that does not (without the turn: the seed keeps clear of ties there).  bf16: keys
    already carry 2^-8, which may move a value to the next code; the bar holds all the same."""
    m = dataclasses.replace(m, cache8=True, rotary=rotary)
    blob, fr, masks = cached_case(m, SEED)
    emb, _, toks = streamed(m, blob, fr, masks)
    if m.dtype == "bf16" or not rotary:
        r = oracle.encode(fr, blob, m.as_dict(), 4, masks=masks, cached8=CARRIED)
        check_close(emb, r["emb"], m.dtype, "embeddings")
        check_close(toks, r["tokens"], m.dtype, "tokens")
    if m.dtype == "f32":
        r = oracle.encode(fr, blob, m.as_dict(), 4, masks=masks)
        with pytest.raises(AssertionError):
            check_close(emb, r["emb"], "f32", "unquantised")
    # frames that find their reference in their own call are not affected, to the bit
    plain = streamed(dataclasses.replace(m, cache8=False), blob, fr, masks)
    for a, b in ((emb, plain[0]), (toks, plain[2])):
        assert np.array_equal(a[~CARRIED], b[~CARRIED]) and not np.array_equal(a[CARRIED], b[CARRIED])


@gpu
def test_cached_reference_takes_less_memory():
    """Per layer and reference 2 N D elements become as many bytes (in whole pages) and two scales a
    page and head."""
    import paper_2506_14107_amd.dejavu as dj
    for m in (SMALL_F32, MID, H80):
        size = [dj.dv_workspace_bytes(encoder(dataclasses.replace(m, cache8=c), synth.make_blob(m, 1), 8).handle)
                for c in (False, True)]
        el, pages = 2 if m.dtype == "bf16" else 4, -(-m.n_tokens // 64)
        was = m.depth * m.n_tokens * 2 * m.width * el
        now = m.depth * pages * 2 * (64 * m.width + 4 * m.heads)
        assert abs((size[0] - size[1]) - (was - now)) <= 4 * 256


@gpu
def test_cached_reference_under_reordering_and_restoration():
    """The other modes run with the 8-bit cache: calls that end on group boundaries give bitwise the plain
    cache's results, and so do, in calls that do not, all frames but those whose group's reference
    came in an earlier call."""
    for kw in (dict(reorder=True), dict(restore=True), dict(decision=True)):
        m = dataclasses.replace(MID, **kw)
        m8 = dataclasses.replace(m, cache8=True)
        blob = synth.make_blob(m, 75, perturb_ln=True)
        fr = frames(m, 17)
        tau = 0.0 if m.decision else 0.9
        outs = []
        for model in (m, m8):
            enc = encoder(model, blob, 16)
            whole = [enc.stream_encode(dev(fr[:16]), 8, tau)[0]]
            enc.stream_reset()
            cut = [enc.stream_encode(dev(fr[a:b]), 8, tau)[0] for a, b in ((0, 9), (9, 13), (13, 17))]
            cut.append(enc.stream_flush()[0])
            outs.append([np.concatenate([host(o) for o in part]) for part in (whole, cut)])
        assert np.array_equal(outs[0][0], outs[1][0])
        assert outs[1][1].shape[0] == 17 and np.isfinite(outs[1][1]).all()
        own = np.r_[0:9, 16]
        assert np.array_equal(outs[0][1][own], outs[1][1][own])
        assert not np.array_equal(outs[0][1], outs[1][1])
