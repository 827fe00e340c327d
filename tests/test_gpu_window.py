"""Attention with a window and first keys that stay visible, against plain 64-bit versions."""
import numpy as np
import pytest

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import ATTENTION, LARGE, close, filled, ints, normal, values
from .test_gpu_cache_edges import SIZES, store

pytestmark = pytest.mark.gpu


def seen(length, n, causal, window, sinks):
    """[rows, keys] that the n last rows of a sequence see."""
    e = (np.maximum(length - n + np.arange(n) + 1, 0) if causal else np.full(n, length))[:, None]
    j = np.arange(length)[None]
    return (j < e) & ((j < sinks) | (j >= e - window))


def spoil(p, table, lengths, counts, causal, window, sinks, rng):
    """Takes away pages that no row sees (some of them), and puts NaN in the places that none sees in the others.  Returns the
    table."""
    torch = require_gpu()
    table, pt = table.copy(), p.m.pt
    k, v = p.c.k.view(torch.uint8), p.c.v.view(torch.uint8)
    for s, (length, n) in enumerate(zip(lengths, counts)):
        used = seen(length, n, causal, window, sinks).any(0) if n else np.zeros(length, bool)
        for j in range(-(-length // pt)):
            here = used[j * pt:(j + 1) * pt]
            hidden = torch.from_numpy(np.flatnonzero(~here)).cuda()
            page = int(table[s, j])
            if not here.any() and rng.random() < 0.5:
                table[s, j] = rng.choice([-1, 1 << 30])
            elif len(hidden):
                k[page, :, hidden] = 0x7F
                v[page, :, :, hidden] = 0xFF
    return table


def window_case(heads, group, dh, pt, counts, lengths, pad, name, dtype, causal, window, sinks):
    rng = np.random.default_rng(11)
    p, table = filled(rng, heads, dh, pt, lengths)
    torn = spoil(p, table, lengths, counts, causal, window, sinks, rng)
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows = int(offs[-1]) + pad
    wide, wide64 = normal(rng, (rows, heads * group + 3, dh), dtype)
    q, q64 = wide[:, 2:-1], wide64[:, 2:-1]
    calls = [(ints(offs), most) for most in (0, max(counts))] + [(None, 0)] * all(c == 1 for c in counts)
    for o, most in calls:
        out = q.new_full((rows, heads * group, dh), 9.0)
        got = p.c.attention(q, ints(lengths), o, ints(torn), causal=causal, max_rows=most, out=out, window=window, sinks=sinks)
        assert got is out and (out[int(offs[-1]):] == 9.0).all()
        got = values(got)
        for s, length in enumerate(lengths):
            a, b = offs[s], offs[s + 1]
            if a == b:
                continue
            k, v, _ = p.m.history(table.tolist(), s, length)
            want, mass, size = ref.attention(q64[a:b], k, v, seen(length, b - a, causal, window, sinks), dh ** -0.5)
            tol = ref.attention_tolerance(want, mass, size, dtype, dh, max(1, min(length, window + sinks)))
            close(got[a:b], want, tol, f"{name} max_rows {most}, sequence {s}")


MORE = {
    "splits": (2, 4, 128, 64, [1] * 3, [20000, 9000, 1], 0),
    "one-long": (8, 1, 64, 128, [1], [30000], 0),
    "edges": (1, 2, 64, 64, [1] * 8, [126, 127, 128, 129, 130, 191, 192, 193], 0),
}
WINDOWS = [(1, 0), (1, 1), (5, 3), (64, 64), (63, 65), (130, 17), (40, 130)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ATTENTION)
def test_window(name, dtype, causal):
    i = sorted(ATTENTION).index(name)
    for window, sinks in (WINDOWS[i % 7], WINDOWS[(3 * i + 2 + causal) % 7]):
        window_case(*ATTENTION[name], name, dtype, causal, window, sinks)


@pytest.mark.parametrize("window,sinks", [(700, 130), (5000, 1000), (64, 0), (6000, 1 << 30), (1 << 31, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", MORE)
def test_window_over_long_sequences(name, dtype, window, sinks):
    window_case(*MORE[name], name, dtype, True, window, sinks)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", LARGE)
def test_window_large_tiles(name, causal):
    i = sorted(LARGE).index(name)
    window_case(*LARGE[name], name, "bf16", causal, *[(37, 5), (100, 70), (64, 0), (1, 64), (300, 1)][(i + causal) % 5])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", SIZES)
def test_every_key_counts_once(name, dtype):
    """Queries of zeros weigh the seen keys alike, and key j's value is 256 in channel j % dh, 0 elsewhere: one key lost or taken
    twice is more than 2^-7 of an output (as of attention without a window)."""
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths = SIZES[name]
    k64 = np.random.default_rng(3).standard_normal((sum(lengths), heads, dh))
    v64 = np.zeros((sum(lengths), heads, dh))
    for a, length in zip(np.cumsum([0] + lengths), lengths):
        for j in range(length):
            v64[a + j, :, j % dh] = 256
    p, table, _ = store(heads, dh, pt, lengths, k64, v64)
    offs = np.concatenate([[0], np.cumsum(counts)])
    q = torch.zeros(int(offs[-1]), heads * group, dh, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dtype], device="cuda")
    for window, sinks, causal in ((1, 0, True), (33, 7, True), (200, 64, True), (65, 300, False), (2000, 100, False)):
        got = values(p.c.attention(q, ints(lengths), ints(offs), ints(table), causal=causal, window=window, sinks=sinks))
        for s, (n, length) in enumerate(zip(counts, lengths)):
            sees = seen(length, n, causal, window, sinks)
            ch = (np.arange(length) % dh)[:, None] == np.arange(dh)[None]
            total = sees.sum(1)
            want = np.where(total[:, None] > 0, 256 * (sees @ ch.astype(float)) / np.maximum(total, 1)[:, None], 0.0)
            want = np.broadcast_to(want[:, None], (n, heads * group, dh))
            close(got[offs[s]:offs[s + 1]], want, want * (ref.HALF[dtype] + 4 * 2.0 ** -24), f"{name} {window} {sinks}, sequence {s}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", SIZES)
def test_a_window_that_holds_all_is_none(name, dtype):
    """Bit for bit, whatever the sinks."""
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths = SIZES[name]
    rng = np.random.default_rng(4)
    p, table = filled(rng, heads, dh, pt, lengths)
    offs = ints(np.concatenate([[0], np.cumsum(counts)]))
    q, _ = normal(rng, (sum(counts), heads * group, dh), dtype)
    want = p.c.attention(q, ints(lengths), offs, ints(table))
    for sinks in (0, 5, 1 << 30):
        assert torch.equal(p.c.attention(q, ints(lengths), offs, ints(table), window=1 << 30, sinks=sinks), want)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", SIZES)
def test_nan_and_infinite_values_reach_the_rows_that_see_them(name, dtype, causal):
    """A NaN, an infinity or both in values of the first, some middle and the last places."""
    heads, group, dh, pt, counts, lengths = SIZES[name]
    rng = np.random.default_rng(5)
    top = float(np.finfo(np.float32).max)
    first = np.cumsum([0] + lengths)[:-1]
    # (rounded to what the kernels get: the model would else take another code where a value is next to a border)
    k64, v64 = [rng.standard_normal((sum(lengths), heads, dh)).astype(np.float32).astype(np.float64) for _ in range(2)]
    at = {}
    for s, length in enumerate(lengths):
        at[s] = sorted({0, length // 3, length // 2, max(0, length - 9), length - 1})
        for i, j in enumerate(at[s]):
            v64[first[s] + j] = 0
            v64[first[s] + j, :, 3 + i] = top if i % 2 else -top
            v64[first[s] + j, :, 9] = np.nan
            v64[first[s] + j, :, 11] = top
    p, table, _ = store(heads, dh, pt, lengths, k64, v64)
    offs = np.concatenate([[0], np.cumsum(counts)])
    q, q64 = normal(rng, (int(offs[-1]), heads * group, dh), dtype)
    for window, sinks in ((4, 1), (70, 0), (30, 40)):
        got = values(p.c.attention(q, ints(lengths), ints(offs), ints(table), causal=causal, scale=0.02, window=window, sinks=sinks))
        for s, (n, length) in enumerate(zip(counts, lengths)):
            k, v, _ = p.m.history(table.tolist(), s, length)
            v = np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
            odd = ~np.isfinite(v)
            sees = seen(length, n, causal, window, sinks)
            part = got[offs[s]:offs[s + 1]].copy()
            some = [np.broadcast_to(((sees @ x.any(1).astype(float)) > 0)[:, None], part.shape) for x in
                    (v == np.inf, v == -np.inf, np.isnan(v))]
            want, mass, size = ref.attention(q64[offs[s]:offs[s + 1]], k, np.where(odd, 0.0, v), sees, 0.02)
            tol = ref.attention_tolerance(want, mass, size, dtype, dh, length)
            want = np.where(some[0], np.inf, np.where(some[1], -np.inf, want))
            want = np.where(some[2] | (some[0] & some[1]), np.nan, want)
            assert np.array_equal(np.isnan(part), np.isnan(want)), (name, s, window)
            far = np.isinf(want)
            assert np.array_equal(part[far], want[far])
            ok = np.isfinite(want)
            close(np.where(ok, part, 0), np.where(ok, want, 0), np.where(ok, tol, 1), f"{name} {window}, sequence {s}")


@pytest.mark.parametrize("name", ["prompt-mixed", "long"])
def test_rows_before_the_first_sequence_are_left_alone(name):
    torch = require_gpu()
    for heads, group, dh, pt, counts, lengths, _ in (ATTENTION[name], LARGE["mixed-128"]):
        rng = np.random.default_rng(27)
        p, table = filled(rng, heads, dh, pt, lengths)
        offs = 5 + np.concatenate([[0], np.cumsum(counts)])
        q, q64 = normal(rng, (int(offs[-1]) + 2, heads * group, dh), "bf16")
        out = torch.full_like(q, 9)
        p.c.attention(q, ints(lengths), ints(offs), ints(table), out=out, window=70, sinks=3)
        assert (out[:5] == 9).all() and (out[-2:] == 9).all()
        got = values(out)
        for s, length in enumerate(lengths):
            a, b = offs[s], offs[s + 1]
            if a == b:
                continue
            k, v, _ = p.m.history(table.tolist(), s, length)
            want, mass, size = ref.attention(q64[a:b], k, v, seen(length, b - a, True, 70, 3), dh ** -0.5)
            close(got[a:b], want, ref.attention_tolerance(want, mass, size, "bf16", dh, max(1, min(length, 73))), f"{name}, sequence {s}")


@pytest.mark.parametrize("name", ["prompt-mixed", "long"])
def test_in_place_on_a_stream_and_with_a_workspace(name):
    torch = require_gpu()
    for heads, group, dh, pt, counts, lengths, _ in (ATTENTION[name], LARGE["mixed-128"], MORE["splits"]):
        rng = np.random.default_rng(22)
        p, table = filled(rng, heads, dh, pt, lengths)
        q, _ = normal(rng, (sum(counts), heads * group, dh), "bf16")
        offs = ints(np.concatenate([[0], np.cumsum(counts)]))
        kw = dict(window=4000, sinks=3)
        want = p.c.attention(q, ints(lengths), offs, ints(table), **kw)
        need = p.c.attention_workspace(len(counts), sum(counts), heads * group, table.shape[1], **kw)
        ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        got = p.c.attention(q, ints(lengths), offs, ints(table), workspace=ws[:need], stream=side, out=q, **kw)
        side.synchronize()
        assert got is q and torch.equal(q, want) and (ws[need:] == 255).all()


def test_captured_steps_replay():
    """A graph of a step of streams whose windows move on: replayed with growing lengths, each equals the eager call."""
    torch = require_gpu()
    heads, group, dh, pt = 2, 4, 128, 64
    rng = np.random.default_rng(16)
    p, table = filled(rng, heads, dh, pt, [6000, 300, 4000])
    t, lengths = ints(table), ints([5000, 200, 3000])
    q = torch.randn(3, heads * group, dh, device="cuda").bfloat16()
    kw = dict(window=1500, sinks=257)
    p.c.attention(q, lengths, None, t, **kw)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = p.c.attention(q, lengths, None, t, **kw)
    for _ in range(5):
        lengths += 19
        q.copy_(torch.randn(q.shape, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, p.c.attention(q, lengths, None, t, **kw))
        torch.randn(1 << 16, device="cuda").sum().item()
