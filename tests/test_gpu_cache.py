"""Rotary positions, the 8-bit cache and attention over it on the GPU, against plain 64-bit versions
(cache_ref.py, which derives the tolerances)."""
import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from . import cache_ref as ref
from .gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def types(torch):
    return {"bf16": torch.bfloat16, "f32": torch.float32}


def normal(rng, shape, dtype, size=1.0):
    """(tensor, its values in 64 bits)."""
    torch = require_gpu()
    t = torch.from_numpy((rng.standard_normal(shape) * size).astype(np.float32)).to(types(torch)[dtype])
    return t.cuda(), t.double().numpy()


def ints(a):
    torch = require_gpu()
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def values(t):
    return t.detach().double().cpu().numpy()


def close(got, want, tol, what):
    got = values(got) if hasattr(got, "detach") else got
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    d = np.abs(got - want)
    bad = d > tol
    assert not np.any(bad), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.nanmax(d / (tol + 1e-300)):.3g} of " \
        f"the tolerance at {np.argwhere(bad)[0]}"


# ---- rotary positions ----------------------------------------------------------------------------
ROTARY = {
    # rows, heads, dh, sections, layout, per_axis, base, far, row padding, first element
    "frames": (257, 24, 64, (8, 12, 12), "halves", False, 1e4, 600, 0, 0),
    "pairs": (33, 3, 128, (24, 20, 20), "pairs", True, 100.0, 60000, 64, 0),
    "part": (7, 5, 96, (8, 8, 8), "halves", False, 5e5, 60000, 16, 8),
    "part-pairs": (7, 5, 80, (0, 3, 5), "pairs", False, 1e4, 1000, 0, 0),
    "odd-section": (5, 2, 48, (5, 3, 3), "halves", True, 1e4, 1000, 0, 0),
    "unaligned": (9, 2, 64, (8, 12, 12), "halves", False, 1e4, 1000, 1, 1),
    "narrow": (1, 1, 6, (1, 0, 1), "pairs", False, 1e4, 1000, 3, 3),
    "far": (64, 2, 64, (8, 12, 12), "halves", False, 1e4, 1 << 30, 0, 0),
    "wide-head": (3, 2, 200, (20, 20, 24), "halves", False, 1e4, 1000, 0, 0),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ROTARY)
def test_rotary(name, dtype):
    torch = require_gpu()
    rows, heads, dh, sec, layout, per_axis, base, far, pad, first = ROTARY[name]
    rng = np.random.default_rng(3)
    flat, flat64 = normal(rng, first + rows * (heads * dh + pad), dtype)
    shape, st = (rows, heads, dh), (heads * dh + pad, dh, 1)
    x = flat.as_strided(shape, st, first)
    x64 = np.lib.stride_tricks.as_strided(flat64[first:], shape, [8 * s for s in st])
    pos = rng.integers(-far, far, (rows, 3))
    rot = dj.Rotary(sec, layout, per_axis, base)
    want, size = ref.turn(x64, pos, sec, layout, per_axis, base)
    tol = ref.turn_tolerance(want, size, dtype, far)
    before = flat.clone()
    got = dj.rotary(x, ints(pos), rot)
    close(got, want, tol, "new tensor")
    if 2 * sum(sec) < dh:
        assert torch.equal(got[..., 2 * sum(sec):], x[..., 2 * sum(sec):])
    assert torch.equal(flat, before)
    assert dj.rotary(x, ints(pos), rot, out=x) is x
    assert torch.equal(x, got)
    outside = torch.ones_like(flat, dtype=torch.bool)
    outside.as_strided(shape, st, first)[:] = False
    assert torch.equal(flat[outside], before[outside])


def test_rotary_is_undone_by_negated_positions():
    """The transpose of the turn, which is its gradient: <turn(x), y> = <x, turn back(y)>."""
    rng = np.random.default_rng(4)
    x, x64 = normal(rng, (40, 3, 64), "f32")
    pos = rng.integers(-100000, 100000, (40, 3))
    rot = dj.Rotary((8, 12, 12))
    y = dj.rotary(x, ints(pos), rot)
    back = dj.rotary(y, ints(-pos), rot)
    _, size = ref.turn(x64, pos, (8, 12, 12))
    _, size2 = ref.turn(values(y), pos, (8, 12, 12))
    close(back, x64, ref.TURN * 2 * (size + size2), "undone")


def test_rotary_one_row_and_none():
    torch = require_gpu()
    rot = dj.Rotary((4, 2, 2))
    x = torch.randn(0, 2, 16, device="cuda")
    assert dj.rotary(x, ints(np.zeros((0, 3))), rot).shape == (0, 2, 16)
    x = torch.randn(1, 1, 16, device="cuda")
    assert torch.equal(dj.rotary(x, ints(np.zeros((1, 3))), rot), x)


# ---- write and read ------------------------------------------------------------------------------
class Pair:
    """A cache on the GPU over pages full of arbitrary bytes, and its 64-bit model."""

    def __init__(self, pages, heads, dh, pt, seed=0):
        torch = require_gpu()
        rng = np.random.default_rng(seed)
        self.c = dj.TokenCache(pages, heads, dh, pt)
        for t in (self.c.k, self.c.v):
            t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 256, t.shape, dtype=np.uint8)))
        self.c.k_scale.fill_(float("nan"))
        self.c.v_scale.fill_(float("nan"))
        self.m = ref.Cache(pages, heads, pt, dh)

    def bytes(self):
        torch = require_gpu()
        torch.cuda.synchronize()
        return [t.view(torch.uint8).cpu().numpy().copy() for t in (self.c.k, self.c.v)]

    def decoded(self):
        """Keys and values as they stand, token first."""
        k, v = self.bytes()
        lut = ref.codes_table()
        return [lut[k] * values(self.c.k_scale)[:, :, None, None],
                lut[v.transpose(0, 1, 3, 2)] * values(self.c.v_scale)[:, :, None, None]]


def table_of(rng, n, tp, pages):
    return rng.permutation(pages)[:n * tp].reshape(n, tp)


def live(table, lengths, pt, pages):
    """[pages, pt] places that sequences of these lengths hold."""
    m = np.zeros((pages, pt), bool)
    for s, n in enumerate(lengths):
        for p in range(n):
            if p // pt < table.shape[1] and 0 <= table[s][p // pt] < pages:
                m[table[s][p // pt], p % pt] = True
    return m


WRITE = {
    # heads, dh, page, counts, starts, padding rows
    "one": (1, 16, 16, [1], [0], 0),
    "short-pages": (3, 80, 16, [5, 0, 33, 16], [0, 4, 32, 0], 3),
    "reference": (12, 64, 64, [257], [0], 0),
    "wide": (8, 128, 64, [64, 65, 1, 0, 130], [0, 64, 0, 0, 0], 0),
    "long-pages": (2, 128, 128, [300, 127], [0, 128], 1),
    "long-pages-112": (2, 112, 128, [130, 1], [0, 0], 0),
    "48": (2, 48, 32, [70, 31], [0, 32], 0),
    "many": (1, 32, 16, [1, 2, 3] * 50, [0] * 150, 5),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", WRITE)
def test_write_and_read_whole_pages(name, dtype):
    """Writes that start pages: codes and scales are the model's exactly (their arithmetic is exact but
    for the rounding to e4m3), nothing else changes, and reads give what the codes stand for."""
    torch = require_gpu()
    heads, dh, pt, counts, starts, pad = WRITE[name]
    rng = np.random.default_rng(5)
    n, tp = len(counts), max(-(-(a + c) // pt) for a, c in zip(starts, counts)) or 1
    pages = n * tp + 2
    p = Pair(pages, heads, dh, pt)
    table = table_of(rng, n, tp, pages)
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows = int(offs[-1]) + pad
    k, k64 = normal(rng, (rows, heads, dh), dtype)
    both, both64 = normal(rng, (rows, 2 * heads + 1, dh), dtype, 40.0)     # values inside wider rows
    v, v64 = both[:, 1:heads + 1], both64[:, 1:heads + 1]
    before = p.bytes()
    p.c.write(k, v, ints(starts), ints(offs), ints(table))
    p.m.write(table.tolist(), offs, starts, k64, v64)
    lengths = [a + c for a, c in zip(starts, counts)]
    wrote = live(table, lengths, pt, pages) & ~live(table, starts, pt, pages)
    touched = wrote.any(1)
    got = p.decoded()
    for w, sc in enumerate((p.c.k_scale, p.c.v_scale)):
        assert np.array_equal(values(sc)[touched], p.m.scale[w][touched])
        assert np.isnan(values(sc)[~touched]).all()
        m = np.broadcast_to(wrote[:, None, :, None], got[w].shape)
        assert np.array_equal(got[w][m], p.m.x[w][m])
    after = p.bytes()
    rest = ~np.broadcast_to(wrote[:, None, :, None], before[0].shape)
    assert np.array_equal(after[0][rest], before[0][rest])
    rest = rest.transpose(0, 1, 3, 2)
    assert np.array_equal(after[1][rest], before[1][rest])

    for out_dtype in ("f32", "bf16"):
        wide = torch.full((rows, 2 * heads, dh), 7.0, dtype=types(torch)[out_dtype], device="cuda")
        p.c.read(ints(starts), ints(offs), ints(table), out=(wide[:, heads:], wide[:, :heads]))
        for w, part in ((0, wide[:, heads:]), (1, wide[:, :heads])):
            want = np.full((rows, heads, dh), 7.0)
            for s in range(n):
                for i in range(counts[s]):
                    q = starts[s] + i
                    want[offs[s] + i] = p.m.x[w][table[s][q // pt], :, q % pt]
            assert np.array_equal(values(part), want)      # e4m3 times a power of two: exact in bf16


@pytest.mark.parametrize("pt,dh", [(16, 64), (64, 128), (32, 80), (128, 16)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_appends_grow_the_scale(dtype, pt, dh):
    """Calls of different lengths fill pages; later tokens are larger or smaller.  Codes and scales
    are the model's exactly, and every value is near what was written: half a step, and below 2^-6 of
    the scale half of 2^-9 of it for each growth (at most 2^-9 in all, each scale being at least twice
    the one before)."""
    rng = np.random.default_rng(6)
    heads, n = 3, 4
    total = 2 * pt + 9
    tp = -(-total // pt)
    p = Pair(n * tp, heads, dh, pt)
    table = table_of(rng, n, tp, n * tp)
    done = np.zeros(n, int)
    wrote = [np.zeros((n, total, heads, dh)) for _ in range(2)]
    step = 0
    while done.min() < total:
        counts = np.minimum(rng.integers(0, 2 + step % 3 * pt // 2, n), total - done)
        offs = np.concatenate([[0], np.cumsum(counts)])
        step += 1
        if offs[-1] == 0:
            continue
        rows = int(offs[-1])
        size = np.exp2(rng.integers(-12, 13))
        k, k64 = normal(rng, (rows, heads, dh), dtype, size)
        v, v64 = normal(rng, (rows, heads, dh), dtype, 1 / size)
        p.c.write(k, v, ints(done), ints(offs), ints(table))
        p.m.write(table.tolist(), offs, done.tolist(), k64, v64)
        for s in range(n):
            for w, x in enumerate((k64, v64)):
                wrote[w][s, done[s]:done[s] + counts[s]] = x[offs[s]:offs[s + 1]]
        done += counts
    held = live(table, done, pt, n * tp)
    got = p.decoded()
    for w, sc in enumerate((p.c.k_scale, p.c.v_scale)):
        assert np.array_equal(values(sc), p.m.scale[w])
        m = np.broadcast_to(held[:, None, :, None], got[w].shape)
        assert np.array_equal(got[w][m], p.m.x[w][m])
        for s in range(n):
            for q in range(total):
                page = table[s][q // pt]
                x, z = wrote[w][s, q], values(sc)[page][:, None]
                close(got[w][page, :, q % pt], x, 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * z, "value")


def test_write_turns_keys_and_queries():
    """Keys are quantised from their turned values in fp32: within the turn's error of the 64-bit
    ones before a rounding of half a step of e4m3, at a scale of a magnitude that close."""
    for dtype in ("f32", "bf16"):
        for sec, layout, qh in (((8, 12, 12), "halves", 8), ((4, 4, 2), "pairs", 2), ((3, 2, 2), "halves", 5)):
            rng = np.random.default_rng(7)
            heads, dh, pt, n = 2, 64, 32, 3
            counts, starts = [40, 1, 7], [0, 5, 0]
            offs = np.concatenate([[0], np.cumsum(counts)])
            rows = int(offs[-1]) + 2
            table = table_of(rng, n, 3, 9)
            p = Pair(9, heads, dh, pt)
            k, k64 = normal(rng, (rows, heads, dh), dtype)
            v, v64 = normal(rng, (rows, heads, dh), dtype)
            q, q64 = normal(rng, (rows, qh, dh), dtype)
            zero = [normal(rng, (5, heads, dh), dtype) for _ in range(2)]
            p.c.write(zero[0][0], zero[1][0], ints([0]), ints([0, 5]), ints(table[1:2]))
            p.m.write(table[1:2].tolist(), [0, 5], [0], zero[0][1], zero[1][1])
            pos = rng.integers(0, 5000, (rows, 3))
            q_out = q.new_full(q.shape, 3.0)
            got_q = p.c.write(k, v, ints(starts), ints(offs), ints(table), dj.Rotary(sec, layout),
                              ints(pos), q, q_out)
            assert got_q is q_out
            want, size = ref.turn(q64, pos, sec, layout)
            live_rows = int(offs[-1])
            close(q_out[:live_rows], want[:live_rows], ref.turn_tolerance(want, size, dtype, 5000)[:live_rows], "q")
            assert (q_out[live_rows:] == 3.0).all()
            want, size = ref.turn(k64, pos, sec, layout)
            err = ref.turn_tolerance(want, size, "f32", 5000)
            got = p.decoded()
            for s in range(n):
                for i in range(counts[s]):
                    at, row = starts[s] + i, offs[s] + i
                    page = table[s][at // pt]
                    z = values(p.c.k_scale)[page][:, None]
                    x = want[row]
                    close(got[0][page, :, at % pt], x,
                          err[row] + np.maximum(2.0 ** -4 * (np.abs(x) + err[row]), 2.0 ** -10 * z), "k")
                    assert np.array_equal(got[1][page, :, at % pt], ref.e4m3(
                        v64[row] / values(p.c.v_scale)[page][:, None]) * values(p.c.v_scale)[page][:, None])
            p.m.write(table.tolist(), offs, starts, want, v64)
            assert np.array_equal(values(p.c.v_scale)[np.unique(table[0, :2])], p.m.scale[1][np.unique(table[0, :2])])
            for page in (table[0][0], table[0][1], table[1][0], table[2][0]):
                near = [p.m.scale[0][page] * f for f in (0.5, 1.0, 2.0)]
                z = values(p.c.k_scale)[page]
                assert all(z[h] in (near[0][h], near[1][h], near[2][h]) for h in range(heads))


@pytest.mark.parametrize("first", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write_turns_whole_heads_on_long_pages(dtype, first):
    """All of 128 channels turned on pages of 128 tokens (the most angles a block holds), with rows that
    start on 16 bytes and rows that do not."""
    rng = np.random.default_rng(19)
    heads, dh, pt, rows, sec = 2, 128, 128, 200, (24, 20, 20)
    p = Pair(2, heads, dh, pt)
    flat, flat64 = normal(rng, first + 2 * rows * heads * dh, dtype)
    k, v = flat[first:].view(2, rows, heads, dh)
    k64, v64 = flat64[first:].reshape(2, rows, heads, dh)
    q, q64 = normal(rng, (rows, 3, dh), dtype)
    pos = rng.integers(0, 5000, (rows, 3))
    q_out = p.c.write(k, v, ints([0]), ints([0, rows]), None, dj.Rotary(sec), ints(pos), q)
    want, size = ref.turn(q64, pos, sec)
    close(q_out, want, ref.turn_tolerance(want, size, dtype, 5000), "q")
    want, size = ref.turn(k64, pos, sec)
    err = ref.turn_tolerance(want, size, "f32", 5000)
    got, z = p.decoded(), values(p.c.k_scale)
    for i in range(rows):
        x, zi = want[i], z[i // pt][:, None]
        close(got[0][i // pt, :, i % pt], x, err[i] + np.maximum(2.0 ** -4 * (np.abs(x) + err[i]), 2.0 ** -10 * zi), "k")
    p.m.write([[0, 1]], [0, rows], [0], k64, v64)
    assert np.array_equal(values(p.c.v_scale), p.m.scale[1])
    assert np.array_equal(got[1][0], p.m.x[1][0]) and np.array_equal(got[1][1, :, :rows - pt], p.m.x[1][1, :, :rows - pt])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_start_on_odd_elements(dtype):
    """Rows off 16 bytes, an odd number of elements apart, write the same codes, scales and queries, read the
    same values and attend alike."""
    torch = require_gpu()
    heads, dh, pt, rows = 3, 80, 32, 70
    rng = np.random.default_rng(20)
    whole = [normal(rng, (rows, h, dh), dtype)[0] for h in (heads, heads, 2 * heads)]

    def odd(x):
        flat = torch.zeros(1 + rows * (x[0].numel() + 1), dtype=x.dtype, device="cuda")
        y = flat.as_strided(x.shape, (x[0].numel() + 1, dh, 1), 1)
        y.copy_(x)
        return y

    offs, table, rot = ints([0, 30, 70]), ints([[4, 1], [0, 3]]), dj.Rotary((8, 8, 8))
    pos, starts, lengths = ints(rng.integers(0, 5000, (rows, 3))), ints([0, 0]), ints([30, 40])
    got = []
    for move in (lambda x: x, odd):
        p = Pair(5, heads, dh, pt)
        k, v, q = [move(x) for x in whole]
        q_out = move(torch.zeros_like(whole[2]))
        p.c.write(k, v, starts, offs, table, rot, pos, q, q_out)
        rows_out = [move(torch.zeros_like(x)) for x in whole[:2]]
        p.c.read(starts, offs, table, out=rows_out)
        got.append([p.bytes(), p.c.k_scale, p.c.v_scale, q_out, *rows_out,
                    p.c.attention(q_out, lengths, offs, table)])
    for a, b in zip(got[0][0], got[1][0]):
        assert np.array_equal(a, b)
    for a, b in zip(got[0][1:], got[1][1:]):
        assert np.array_equal(values(a), values(b), equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_before_the_first_sequence_are_left_alone(dtype):
    torch = require_gpu()
    heads, dh, pt, lead, n = 2, 64, 16, 5, 20
    rng = np.random.default_rng(21)
    rows = lead + n + 2
    k, v = [normal(rng, (rows, heads, dh), dtype)[0] for _ in range(2)]
    q, _ = normal(rng, (rows, 2 * heads, dh), dtype)
    rot, pos = dj.Rotary((8, 12, 12)), ints(rng.integers(0, 500, (rows, 3)))
    starts, lengths = ints([0, 0]), ints([13, 7])
    got = []
    for a, b, offs in ((0, rows, [lead, lead + 13, lead + n]), (lead, lead + n, [0, 13, n])):
        p = Pair(4, heads, dh, pt)
        q_out = torch.full_like(q, 3.0)
        p.c.write(k[a:b], v[a:b], starts, ints(offs), None, rot, pos[a:b], q[a:b], q_out[a:b])
        out = [torch.full_like(x, 5.0) for x in (k, v, q)]
        p.c.read(starts, ints(offs), out=(out[0][a:b], out[1][a:b]))
        p.c.attention(q_out[a:b], lengths, ints(offs), out=out[2][a:b])
        for x, fill in ((q_out, 3.0), (out[0], 5.0), (out[1], 5.0), (out[2], 5.0)):
            assert (x[:lead] == fill).all() and (x[lead + n:] == fill).all()
        got.append([p.c.k, p.c.v, q_out, *out])
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*got))


def test_the_smallest_scale():
    """All codes at 2^-126 and 2^-120: fp32 holds code times scale exactly, bf16 where it is no smaller than
    2^-126; below that it may be off by its step there, 2^-133."""
    torch = require_gpu()
    c = dj.TokenCache(2, 1, 128, 16)
    for t in (c.k, c.v):
        t.view(torch.uint8).copy_(torch.from_numpy(np.resize(np.arange(256), t.shape).astype(np.uint8)))
    for s in (c.k_scale, c.v_scale):
        s.copy_(torch.tensor([[2.0 ** -126], [2.0 ** -120]]))
    lut = ref.codes_table()
    want = [lut[t.view(torch.uint8).cpu().numpy()] * values(s)[:, :, None, None]
            for t, s in ((c.k, c.k_scale), (c.v, c.v_scale))]
    want[1] = want[1].transpose(0, 1, 3, 2)
    for dtype, tol in (("f32", 0.0), ("bf16", 2.0 ** -133)):
        for w, got in enumerate(c.read(ints([0, 0]), ints([0, 16, 32]), rows=32, dtype=types(torch)[dtype])):
            x = want[w].transpose(0, 2, 1, 3).reshape(32, 1, 128)
            close(got, x, np.where(np.abs(x) < 2.0 ** -126, tol, 0.0), dtype)


def test_write_keeps_nan_and_ignores_it_for_the_scale():
    torch = require_gpu()
    heads, dh, pt = 2, 32, 16
    rng = np.random.default_rng(8)
    p = Pair(2, heads, dh, pt)
    k, k64 = normal(rng, (20, heads, dh), "f32")
    v, v64 = normal(rng, (20, heads, dh), "bf16")
    v, v64 = v.float(), v64.copy()
    for t, x in ((k, k64), (v, v64)):
        for row, ch, bad in ((3, 5, np.nan), (4, 0, np.inf), (19, 31, -np.inf)):
            t[row, 1, ch] = float(bad)
            x[row, 1, ch] = np.nan
    v[6], v64[6] = 0.0, 0.0
    p.c.write(k, v, ints([0]), ints([0, 20]))
    p.m.write([[0, 1]], [0, 20], [0], k64, v64)
    got = p.decoded()
    for w, sc in enumerate((p.c.k_scale, p.c.v_scale)):
        assert np.array_equal(values(sc), p.m.scale[w])
        flat = [got[w][0].transpose(1, 0, 2), got[w][1].transpose(1, 0, 2)[:4]]
        assert np.array_equal(np.concatenate(flat), np.concatenate(
            [p.m.x[w][0].transpose(1, 0, 2), p.m.x[w][1].transpose(1, 0, 2)[:4]]), equal_nan=True)
    # a page of zeros, and one of the smallest magnitudes
    tiny = torch.full((1, heads, dh), 1e-44, device="cuda")
    p.c.write(torch.zeros_like(tiny), tiny, ints([0]), ints([0, 1]))
    assert (values(p.c.k_scale)[0] == 2.0 ** -126).all() and (values(p.c.v_scale)[0] == 2.0 ** -126).all()
    assert (p.decoded()[0][0, :, 0] == 0).all()
    # the largest fp32 values
    huge = torch.full((1, heads, dh), torch.finfo(torch.float32).max, device="cuda")
    p.c.write(huge, -huge, ints([0]), ints([0, 1]))
    assert (values(p.c.k_scale)[0] == 2.0 ** 120).all()
    assert (p.decoded()[1][0, :, 0] == -(2.0 ** 128)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_that_are_not_there(dtype):
    """Rows for pages outside the cache, past the table or of a negative start are dropped; nothing
    else changes; they read as zeros (rows of a negative start stay as they were)."""
    torch = require_gpu()
    heads, dh, pt, pages = 2, 48, 16, 5
    rng = np.random.default_rng(9)
    p = Pair(pages, heads, dh, pt)
    table = np.array([[0, -1, 2], [pages, 1 << 30, 3], [-(1 << 31), 4, 1]])
    counts, starts = [60, 40, 8], [0, 3, -2]
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows = int(offs[-1])
    k, k64 = normal(rng, (rows, heads, dh), dtype)
    v, v64 = normal(rng, (rows, heads, dh), dtype)
    before = p.bytes()
    p.c.write(k, v, ints(starts), ints(offs), ints(table))
    p.m.write(table.tolist(), offs, starts, k64, v64)
    after, got = p.bytes(), p.decoded()
    for w in range(2):
        for page in (1, 4):
            assert np.array_equal(after[w][page], before[w][page])
        for page in (0, 2):
            assert np.array_equal(got[w][page], p.m.x[w][page])
        assert np.array_equal(got[w][3, :, :43 - 32], p.m.x[w][3, :, :43 - 32])
    out = [torch.full((rows, heads, dh), 5.0, device="cuda") for _ in range(2)]
    p.c.read(ints(starts), ints(offs), ints(table), out=out)
    for w in range(2):
        want = np.zeros((rows, heads, dh))
        want[offs[2]:] = 5.0
        for s in range(2):
            for i in range(counts[s]):
                q = starts[s] + i
                page = p.m.page(table.tolist(), s, q)
                if page >= 0:
                    want[offs[s] + i] = p.m.x[w][page, :, q % pt]
        assert np.array_equal(values(out[w]), want)


def test_one_row_each_without_offsets():
    """The form for single tokens: no offsets, a table or none."""
    heads, dh, pt, n = 4, 64, 16, 70
    rng = np.random.default_rng(10)
    for table in (None, table_of(rng, n, 2, 2 * n)):
        p = Pair(2 * n, heads, dh, pt)
        plain = np.arange(2 * n).reshape(n, 2) if table is None else table
        t = None if table is None else ints(table)
        for at in range(3):
            starts = [15 * (s % 2) + at for s in range(n)]
            k, k64 = normal(rng, (n, heads, dh), "bf16", at + 1.0)
            v, v64 = normal(rng, (n, heads, dh), "bf16")
            if at == 0:      # odd sequences: places before the first token of the test
                k0, k064 = normal(rng, (15 * n, heads, dh), "bf16")
                offs = np.cumsum([0] + [15 * (s % 2) for s in range(n)])
                p.c.write(k0[:offs[-1]], k0[:offs[-1]], ints([0] * n), ints(offs), t)
                p.m.write(plain.tolist(), offs, [0] * n, k064, k064)
            p.c.write(k, v, ints(starts), None, t)
            p.m.write(plain.tolist(), np.arange(n + 1), starts, k64, v64)
        out = p.c.read(ints(starts), None, t)
        for w in range(2):
            want = np.stack([p.m.x[w][plain[s][starts[s] // pt], :, starts[s] % pt] for s in range(n)])
            assert np.array_equal(values(out[w]), want)


# ---- attention -----------------------------------------------------------------------------------
def filled(rng, heads, dh, pt, lengths, extra=3, size=1.0):
    """A cache holding sequences of these lengths in scattered pages (in pages full of arbitrary bytes),
    its model, and the table."""
    n = len(lengths)
    tp = max(1, max(-(-x // pt) for x in lengths))
    p = Pair(n * tp + extra, heads, dh, pt, seed=int(rng.integers(1 << 30)))
    table = table_of(rng, n, tp, n * tp + extra)
    offs = np.concatenate([[0], np.cumsum(lengths)])
    if offs[-1]:
        k, k64 = normal(rng, (int(offs[-1]), heads, dh), "f32", size)
        v, v64 = normal(rng, (int(offs[-1]), heads, dh), "f32")
        p.c.write(k, v, ints([0] * n), ints(offs), ints(table))
        p.m.write(table.tolist(), offs, [0] * n, k64, v64)
    return p, table


def check_attention(p, table, q, q64, lengths, offs, causal, dtype, got, what, scale=None):
    dh = q64.shape[2]
    scale = dh ** -0.5 if scale is None else scale
    got = values(got)
    for s, length in enumerate(lengths):
        length = max(0, min(length, table.shape[1] * p.m.pt))
        a, b = offs[s], offs[s + 1]
        if a == b:
            continue
        k, v, there = p.m.history(table.tolist(), s, length)
        sees = np.broadcast_to(there, (b - a, length)).copy()
        if causal:
            sees &= np.arange(length)[None] <= (length - (b - a) + np.arange(b - a))[:, None]
        out, mass, size = ref.attention(q64[a:b], k, v, sees, scale)
        tol = ref.attention_tolerance(out, mass, size, dtype, dh, max(length, 1))
        close(got[a:b], out, tol, f"{what}, sequence {s}")


ATTENTION = {
    # kv heads, group, dh, page, rows of each sequence, lengths, padding rows
    "token": (2, 1, 64, 64, [1], [257], 0),
    "one-key": (1, 1, 16, 16, [1, 1], [1, 2], 0),
    "tokens": (2, 4, 128, 64, [1] * 5, [1, 63, 64, 65, 700], 0),
    "empty": (2, 2, 32, 16, [3, 2, 0, 1], [0, 1, 40, 5], 2),
    "more-rows-than-keys": (1, 4, 64, 16, [9, 40], [4, 39], 1),
    "group-16": (1, 16, 64, 32, [2, 1], [100, 31], 0),
    "group-20": (2, 20, 48, 32, [3, 1], [70, 130], 0),
    "group-5": (3, 5, 80, 16, [7, 1, 20], [90, 17, 64], 3),
    "96": (2, 3, 96, 128, [4, 6], [300, 129], 0),
    "112": (1, 2, 112, 64, [17], [200], 0),
    "long": (1, 4, 128, 64, [2, 1], [3001, 2100], 0),
    "prompt": (2, 2, 64, 64, [130, 70], [200, 70], 0),
    "prompt-128": (1, 4, 128, 32, [150], [333], 4),
    "prompt-mixed": (2, 4, 80, 16, [1, 140, 2, 0, 33], [400, 140, 90, 10, 500], 0),
}
# bf16 batches that take large tiles: all of them, or (with several lengths) the longer sequences
LARGE = {
    "one": (56, 4, 64, 64, [141], [300], 3),
    "page-128": (34, 2, 128, 128, [250], [250], 0),
    "page-16": (54, 1, 80, 16, [460], [463], 0),
    "32": (96, 1, 32, 32, [350], [400], 1),
    "16": (122, 1, 16, 64, [257], [1100], 0),
    "48": (122, 1, 48, 64, [257], [64], 0),
    "96": (62, 2, 96, 16, [129], [150], 0),
    "112": (66, 1, 112, 128, [241], [300], 0),
    "group-20": (8, 20, 64, 64, [210], [700], 0),
    "alike": (52, 2, 64, 64, [100, 100, 100], [100, 400, 1], 2),
    "mixed": (46, 4, 64, 32, [1, 120, 17, 0, 16, 3], [900, 130, 17, 4, 600, 2], 0),
    "mixed-128": (14, 4, 128, 64, [20, 1, 260, 2], [40, 3000, 260, 0], 0),
    "split": (7, 8, 128, 64, [300], [1200], 0),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", LARGE)
def test_attention_large_tiles(name, causal):
    attention_case(*LARGE[name], name, "bf16", causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ATTENTION)
def test_attention(name, dtype, causal):
    attention_case(*ATTENTION[name], name, dtype, causal)


def attention_case(heads, group, dh, pt, counts, lengths, pad, name, dtype, causal):
    rng = np.random.default_rng(11)
    p, table = filled(rng, heads, dh, pt, lengths)
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows = int(offs[-1]) + pad
    wide, wide64 = normal(rng, (rows, heads * group + 3, dh), dtype)
    q, q64 = wide[:, 2:-1], wide64[:, 2:-1]
    for most in (0, max(counts)):
        out = q.new_full((rows, heads * group, dh), 9.0)
        got = p.c.attention(q, ints(lengths), ints(offs), ints(table), causal=causal, max_rows=most, out=out)
        assert got is out
        check_attention(p, table, q, q64, lengths, offs, causal, dtype, got, f"{name} max_rows {most}")
        assert (out[int(offs[-1]):] == 9.0).all()
    if all(c == 1 for c in counts):
        got = p.c.attention(q, ints(lengths), None, ints(table), causal=causal)
        check_attention(p, table, q, q64, lengths, offs, causal, dtype, got, f"{name} without offsets")


@pytest.mark.parametrize("dtype,rows,heads", [("f32", 1, 2), ("bf16", 1, 2), ("f32", 40, 2), ("bf16", 40, 2),
                                              ("bf16", 80, 64)])
def test_attention_extremes(rows, dtype, heads):
    """Scores far apart and a scale of the caller's; missing pages; lengths past the table and below zero;
    NaN and infinities among keys and values that a row does not see."""
    group, dh, pt, length = 2, 64, 16, 150
    rng = np.random.default_rng(12)
    p, table = filled(rng, heads, dh, pt, [length] * 3, size=20.0)
    offs = np.arange(4) * rows
    q, q64 = normal(rng, (3 * rows, heads * group, dh), dtype, 5.0)
    got = p.c.attention(q, ints([length] * 3), ints(offs), ints(table), scale=2.5)
    check_attention(p, table, q, q64, [length] * 3, offs, True, dtype, got, "far apart", 2.5)

    torn = table.copy()
    torn[0, 2], torn[1, 0], torn[1, 9], torn[2, :] = -1, 1 << 30, -7, -1
    for causal in (True, False):
        lengths = [length, 1 << 30, -5]
        got = p.c.attention(q, ints(lengths), ints(offs), ints(torn), causal=causal, scale=0.01)
        check_attention(p, torn, q, q64, lengths, offs, causal, dtype, got, f"torn {causal}", 0.01)

    # the last two places of sequence 0 hold NaN: rows before them do not see it, the others do
    bad, _ = normal(rng, (2, heads, dh), dtype)
    bad[0, :, 3], bad[1, :, 7] = float("nan"), float("inf")
    p.c.write(bad, bad, ints([length - 2]), ints([0, 2]), ints(table[:1]))
    p.m.write(table[:1].tolist(), [0, 2], [length - 2], values(bad), values(bad))
    got = values(p.c.attention(q, ints([length] * 3), ints(offs), ints(table), scale=0.01))
    assert np.isnan(got[rows - 1]).all()
    clean = table.copy()
    if rows > 2:
        k, v, there = p.m.history(clean.tolist(), 0, length)
        k[length - 2:], v[length - 2:] = 0, 0
        sees = np.arange(length)[None] <= (length - rows + np.arange(rows - 2))[:, None]
        out, mass, size = ref.attention(q64[:rows - 2], k, v, sees, 0.01)
        close(got[:rows - 2], out, ref.attention_tolerance(out, mass, size, dtype, dh, length), "before NaN")
    # NaN in values alone reaches its own channels only
    ok, _ = normal(rng, (2, heads, dh), dtype)
    p.c.write(ok, bad, ints([length - 2]), ints([0, 2]), ints(table[:1]))
    got = values(p.c.attention(q, ints([length] * 3), ints(offs), ints(table), scale=0.01))
    assert np.isnan(got[rows - 1][:, [3, 7]]).all() and not np.isnan(np.delete(got[rows - 1], [3, 7], 1)).any()
    if rows > 1:
        assert np.isnan(got[rows - 2][:, 3]).all() and not np.isnan(np.delete(got[rows - 2], 3, 1)).any()
        assert not np.isnan(got[:rows - 2]).any()


def test_attention_of_nan_queries_stays_in_its_rows():
    dh = 64
    rng = np.random.default_rng(13)
    for dtype, heads, rows in (("bf16", 2, 20), ("f32", 2, 20), ("bf16", 100, 80)):   # the last: large tiles
        p, table = filled(rng, heads, dh, 16, [90])
        q, q64 = normal(rng, (rows, heads, dh), dtype)
        q[4, 1, 9], q64[4, 1, 9] = float("nan"), np.nan
        got = values(p.c.attention(q, ints([90]), ints([0, rows]), ints(table)))
        assert np.isnan(got[4, 1]).all() and np.isnan(got).sum() == dh
        want = q64.copy()
        want[4, 1] = 0
        got[4, 1] = 0
        k, v, _ = p.m.history(table.tolist(), 0, 90)
        sees = np.arange(90)[None] <= (90 - rows + np.arange(rows))[:, None]
        out, mass, size = ref.attention(want, k, v, sees, dh ** -0.5)
        out[4, 1] = 0
        close(got, out, ref.attention_tolerance(out, mass, size, dtype, dh, 90), "others")


def test_pages_past_32_bit_offsets():
    """More than 4 GiB of codes: pages at the cache's end are read and written at their place."""
    torch = require_gpu()
    heads, dh, pt, pages = 8, 128, 128, 36000
    c = dj.TokenCache(pages, heads, dh, pt)
    assert c.k.numel() > 1 << 32
    first = torch.zeros_like(c.k[:64].view(torch.uint8))
    c.k[:64].view(torch.uint8).copy_(first)
    c.v[:64].view(torch.uint8).copy_(first)
    rng = np.random.default_rng(14)
    table = np.array([[pages - 1, pages - 3, 33000]])
    rows = 300
    k, k64 = normal(rng, (rows, heads, dh), "bf16")
    v, v64 = normal(rng, (rows, heads, dh), "bf16")
    c.write(k, v, ints([0]), ints([0, rows]), ints(table))
    m = ref.Cache(3, heads, pt, dh)
    m.write([[0, 1, 2]], [0, rows], [0], k64, v64)
    got = c.read(ints([0]), ints([0, rows]), ints(table), rows=rows)
    hk, hv, _ = m.history([[0, 1, 2]], 0, rows)
    assert np.array_equal(values(got[0]), hk) and np.array_equal(values(got[1]), hv)
    assert torch.equal(c.k[:64].view(torch.uint8), first) and torch.equal(c.v[:64].view(torch.uint8), first)
    q, q64 = normal(rng, (2, heads, dh), "bf16")
    out, mass, size = ref.attention(q64, hk, hv, np.tril(np.ones((2, rows), bool), rows - 2), dh ** -0.5)
    got = c.attention(q, ints([rows]), ints([0, 2]), ints(table))
    close(got, out, ref.attention_tolerance(out, mass, size, "bf16", dh, rows), "attention")


# ---- together ------------------------------------------------------------------------------------
def answer(c, rot, table, k, v, q, pos, starts, offs, lengths):
    """One step of answers in progress: their new tokens are written, and their queries attend."""
    turned = c.write(k, v, starts, offs, table, rot, pos, q)
    return c.attention(turned, lengths, offs, table)


def test_answers_over_a_video():
    """As they would be used: two clips' tokens are written as a prompt with their places in time and
    space, then tokens of answers one by one; every output against dense attention in 64 bits over
    the values that the cache holds.  Turned queries are rounded to bf16 before the attention: the tolerance
    counts their error in the scores."""
    torch = require_gpu()
    heads, group, dh, pt, n = 2, 4, 64, 16, 2
    sec = (8, 12, 12)
    rot = dj.Rotary(sec)
    rng = np.random.default_rng(15)
    counts = [70, 45]
    tp = 6
    p = Pair(n * tp + 1, heads, dh, pt)
    table = table_of(rng, n, tp, n * tp + 1)
    done = np.zeros(n, int)
    for step in range(8):
        counts = counts if step == 0 else [1, 1]
        offs = np.concatenate([[0], np.cumsum(counts)])
        rows = int(offs[-1])
        k, k64 = normal(rng, (rows, heads, dh), "bf16")
        v, v64 = normal(rng, (rows, heads, dh), "bf16")
        q, q64 = normal(rng, (rows, heads * group, dh), "bf16")
        pos = np.concatenate([np.stack([np.arange(a, a + c) // 16, np.arange(a, a + c) // 4 % 4,
                                        np.arange(a, a + c) % 4], 1) for a, c in zip(done, counts)])
        lengths = done + counts
        got = answer(p.c, rot, ints(table), k, v, q, ints(pos), ints(done), ints(offs), ints(lengths))
        p.m.x = p.decoded()
        tq, size = ref.turn(q64, pos, sec)
        for s in range(n):
            a, b = offs[s], offs[s + 1]
            hk, hv, _ = p.m.history(table.tolist(), s, lengths[s])
            sees = np.arange(lengths[s])[None] <= (done[s] + np.arange(counts[s]))[:, None]
            out, mass, top = ref.attention(tq[a:b], hk, hv, sees, dh ** -0.5)
            tol = ref.attention_tolerance(out, mass, top, "bf16", dh, int(lengths[s]))
            # scores off by sum |dq| |k| <= 2^-8 sum |q| |k| (and the turn's own): twice that in p
            tol += 2.2 * (ref.HALF["bf16"] + 2 * ref.TURN) * top[..., None] * mass
            close(got[a:b], out, tol, f"step {step}, sequence {s}")
        done = lengths
    back = p.c.read(ints([0, 0]), ints([0, done[0], done[0] + done[1]]), ints(table), rows=int(done.sum()))
    for w in range(2):
        want = np.concatenate([p.m.history(table.tolist(), s, done[s])[w] for s in range(n)])
        assert np.array_equal(values(back[w]), want)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("rows", [1, 33])
def test_captured_steps_replay(rows):
    """Two graphs of a write and an attention, captured with allocations of their own and replayed in
    turn with eager work between: every replay equals the eager step on the same inputs."""
    torch = require_gpu()
    heads, group, dh, pt, n = 2, 4, 128, 64, 3
    rot = dj.Rotary((16, 24, 24))
    rng = np.random.default_rng(16)
    lengths = [2100, 70, 900]
    p, table = filled(rng, heads, dh, pt, lengths)
    t = ints(table)
    offs = ints(np.arange(n + 1) * rows)
    starts, after = ints(np.array(lengths) - rows), ints(lengths)
    pos = ints(rng.integers(0, 1000, (n * rows, 3)))
    ins = [[torch.empty(n * rows, h, dh, dtype=torch.bfloat16, device="cuda") for h in (heads, heads, heads * group)]
           for _ in range(2)]
    fresh = lambda: [torch.randn(n * rows, h, dh, device="cuda").bfloat16() for h in (heads, heads, heads * group)]  # noqa: E731
    for i in range(2):
        for a, b in zip(ins[i], fresh()):
            a.copy_(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(2):
            answer(p.c, rot, t, *ins[i], pos, starts, offs, after)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(answer(p.c, rot, t, *ins[i], pos, starts, offs, after))
        graphs.append(g)
    for k in range(4):
        news = [fresh() for _ in range(2)]
        for i in range(2):
            for a, b in zip(ins[i], news[i]):
                a.copy_(b)
        for i in (0, 1) if k % 2 else (1, 0):
            graphs[i].replay()
            torch.cuda.synchronize()
            got, scales = outs[i].clone(), p.c.k_scale.nan_to_num(0.0)   # unused pages: NaN
            want = answer(p.c, rot, t, *news[i], pos, starts, offs, after)
            assert torch.equal(got, want), (k, i)
            assert torch.equal(scales, p.c.k_scale.nan_to_num(0.0))
            torch.randn(1 << 16, device="cuda").sum().item()


def test_on_a_stream_of_the_callers():
    """Everything on a given stream, behind work that takes a while there: results are those of the
    default stream, and the caller's streams stay as they were."""
    torch = require_gpu()
    heads, group, dh, pt = 2, 2, 64, 16
    rng = np.random.default_rng(17)
    p, table = filled(rng, heads, dh, pt, [2000, 40])
    q, _ = normal(rng, (2, heads * group, dh), "bf16")
    k, _ = normal(rng, (2, heads, dh), "bf16")
    pos = ints(rng.integers(0, 100, (2, 3)))
    rot = dj.Rotary((8, 12, 12))
    t, starts, lengths = ints(table), ints([1999, 39]), ints([2000, 40])
    want_q = p.c.write(k, k, starts, None, t, rot, pos, q)
    want = p.c.attention(want_q, lengths, None, t)
    want_rows = p.c.read(starts, None, t)
    want_x = dj.rotary(q, pos, rot)
    torch.cuda.synchronize()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(5):
            big @ big
        late = torch.empty_like(q)
        late.copy_(q)
    got_q = p.c.write(k, k, starts, None, t, rot, pos, late, stream=side)
    got = p.c.attention(got_q, lengths, None, t, stream=side)
    got_rows = p.c.read(starts, None, t, stream=side)
    got_x = dj.rotary(late, pos, rot, stream=side)
    assert torch.cuda.current_stream() == here
    side.synchronize()
    assert torch.equal(got_q, want_q) and torch.equal(got, want) and torch.equal(got_x, want_x)
    assert all(torch.equal(a, b) for a, b in zip(got_rows, want_rows))


@pytest.mark.parametrize("name", ["prompt-mixed", "long", "group-20"])
def test_attention_in_place(name):
    """out = q, with one split and several, in both kernels."""
    torch = require_gpu()
    for heads, group, dh, pt, counts, lengths, _ in (ATTENTION[name], LARGE["mixed-128"]):
        rng = np.random.default_rng(22)
        p, table = filled(rng, heads, dh, pt, lengths)
        q, _ = normal(rng, (sum(counts), heads * group, dh), "bf16")
        offs = ints(np.concatenate([[0], np.cumsum(counts)]))
        want = p.c.attention(q, ints(lengths), offs, ints(table))
        assert p.c.attention(q, ints(lengths), offs, ints(table), out=q) is q
        assert torch.equal(q, want)


def test_two_streams_at_once():
    """Calls whose splits meet in workspaces of their own, on two streams in turn."""
    torch = require_gpu()
    rng = np.random.default_rng(23)
    p, table = filled(rng, 2, 128, 64, [9000, 100, 8000])
    t, lengths, offs = ints(table), ints([9000, 100, 8000]), ints([0, 1, 2, 3])
    qs = [normal(rng, (3, 8, 128), "bf16")[0] for _ in range(2)]
    want = [p.c.attention(q, lengths, offs, t, max_rows=1) for q in qs]
    need = p.c.attention_workspace(3, 3, 8, table.shape[1], True, 1)
    assert need > 0
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in qs]
    out = [torch.empty_like(q) for q in qs]
    side = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(side):
            p.c.attention(qs[i], lengths, offs, t, max_rows=1, workspace=ws[i], out=out[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_workspace_of_the_callers():
    torch = require_gpu()
    rng = np.random.default_rng(18)
    p, table = filled(rng, 2, 64, 64, [5000, 100])
    q, q64 = normal(rng, (2, 4, 64), "bf16")
    need = p.c.attention_workspace(2, 2, 4, table.shape[1], True, 1)
    assert need > 0
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    got = p.c.attention(q, ints([5000, 100]), ints([0, 1, 2]), ints(table), max_rows=1, workspace=ws[:need])
    check_attention(p, table, q, q64, [5000, 100], [0, 1, 2], True, "bf16", got, "workspace")
    assert (ws[need:] == 255).all()
    with pytest.raises(dj.DejaVuError) as e:
        p.c.attention(q, ints([5000, 100]), ints([0, 1, 2]), ints(table), max_rows=1, workspace=ws[:need - 1])
    assert e.value.code == dj.DV_EINVAL


def test_wrapper_refuses():
    torch = require_gpu()
    c = dj.TokenCache(8, 2, 64, 16)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    at, pos = ints([0]), ints(np.zeros((4, 3)))
    offs, rot = ints([0, 4]), dj.Rotary((8, 12, 12))
    for bad in (dict(k=x[:, :1]), dict(v=x[:3]), dict(v=x.float()), dict(k=x[..., :32]), dict(k=x.half(), v=x.half()),
                dict(k=x.transpose(0, 1)), dict(starts=at.long()), dict(offsets=ints([0, 2, 4])),
                dict(table=ints([0, 1])), dict(rotary=rot), dict(positions=pos), dict(q_out=x),
                dict(rotary=rot, positions=pos[:3]), dict(rotary=rot, positions=pos, q=x.float()),
                dict(k=torch.zeros(4, 2, 128, dtype=x.dtype, device="cuda")[..., ::2])):
        with pytest.raises(ValueError):
            c.write(**dict(dict(k=x, v=x, starts=at, offsets=offs), **bad))
    with pytest.raises(ValueError):
        c.attention(x[..., :32], at, offs)
    with pytest.raises(ValueError):
        c.attention(x, at, offs, out=x[:2])
    with pytest.raises(dj.DejaVuError):
        c.attention(x[:, :1], at, offs)
    with pytest.raises(ValueError):
        dj.rotary(x, pos[:3], rot)
    with pytest.raises(ValueError):
        dj.rotary(x, pos, rot, out=x.float())
