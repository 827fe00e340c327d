"""Heads normed and turned in one pass, on rows and on their way into the 8-bit cache, against plain 64-bit versions."""
import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import Pair, close, ints, normal, table_of, types, values

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def norm(x, w, eps, dh):
    """(x w / sqrt(mean x^2 + eps), how far a kernel may be from it before its turn and last rounding).

    The sum of dh squares, none negative: a thread adds 16 of them (an fma each) and the head's dh / 16 sums, or a
    lane dh / 64 and the lanes in 6 steps: (16 + dh / 16) U relative at most, or less.  The division and the sum with eps:
    2 U more.  The root halves that and is off by 2 steps itself (4 U); two products: 2 U; eps
    is rounded to a float itself: U, halved.  In all (16 + dh / 32) U, and 2^-10 of that for errors of errors."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else w)
    return y, (16 + dh / 32) * U * (1 + 2.0 ** -10) * np.abs(y)


def turned(y, err, pos, sec, layout, far):
    """(y turned, error): an error of the parts of a pair counts in both, at most in full."""
    if sec is None:
        return y, err
    want, size = ref.turn(y, pos, sec, layout)
    _, both = ref.turn(err, np.zeros_like(pos), sec, layout)
    return want, (ref.TURN + far * 2.0 ** -52) * size + both * 1.001


def rounded(want, err, dtype):
    return err + ref.HALF[dtype] * (np.abs(want) + err)


NORM = {
    # rows, heads, dh, sections, layout, weight, eps, far, row padding, first element
    "frames": (257, 24, 64, (8, 12, 12), "halves", "head", 1e-6, 600, 0, 0),
    "pairs": (33, 3, 128, (24, 20, 20), "pairs", "all", 1e-6, 60000, 64, 0),
    "packed": (65, 16, 80, (14, 13, 13), "halves", "all", 1e-5, 100, 1040, 0),
    "part": (7, 5, 96, (8, 8, 8), "halves", "head", 1e-6, 1000, 16, 8),
    "part-pairs": (9, 5, 80, (0, 3, 5), "pairs", "all", 1e-6, 1000, 0, 0),
    "unturned": (100, 7, 112, None, "halves", "all", 1e-6, 1, 0, 0),
    "unturned-ones": (5, 1, 16, None, "halves", None, 1e-3, 1, 0, 0),
    "odd-section": (5, 2, 48, (5, 3, 3), "halves", "head", 1e-6, 1000, 0, 0),
    "quarters": (60, 12, 48, (4, 4, 4), "pairs", "head", 1e-6, 1000, 0, 0),
    "unaligned": (9, 2, 64, (8, 12, 12), "halves", "all", 1e-6, 1000, 1, 1),
    "four-apart": (9, 3, 64, (8, 12, 12), "halves", "head", 1e-6, 1000, 4, 4),
    "narrow": (3, 5, 6, (1, 0, 1), "pairs", "head", 1e-6, 1000, 3, 3),
    "wide-head": (3, 2, 200, (20, 20, 24), "halves", "all", 1e-6, 1000, 0, 0),
    "208": (3, 2, 208, (20, 20, 24), "halves", "all", 1e-6, 1000, 0, 0),
    "long-rows": (3, 301, 128, (24, 20, 20), "halves", "head", 1e-6, 1000, 0, 0),
    "one": (1, 1, 32, (4, 6, 6), "halves", "all", 1e-6, 1 << 30, 0, 0),
    "huge-head": (2, 1, 17000, (20, 20, 24), "halves", "all", 1e-6, 1000, 0, 0),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", NORM)
def test_norm_rotary(name, dtype):
    torch = require_gpu()
    rows, heads, dh, sec, layout, weight, eps, far, pad, first = NORM[name]
    rng = np.random.default_rng(3)
    flat, flat64 = normal(rng, first + rows * (heads * dh + pad), dtype, 3.0)
    shape, st = (rows, heads, dh), (heads * dh + pad, dh, 1)
    x = flat.as_strided(shape, st, first)
    x64 = np.lib.stride_tricks.as_strided(flat64[first:], shape, [8 * s for s in st])
    w = w64 = None
    if weight:
        w, w64 = normal(rng, (heads, dh) if weight == "head" else (dh,), dtype)
    pos = rng.integers(-far, far, (rows, 3))
    y, err = norm(x64, w64, eps, dh)
    want, err = turned(y, err, pos, sec, layout, far)
    tol = rounded(want, err, dtype)
    before = flat.clone()
    args = (w, eps) + ((ints(pos), dj.Rotary(sec, layout)) if sec else ())
    got = dj.norm_rotary(x, *args)
    close(got, want, tol, "new tensor")
    assert torch.equal(flat, before)
    assert dj.norm_rotary(x, *args, out=x) is x if sec else dj.norm_rotary(x, w, eps, out=x) is x
    assert torch.equal(x, got)
    outside = torch.ones_like(flat, dtype=torch.bool)
    outside.as_strided(shape, st, first)[:] = False
    assert torch.equal(flat[outside], before[outside])


@pytest.mark.parametrize("dh", [64, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_zeros_stay_and_a_nan_stays_in_its_head(dtype, dh):
    torch = require_gpu()
    rng = np.random.default_rng(4)
    x, x64 = normal(rng, (4, 3, dh), dtype)
    pos = ints(rng.integers(0, 100, (4, 3)))
    rot = dj.Rotary((4, 6, 6))
    clean = dj.norm_rotary(x, None, 1e-6, pos, rot)
    x[1, 1] = 0
    x[2, 0, 5] = float("nan")
    x[3, 2, 7] = float("inf")
    got = dj.norm_rotary(x, None, 1e-6, pos, rot)
    assert (got[1, 1] == 0).all() and got[2, 0].isnan().all()
    clean[1, 1] = 0
    for r, h in ((2, 0), (3, 2)):
        clean[r, h] = got[r, h] = 1
    assert torch.equal(got, clean)


@pytest.mark.parametrize("size", [1e-12, 1e-3, 2.0 ** 50])
def test_eps_against_small_and_large_heads(size):
    """eps settles heads much smaller than its root, and does nothing to large ones."""
    rng = np.random.default_rng(5)
    x, x64 = normal(rng, (5, 4, 96), "f32", size)
    want, err = norm(x64, None, 1e-6, 96)
    close(dj.norm_rotary(x), want, rounded(want, err, "f32"), f"size {size}")


def test_norm_rotary_of_no_rows():
    torch = require_gpu()
    x = torch.randn(0, 2, 16, device="cuda")
    assert dj.norm_rotary(x).shape == (0, 2, 16)


# ---- into the cache ---------------------------------------------------------------------------------
WRITE = {
    # heads, query heads, dh, page, sections, layout, weight, first element
    "halves": (2, 8, 64, 32, (8, 12, 12), "halves", "head", 0),
    "pairs-part": (2, 2, 64, 32, (4, 2, 2), "pairs", "all", 0),
    "odd-section": (2, 5, 64, 32, (3, 2, 2), "halves", "head", 0),
    "80": (5, 5, 80, 16, (14, 13, 13), "halves", "all", 0),
    "unturned": (3, 3, 48, 64, None, "halves", "head", 0),
    "unaligned": (3, 6, 48, 64, (8, 8, 8), "halves", "head", 1),
    "long-pages": (2, 4, 128, 128, (24, 20, 20), "halves", "all", 0),
    "long-pages-unaligned": (1, 3, 128, 128, (24, 20, 20), "pairs", "head", 1),
    "ones": (1, 16, 16, 16, (2, 3, 3), "halves", None, 0),
    "quarters": (2, 4, 48, 16, (4, 4, 4), "halves", "head", 0),
    "quarters-pairs": (3, 3, 112, 64, (10, 9, 9), "pairs", "all", 0),
    "four-apart": (2, 4, 80, 32, (14, 13, 13), "halves", "head", 4),
    "four-apart-pairs": (1, 2, 128, 128, (24, 20, 20), "pairs", "head", 4),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", WRITE)
def test_write_norms_keys_and_queries(name, dtype):
    """Queries as norm_rotary gives them; keys quantised from their normed and turned values in fp32: within
    those values' error before a rounding of half a step of e4m3, at a scale of a magnitude that close; values and
    their scales exactly as without norms."""
    heads, qh, dh, pt, sec, layout, weight, first = WRITE[name]
    torch = require_gpu()
    rng = np.random.default_rng(7)
    n, counts, starts = 3, [40 + pt, 1, 7], [0, 5, 0]
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows, tp = int(offs[-1]) + 2, -(-(40 + pt) // pt)
    table = table_of(rng, n, tp, n * tp)
    p = Pair(n * tp, heads, dh, pt)

    def tensor(shape, size=1.0):
        t, t64 = normal(rng, first + int(np.prod(shape)), dtype, size)
        return t[first:].view(shape), t64[first:].reshape(shape)

    (k, k64), (v, v64), (q, q64) = (tensor((rows, h, dh), 3.0) for h in (heads, heads, qh))
    kw = kw64 = qw = qw64 = None
    if weight:
        (kw, kw64), (qw, qw64) = (tensor((h, dh) if weight == "head" else (dh,)) for h in (heads, qh))
    old = [normal(rng, (5, heads, dh), dtype) for _ in range(2)]
    p.c.write(old[0][0], old[1][0], ints([0]), ints([0, 5]), ints(table[1:2]))
    p.m.write(table[1:2].tolist(), [0, 5], [0], old[0][1], old[1][1])
    pos = rng.integers(0, 5000, (rows, 3))
    turn = (dj.Rotary(sec, layout), ints(pos)) if sec else (None, None)
    q_out = q.new_full(q.shape, 3.0)
    got_q = p.c.write(k, v, ints(starts), ints(offs), ints(table), *turn, q, q_out,
                      k_norm=True if kw is None else kw, q_norm=True if qw is None else qw, eps=1e-5)
    assert got_q is q_out
    alive = int(offs[-1])
    y, err = norm(q64, qw64, 1e-5, dh)
    want, err = turned(y, err, pos, sec, layout, 5000)
    close(q_out[:alive], want[:alive], rounded(want, err, dtype)[:alive], "q")
    assert (q_out[alive:] == 3.0).all()
    y, err = norm(k64, kw64, 1e-5, dh)
    want, err = turned(y, err, pos, sec, layout, 5000)
    p.m.write(table.tolist(), offs, starts, want, v64)
    got, z = p.decoded(), values(p.c.k_scale)
    for s in range(n):
        for i in range(counts[s]):
            at, row = starts[s] + i, offs[s] + i
            page = table[s][at // pt]
            tol = err[row] + np.maximum(2.0 ** -4 * (np.abs(want[row]) + err[row]), 2.0 ** -10 * z[page][:, None])
            close(got[0][page, :, at % pt], want[row], tol, "k")
            assert np.array_equal(got[1][page, :, at % pt], p.m.x[1][page, :, at % pt])
        for j in range(starts[s] // pt, -(-(starts[s] + counts[s]) // pt)):
            page = table[s][j]
            assert np.array_equal(values(p.c.v_scale)[page], p.m.scale[1][page])
            assert all(z[page][h] in p.m.scale[0][page][h] * np.array([0.5, 1.0, 2.0]) for h in range(heads))
    for i in range(5):   # what the page held before
        close(got[0][table[1][0], :, i], old[0][1][i],
              2.0 ** -4 * np.abs(old[0][1][i]) + 2.0 ** -9 * z[table[1][0]][:, None], "held")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_outside_the_sequences_are_left_alone(dtype):
    """Rows before the first sequence and behind the last one: neither written nor normed, in place too."""
    torch = require_gpu()
    rng = np.random.default_rng(9)
    k, v, q = (normal(rng, (30, h, 64), dtype)[0] for h in (2, 2, 4))
    pos, rot = ints(rng.integers(0, 99, (30, 3))), dj.Rotary((8, 12, 12))
    before = q.clone()
    c = Pair(3, 2, 64, 16).c
    for t in (c.k_scale, c.v_scale):
        t.fill_(7.0)
    assert c.write(k, v, ints([0, 3]), ints([6, 15, 21]), ints([[0], [2]]), rot, pos, q, q, k_norm=True, q_norm=True) is q
    assert torch.equal(q[:6], before[:6]) and torch.equal(q[21:], before[21:])
    assert torch.equal(q[6:21], dj.norm_rotary(before[6:21], None, 1e-6, pos[6:21].contiguous(), rot))
    assert (c.k_scale[1] == 7).all() and (c.v_scale[1] == 7).all()
    # a sequence with a negative start is passed over; its queries are normed all the same
    c.write(k, v, ints([-1, 0]), ints([0, 15, 30]), ints([[0], [1]]), rot, pos, before.clone(), q, k_norm=True, q_norm=True)
    assert torch.equal(q, dj.norm_rotary(before, None, 1e-6, pos, rot))


@pytest.mark.parametrize("which", ["k", "q"])
def test_either_norm_alone(which):
    """Only keys or only queries normed: the others as without."""
    torch = require_gpu()
    rng = np.random.default_rng(8)
    k, v, q = (normal(rng, (9, h, 64), "bf16")[0] for h in (2, 2, 4))
    pos, rot = ints(rng.integers(0, 99, (9, 3))), dj.Rotary((8, 12, 12))
    out = []
    for kw in ({}, {"k_norm": True, "q_norm": True}, {which + "_norm": True}):
        c = Pair(1, 2, 64, 16).c
        qo = c.write(k, v, ints([0]), ints([0, 9]), None, rot, pos, q, **kw)
        out.append({"k": c.k.view(torch.uint8)[:, :, :9].clone(), "q": qo, "v": c.v.view(torch.uint8)[..., :9].clone()})
    for x in "kqv":
        assert torch.equal(out[2][x], out[1 if x == which else 0][x]), x
    c = Pair(1, 2, 64, 16).c   # without a rotation
    assert torch.equal(c.write(k, v, ints([0]), ints([0, 9]), q=q, q_norm=True), dj.norm_rotary(q))
