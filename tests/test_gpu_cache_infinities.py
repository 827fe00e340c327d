"""Attention over values of the 8-bit cache that decode to infinity: the largest fp32 magnitudes, stored as 256 times
2^120."""
import numpy as np
import pytest

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import close, ints, normal, values
from .test_gpu_cache_edges import SIZES, put, seen, store

pytestmark = pytest.mark.gpu

TOP = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", SIZES)
def test_infinite_values_reach_the_rows_that_see_them(name, dtype, causal):
    """Infinities stand among the second values of the sequences, which all rows but few see, and among their last two:
    they reach, with their sign, the rows that see them, in their channels alone.  The scale keeps all
    probabilities above 2^-100."""
    heads, group, dh, pt, counts, lengths = SIZES[name]
    rng = np.random.default_rng(5)
    first = np.cumsum([0] + lengths)[:-1]
    k64 = rng.standard_normal((sum(lengths), heads, dh))
    v64 = rng.standard_normal((sum(lengths), heads, dh))
    v64[first + 1, :, 11] = -TOP
    p, table, _ = store(heads, dh, pt, lengths, k64, v64)
    bad = np.zeros((2, heads, dh))
    bad[0, :, 3], bad[1, :, 7], bad[0, :, 9], bad[1, :, 9] = TOP, -TOP, TOP, TOP
    for s, length in enumerate(lengths):
        put(p, table[s:s + 1], [length - 2], [0, 2], rng.standard_normal((2, heads, dh)), bad)
    offs = np.concatenate([[0], np.cumsum(counts)])
    q, q64 = normal(rng, (int(offs[-1]), heads * group, dh), dtype)
    scale = 0.02
    for most in (0, max(counts)):
        got = values(p.c.attention(q, ints(lengths), ints(offs), ints(table), causal=causal, scale=scale, max_rows=most))
        for s, (n, length) in enumerate(zip(counts, lengths)):
            k, v, there = p.m.history(table.tolist(), s, length)
            huge = np.abs(v) >= 2.0 ** 128
            assert there.all() and huge.any()
            sees = seen(length, n, causal)
            up, down = [(sees @ (huge & (np.sign(v) == sign)).any(1).astype(float)) > 0 for sign in (1, -1)]
            assert not (up & down).any() and (up | down).any()
            out, mass, size = ref.attention(q64[offs[s]:offs[s + 1]], k, np.where(huge, 0.0, v), sees, scale)
            tol = ref.attention_tolerance(out, mass, size, dtype, dh, length)
            assert size.max() < 60                       # a probability is e^-size and more of the largest
            part = got[offs[s]:offs[s + 1]].copy()
            for at, sign in ((up, 1), (down, -1)):
                at = np.broadcast_to(at[:, None], part.shape)
                assert (part[at] == sign * np.inf).all(), (name, s, sign, np.argwhere(at & (part != sign * np.inf))[:4])
                part[at] = out[at]
            close(part, out, tol, f"{name}, sequence {s}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_of_both_signs_and_nan(dtype):
    """In one channel: infinities of both signs, or one and a NaN, give NaN to the rows that see both."""
    heads, dh, pt, length = 1, 64, 16, 40
    rng = np.random.default_rng(6)
    p, table, _ = store(heads, dh, pt, [length], rng.standard_normal((length, heads, dh)),
                        rng.standard_normal((length, heads, dh)))
    bad = np.zeros((2, heads, dh))
    bad[0, :, 2], bad[1, :, 2], bad[0, :, 5], bad[1, :, 5] = TOP, -TOP, TOP, np.nan
    put(p, table, [length - 2], [0, 2], rng.standard_normal((2, heads, dh)), bad)
    q, _ = normal(rng, (4, heads, dh), dtype)
    got = values(p.c.attention(q, ints([length]), ints([0, 4]), ints(table), scale=0.02))[:, 0]
    assert np.isfinite(got[:2]).all()
    assert (got[2, [2, 5]] == np.inf).all() and np.isnan(got[3, [2, 5]]).all()
    assert np.isfinite(np.delete(got[2:], [2, 5], 1)).all()


def test_the_largest_finite_values_stay():
    """Values of 240 times 2^120, the largest that are finite, alone and beside a smaller one."""
    torch = require_gpu()
    heads, dh, pt = 1, 64, 16
    v64 = np.zeros((2, heads, dh))
    v64[0, :, 1], v64[1, :, 2] = 240 * 2.0 ** 120, -(2.0 ** 120)
    p, table, _ = store(heads, dh, pt, [2], np.zeros((2, heads, dh)), v64)
    assert p.c.v_scale[table[0, 0], 0].item() == 2.0 ** 120 and require_gpu() is torch
    for dtype in (torch.float32, torch.bfloat16):
        got = values(p.c.attention(torch.zeros(2, heads, dh, dtype=dtype, device="cuda"), ints([2]), ints([0, 2]),
                                   ints(table)))[:, 0]
        want = np.zeros((2, dh))
        want[0, 1], want[1, 1], want[1, 2] = 240 * 2.0 ** 120, 120 * 2.0 ** 120, -(2.0 ** 119)
        assert np.array_equal(got, want)
