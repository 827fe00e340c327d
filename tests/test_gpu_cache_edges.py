"""Attention over the 8-bit cache: every key counted once, and scores far past what fp32 tells apart."""
import numpy as np
import pytest

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import Pair, close, ints, table_of, types, values

pytestmark = pytest.mark.gpu

# Sizes that take small tiles alone, large ones alone, both by sequence, and splits of the keys of either.
# kv heads, group, dh, page, rows of each sequence, lengths
SIZES = {
    "token": (2, 4, 128, 64, [1], [700]),
    "rows": (2, 2, 64, 16, [20, 1, 5], [150, 17, 3]),
    "few-split": (1, 4, 128, 64, [1, 3], [3001, 2100]),
    "large": (64, 2, 64, 16, [80, 80, 80], [150, 90, 200]),
    "large-split": (7, 8, 128, 64, [300], [1200]),
    "both": (14, 4, 128, 64, [20, 1, 260, 2], [40, 3000, 260, 5]),
}


def store(heads, dh, pt, lengths, k64, v64):
    """A cache that holds these keys and values, its model and table."""
    rng = np.random.default_rng(2)
    n, tp = len(lengths), max(-(-x // pt) for x in lengths)
    p = Pair(n * tp + 2, heads, dh, pt)
    table = table_of(rng, n, tp, n * tp + 2)
    offs = np.concatenate([[0], np.cumsum(lengths)])
    put(p, table, [0] * n, offs, k64, v64)
    return p, table, offs


def put(p, table, starts, offs, k64, v64):
    torch = require_gpu()
    k, v = [torch.from_numpy(x.astype(np.float32)).cuda() for x in (k64, v64)]
    p.c.write(k, v, ints(starts), ints(offs), ints(table))
    p.m.write(table.tolist(), offs, starts, k64, v64)


def seen(length, n, causal):
    """[rows, keys] that the n last rows of a sequence see."""
    last = length - n + np.arange(n) if causal else np.full(n, length - 1)
    return np.arange(length)[None] <= last[:, None]


# ---- every key counts once ---------------------------------------------------------------------------
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", SIZES)
def test_every_key_counts_once(name, dtype, causal):
    """Queries of zeros weigh all keys alike, and key j's value is 256 in channel j % dh (or (j // dh) % dh) and
    0 elsewhere: an output is 256 / keys times the keys of its channel, 71 at most, so one key lost or taken twice is
    more than 2^-7 of it.  Scores are 0, probabilities 1 and their sums whole numbers: only the division (two
    roundings of fp32) and the output are rounded."""
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths = SIZES[name]
    for by in (1, dh):
        k64 = np.random.default_rng(3).standard_normal((sum(lengths), heads, dh))
        v64 = np.zeros((sum(lengths), heads, dh))
        for a, length in zip(np.cumsum([0] + lengths), lengths):
            for j in range(length):
                v64[a + j, :, j // by % dh] = 256
        p, table, _ = store(heads, dh, pt, lengths, k64, v64)
        offs = np.concatenate([[0], np.cumsum(counts)])
        q = torch.zeros(int(offs[-1]), heads * group, dh, dtype=types(torch)[dtype], device="cuda")
        got = values(p.c.attention(q, ints(lengths), ints(offs), ints(table), causal=causal))
        for s, (n, length) in enumerate(zip(counts, lengths)):
            sees = seen(length, n, causal)
            ch = (np.arange(length) // by % dh)[:, None] == np.arange(dh)[None]
            total = sees.sum(1)
            want = np.where(total[:, None] > 0, 256 * (sees @ ch.astype(float)) / np.maximum(total, 1)[:, None], 0.0)
            want = np.broadcast_to(want[:, None], (n, heads * group, dh))
            tol = want * (ref.HALF[dtype] + 4 * 2.0 ** -24)
            close(got[offs[s]:offs[s + 1]], want, tol, f"{name}, keys by {by}, sequence {s}")


# ---- scores far apart --------------------------------------------------------------------------------
@pytest.mark.parametrize("scale", [2.0 ** 10, 2.0 ** 26, 2.0 ** 60, 3.0e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", SIZES)
def test_the_largest_score_wins_however_large(name, dtype, scale):
    """Queries and keys are small whole numbers, so that q k is exact; times the scale, scores differ by 2^10 and
    more where they differ: all probabilities are 0 but those of the largest, which are alike.  Sums of at most 3001
    ones are exact, sums of values are off by at most their number of roundings of fp32, bf16 holds a 1, and codes
    are exact: 2^-24 a key and the division's, relative to the mean of |v|."""
    heads, group, dh, pt, counts, lengths = SIZES[name]
    rng = np.random.default_rng(4)
    k64 = rng.integers(-7, 8, (sum(lengths), heads, dh)).astype(float)
    v64 = rng.integers(-15, 16, (sum(lengths), heads, dh)).astype(float)
    p, table, _ = store(heads, dh, pt, lengths, k64, v64)
    offs = np.concatenate([[0], np.cumsum(counts)])
    torch = require_gpu()
    q64 = rng.integers(-3, 4, (int(offs[-1]), heads * group, dh)).astype(float)
    q = torch.from_numpy(q64).to(types(torch)[dtype]).cuda()
    got = values(p.c.attention(q, ints(lengths), ints(offs), ints(table), scale=scale))
    for s, (n, length) in enumerate(zip(counts, lengths)):
        sees = seen(length, n, True)
        k, v, there = p.m.history(table.tolist(), s, length)
        assert there.all()
        want, mass = np.zeros((n, heads * group, dh)), np.zeros((n, heads * group, dh))
        for h in range(heads * group):
            z = np.where(sees, q64[offs[s]:offs[s + 1], h] @ k[:, h // group].T, -np.inf)
            w = (z == z.max(1, keepdims=True)) & sees
            w = w / np.maximum(w.sum(1, keepdims=True), 1)
            want[:, h], mass[:, h] = w @ v[:, h // group], w @ np.abs(v[:, h // group])
        t = mass * (length + 4) * 2.0 ** -24
        close(got[offs[s]:offs[s + 1]], want, t + ref.HALF[dtype] * (np.abs(want) + t), f"{name}, sequence {s}")
