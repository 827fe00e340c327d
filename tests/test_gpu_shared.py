"""Attention over shared prefixes and sequences' own places, against plain 64-bit versions."""
import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import Pair, close, ints, normal, types, values

pytestmark = pytest.mark.gpu

# kv heads, group, dh, page, rows of each sequence, lengths, groups, prefixes' lengths, padding rows
CASES = {
    "tokens": (2, 4, 128, 64, [1] * 6, [1, 64, 65, 5, 0, 130], [0, 6], [700], 0),
    "one": (1, 1, 16, 16, [1], [1], [0, 1], [1], 0),
    "only-prefix": (2, 2, 64, 32, [3, 1], [0, 0], [0, 2], [100], 1),
    "no-prefix": (2, 2, 64, 32, [3, 1], [40, 9], [0, 2], [0], 1),
    "nothing": (1, 2, 48, 16, [3, 1], [0, 0], [0, 2], [0], 2),
    "groups": (3, 5, 80, 16, [7, 1, 20, 0, 2, 1], [9, 17, 20, 3, 0, 70], [0, 2, 2, 5, 6], [90, 33, 257, 0], 3),
    "outside": (2, 3, 96, 64, [4, 1, 2, 5], [4, 90, 2, 30], [1, 3], [130], 0),
    "more-rows-than-keys": (1, 4, 64, 16, [9, 40], [4, 39], [0, 1, 2], [30, 31], 1),
    "both-long": (1, 4, 128, 64, [2, 1, 1], [1500, 2100, 3], [0, 2, 3], [3001, 1100], 0),
    "prompts": (2, 2, 112, 128, [130, 70], [200, 70], [0, 2], [300], 4),
    "group-20": (2, 20, 32, 32, [3, 1], [70, 130], [0, 2], [65], 0),
}
# bf16 groups or sequences that take large tiles
LARGE = {
    "tokens": (8, 4, 128, 64, [1] * 64, [3 * i for i in range(64)], [0, 64], [2100], 0),
    "tokens-groups": (40, 4, 64, 64, [1] * 130, [i % 17 for i in range(130)], [0, 100, 102, 130], [500, 70, 129], 2),
    "rows": (56, 4, 64, 16, [141], [200], [0, 1], [100], 3),
    "mixed": (46, 4, 64, 32, [1, 120, 17, 0, 16, 3], [90, 130, 17, 4, 60, 2], [0, 2, 5, 6], [90, 150, 33], 0),
    "80": (54, 2, 80, 64, [230], [230], [0, 1], [64], 0),
    "16": (122, 1, 16, 128, [257], [300], [0, 1], [500], 0),
}
# ... whose tiles take the prefix and then the sequence's own keys; those above do so or not as the sizes have it
BEHIND = {
    "tokens": (2, 4, 128, 64, [1] * 6, [1, 64, 65, 5, 0, 130], [0, 6], [100], 0),
    "split": (1, 4, 64, 32, [1, 2], [2500, 1], [0, 1, 2], [70, 650], 0),
    "pages-16": (3, 5, 80, 16, [7, 1, 20, 0, 2, 1], [9, 17, 20, 3, 0, 70], [0, 2, 2, 5, 6], [90, 33, 57, 0], 3),
    "outside": (2, 3, 96, 64, [4, 1, 2, 5], [4, 90, 2, 30], [1, 3], [63], 0),
    "large": (56, 4, 64, 64, [141], [200], [0, 1], [100], 3),
    "large-16": (54, 2, 80, 16, [100, 130, 100], [130, 130, 9], [0, 2, 3], [65, 40], 0),
    "large-128": (34, 2, 128, 128, [250, 3], [250, 300], [0, 1, 1], [300, 7], 2),
    "mixed": (46, 4, 64, 32, [1, 120, 17, 0, 160, 30], [90, 130, 17, 4, 160, 2], [0, 2, 5, 6], [90, 50, 33], 0),
}
APART = {
    "tokens": (8, 4, 128, 64, [1] * 30, [9] * 30, [0, 30], [3000], 0),
    "f32-groups": (4, 4, 64, 16, [1] * 24, [3, 50, 0] * 8, [0, 15, 24], [4000, 3000], 0),
}
# Prefixes so long, for so many rows, that they take large tiles: alone, beside groups that do not, under sequences that do too
LONG = {
    "tokens": (8, 4, 128, 64, [1] * 76, [1 + i % 90 for i in range(76)], [0, 76], [10048], 0),
    "groups": (8, 4, 128, 64, [1] * 100, [1 + i % 9 for i in range(100)], [0, 90, 92, 100], [9024, 512, 320], 0),
    "prompts": (8, 4, 128, 64, [40] * 64, [40 + i for i in range(64)], [0, 64], [16384], 0),
    "prompts-16": (16, 2, 64, 16, [90, 1, 1, 30] * 16, [90, 5, 1, 200] * 16, [0, 30, 64], [8192, 6400], 3),
    "few": (2, 4, 64, 32, [1] * 10, [40, 1, 7, 2, 3] * 2, [0, 10], [60000], 0),
}


def build(heads, dh, pt, lengths, prefix, rng, size=1.0):
    """A cache that holds prefixes and sequences in scattered pages, its model, and both tables."""
    n, ng = len(lengths), len(prefix)
    tp, ptp = (max(1, max(-(-x // pt) for x in y)) for y in (lengths, prefix))
    total = n * tp + ng * ptp + 2
    p = Pair(total, heads, dh, pt, seed=3)
    order = rng.permutation(total)
    table, ptable = order[:n * tp].reshape(n, tp), order[n * tp:n * tp + ng * ptp].reshape(ng, ptp)
    for t, x in ((table, lengths), (ptable, prefix)):
        offs = np.concatenate([[0], np.cumsum(x)])
        if offs[-1]:
            k, k64 = normal(rng, (int(offs[-1]), heads, dh), "f32", size)
            v, v64 = normal(rng, (int(offs[-1]), heads, dh), "f32")
            p.c.write(k, v, ints([0] * len(x)), ints(offs), ints(t))
            p.m.write(t.tolist(), offs, [0] * len(x), k64, v64)
    return p, table, ptable


def expect(p, table, ptable, q64, counts, lengths, groups, prefix, causal, scale=None):
    """(output, mass, size, keys) of every sequence."""
    offs = np.concatenate([[0], np.cumsum(counts)])
    for s, (n, length) in enumerate(zip(counts, lengths)):
        length = max(0, min(length, table.shape[1] * p.m.pt))
        k, v, there = p.m.history(table.tolist(), s, length)
        sees = np.broadcast_to(there, (n, length)).copy()
        if causal:
            sees &= np.arange(length)[None] <= (length - n + np.arange(n))[:, None]
        g = [i for i in range(len(prefix)) if groups[i] <= s < groups[i + 1]]
        if g:
            pl = max(0, min(prefix[g[0]], ptable.shape[1] * p.m.pt))
            pk, pv, there = p.m.history(ptable.tolist(), g[0], pl)
            k, v = np.concatenate([pk, k]), np.concatenate([pv, v])
            sees = np.concatenate([np.broadcast_to(there, (n, pl)), sees], 1)
        dh = q64.shape[2]
        yield (s, offs[s], offs[s + 1], k, v, sees,
               ref.attention(q64[offs[s]:offs[s + 1]], k, v, sees, dh ** -0.5 if scale is None else scale))


def check(p, table, ptable, q64, counts, lengths, groups, prefix, causal, dtype, got, what, scale=None):
    got = values(got)
    for s, a, b, k, _, _, (out, mass, size) in expect(p, table, ptable, q64, counts, lengths, groups, prefix, causal, scale):
        if b > a:
            close(got[a:b], out, ref.attention_tolerance(out, mass, size, dtype, q64.shape[2], max(1, len(k))),
                  f"{what}, sequence {s}")


def shared_case(heads, group, dh, pt, counts, lengths, groups, prefix, pad, name, dtype, causal):
    rng = np.random.default_rng(11)
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows = int(offs[-1]) + pad
    wide, wide64 = normal(rng, (rows, heads * group + 3, dh), dtype)
    q, q64 = wide[:, 2:-1], wide64[:, 2:-1]
    calls = [(ints(offs), most, ints(groups)) for most in (0, max(counts))]
    if all(c == 1 for c in counts):
        calls.append((None, 0, ints(groups)))
    if groups == [0, len(counts)]:
        calls.append((ints(offs), 0, None))
    for o, most, g in calls:
        out = q.new_full((rows, heads * group, dh), 9.0)
        got = p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), o, ints(table), g, causal=causal, max_rows=most,
                                   out=out)
        assert got is out and (out[int(offs[-1]):] == 9.0).all()
        check(p, table, ptable, q64, counts, lengths, groups, prefix, causal, dtype, got, f"{name} max_rows {most}")


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", CASES)
def test_shared(name, dtype, causal):
    shared_case(*CASES[name], name, dtype, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", LARGE)
def test_shared_large_tiles(name, causal):
    shared_case(*LARGE[name], name, "bf16", causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", BEHIND)
def test_shared_behind(name, dtype, causal):
    shared_case(*BEHIND[name], name, dtype, causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", APART)
def test_shared_apart(name, dtype):
    shared_case(*APART[name], name, dtype, True)


ALL = {**CASES, **{"large-" + k: v for k, v in LARGE.items()}, **{"behind-" + k: v for k, v in BEHIND.items()},
       **{"apart-" + k: v for k, v in APART.items()}, **{"long-" + k: v for k, v in LONG.items()}}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", LONG)
def test_long_prefixes(name, dtype, causal):
    """Prefixes of whole pages, against attention over one table of both (itself tested against 64 bits): either is off by its
    tolerance, with the most that its parts can be: the largest value, the largest |q| |k|."""
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths, groups, prefix, pad = LONG[name]
    rng = np.random.default_rng(26)
    n, ng, tp, ptp = len(counts), len(prefix), max(-(-x // pt) for x in lengths), max(prefix) // pt
    total = n * tp + ng * ptp
    c = dj.TokenCache(total, heads, dh, pt)
    g = torch.Generator("cuda").manual_seed(3)
    for t in (c.k, c.v):
        t.copy_((torch.randn(t.shape, generator=g, device="cuda") * 100).clamp(-448, 448))
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.exp2(torch.randint(-9, -5, t.shape, generator=g, device="cuda").float()))
    order = rng.permutation(total)
    table, ptable = order[:n * tp].reshape(n, tp), order[n * tp:].reshape(ng, ptp)
    offs = np.concatenate([[0], np.cumsum(counts)])
    q = torch.randn(int(offs[-1]) + pad, heads * group, dh, generator=g, device="cuda").to(types(torch)[dtype])
    of = [max(i for i in range(ng) if groups[i] <= s) for s in range(n)]
    both = np.full((n, ptp + tp), -1)
    for s in range(n):
        k = prefix[of[s]] // pt
        both[s, :k], both[s, k:k + tp] = ptable[of[s], :k], table[s]
    after = np.array(lengths) + np.array(prefix)[of]
    got, want = torch.full_like(q, 3), torch.full_like(q, 3)
    c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), ints(offs), ints(table), ints(groups), causal=causal, out=got)
    c.attention(q, ints(after), ints(offs), ints(both), causal=causal, out=want)
    v = (c.v.float().abs().amax((2, 3)) * c.v_scale).max().item()
    kk = (c.k.float().norm(dim=3).amax(2) * c.k_scale).max().item() * q.float().norm(dim=2).max().item() * dh ** -0.5
    one = np.ones((1, 1, 1))
    tol = ref.attention_tolerance(0 * one, v * one, kk * np.ones((1, 1)), dtype, dh, int(after.max())).item()
    d = (got.double() - want.double()).abs()
    assert torch.isfinite(got).all() and d.max().item() <= 2 * tol, (d.max().item(), tol)
    assert d.square().mean().sqrt().item() <= 0.1 * tol      # and far closer nearly everywhere


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ALL)
def test_every_key_counts_once(name, dtype):
    """Queries of zeros weigh all keys alike; key j's value (of prefix and own counted on) is 256 in channel j % dh: an output is
    256 / keys times the keys of its channel.  Scores are 0, so that probabilities, sums and joins are exact but for the
    division and the output."""
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths, groups, prefix, _ = ALL[name]
    rng = np.random.default_rng(3)
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    for t, x, first in ((ptable, prefix, 0), (table, lengths, 5)):
        offs = np.concatenate([[0], np.cumsum(x)])
        v = np.zeros((int(offs[-1]), heads, dh), np.float32)
        for a, length in zip(offs, x):
            for j in range(length):
                v[a + j, :, (first + j) % dh] = 256
        if len(v):
            v = torch.from_numpy(v).cuda()
            p.c.write(torch.randn_like(v), v, ints([0] * len(x)), ints(offs), ints(t))
    offs = np.concatenate([[0], np.cumsum(counts)])
    q = torch.zeros(int(offs[-1]), heads * group, dh, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dtype], device="cuda")
    got = values(p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), ints(offs), ints(table), ints(groups)))
    for s, (n, length) in enumerate(zip(counts, lengths)):
        g = [i for i in range(len(prefix)) if groups[i] <= s < groups[i + 1]]
        pl = prefix[g[0]] if g else 0
        sees = np.concatenate([np.ones((n, pl), bool),
                               np.arange(length)[None] <= (length - n + np.arange(n))[:, None]], 1)
        ch = np.concatenate([np.arange(pl), 5 + np.arange(length)])[:, None] % dh == np.arange(dh)[None]
        total = sees.sum(1)
        want = np.where(total[:, None] > 0, 256 * (sees @ ch.astype(float)) / np.maximum(total, 1)[:, None], 0.0)
        want = np.broadcast_to(want[:, None], (n, heads * group, dh))
        close(got[offs[s]:offs[s + 1]], want, want * (ref.HALF[dtype] + 6 * 2.0 ** -24), f"{name}, sequence {s}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["tokens", "groups", "large-tokens", "large-rows", "behind-split", "behind-large-128", "behind-mixed", "apart-f32-groups"])
def test_scores_far_apart_missing_pages_and_odd_lengths(name, dtype):
    heads, group, dh, pt, counts, lengths, groups, prefix, _ = ALL[name]
    rng = np.random.default_rng(12)
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng, size=20.0)
    offs = np.concatenate([[0], np.cumsum(counts)])
    q, q64 = normal(rng, (int(offs[-1]), heads * group, dh), dtype, 5.0)
    got = p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), ints(offs), ints(table), ints(groups), scale=2.5)
    check(p, table, ptable, q64, counts, lengths, groups, prefix, True, dtype, got, "far apart", 2.5)
    torn, ptorn = table.copy(), ptable.copy()
    torn[0, 0], ptorn[0, -1] = -1, 1 << 30
    if ptable.shape[1] > 2:
        ptorn[0, 1] = -9
    odd = [-3] + list(lengths[1:-1]) + [1 << 30] if len(lengths) > 1 else [1 << 30]
    podd = [1 << 30] + [-4] * (len(prefix) - 1)
    # places past those written hold arbitrary bytes: a model of them
    p.m.x = [np.where(np.isfinite(x), x, 0) for x in p.decoded()]
    torch = require_gpu()
    for t in (p.c.k, p.c.v):
        b = t.view(torch.uint8)
        b[(b & 0x7F) == 0x7F] = 0
    p.c.k_scale.nan_to_num_(1.0)
    p.c.v_scale.nan_to_num_(1.0)
    p.m.x = p.decoded()
    for causal in (True, False):
        got = p.c.attention_shared(q, ints(odd), ints(podd), ints(ptorn), ints(offs), ints(torn), ints(groups), causal=causal, scale=1e-5)
        check(p, torn, ptorn, q64, counts, odd, groups, podd, causal, dtype, got, f"torn {causal}", 1e-5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["tokens", "groups", "large-tokens", "large-rows", "both-long", "behind-split", "behind-large-128", "behind-mixed", "apart-f32-groups"])
def test_nan_and_infinite_values_of_a_prefix_reach_its_group(name, dtype):
    heads, group, dh, pt, counts, lengths, groups, prefix, _ = ALL[name]
    rng = np.random.default_rng(13)
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    top = float(np.finfo(np.float32).max)
    bad = np.zeros((2, heads, dh), np.float32)
    bad[0, :, 2], bad[1, :, 5], bad[0, :, 7], bad[1, :, 7] = np.nan, -top, top, top
    torch = require_gpu()
    k = torch.randn(2, heads, dh, device="cuda")
    last = prefix[0] - 2
    p.c.write(k, torch.from_numpy(bad).cuda(), ints([last]), ints([0, 2]), ints(ptable[:1]))
    p.m.write(ptable[:1].tolist(), [0, 2], [last], values(k), bad.astype(np.float64))
    offs = np.concatenate([[0], np.cumsum(counts)])
    q, q64 = normal(rng, (int(offs[-1]), heads * group, dh), dtype)
    got = values(p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), ints(offs), ints(table), ints(groups), scale=0.02))
    p.m.x[1] = np.where(np.abs(p.m.x[1]) >= 2.0 ** 128, 0.0, np.nan_to_num(p.m.x[1]))
    for s, a, b, kk, _, _, (out, mass, size) in expect(p, table, ptable, q64, counts, lengths, groups, prefix, True, 0.02):
        if a == b:
            continue
        part, tol = got[a:b].copy(), ref.attention_tolerance(out, mass, size, dtype, dh, max(1, len(kk)))
        if groups[0] <= s < groups[1]:
            assert np.isnan(part[..., 2]).all() and (part[..., 5] == -np.inf).all() and (part[..., 7] == np.inf).all()
            part[..., [2, 5, 7]] = out[..., [2, 5, 7]]
        close(part, out, tol, f"sequence {s}")


@pytest.mark.parametrize("name", ["groups", "both-long", "large-tokens", "large-mixed", "behind-split", "behind-mixed", "apart-tokens"])
def test_in_place_on_a_stream_and_with_a_workspace(name):
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths, groups, prefix, _ = ALL[name]
    rng = np.random.default_rng(22)
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    q, _ = normal(rng, (sum(counts), heads * group, dh), "bf16")
    args = (ints(lengths), ints(prefix), ints(ptable), ints(np.concatenate([[0], np.cumsum(counts)])), ints(table), ints(groups))
    want = p.c.attention_shared(q, *args)
    need = p.c.attention_shared_workspace(len(counts), sum(counts), heads * group, ptable.shape[1], len(prefix), table.shape[1])
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = p.c.attention_shared(q, *args, workspace=ws[:need], stream=side, out=q)
    side.synchronize()
    assert got is q and torch.equal(q, want) and (ws[need:] == 255).all()


def test_one_prefix_equals_one_sequence():
    """A prefix and an own part of whole pages, against one sequence whose table has both: the same up to the joins' roundings."""
    torch = require_gpu()
    heads, group, dh, pt, n = 2, 4, 64, 16, 5
    rng = np.random.default_rng(24)
    lengths, prefix = [32, 48, 7, 1, 100], [160]
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    q, q64 = normal(rng, (n, heads * group, dh), "f32")
    got = p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), None, ints(table))
    both = np.concatenate([np.repeat(ptable, n, 0), table], 1)
    want = p.c.attention(q, ints(np.array(lengths) + 160), None, ints(both))
    _, mass, size = ref.attention(q64[:1], *p.m.history(both.tolist(), 0, 192)[:2], np.ones((1, 192), bool), dh ** -0.5)
    assert (got - want).abs().max().item() <= 2 * float(np.max(ref.attention_tolerance(0 * mass + 3, mass * 0 + 3, size, "f32", dh, 260)))
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("name", ["groups", "behind-large-128", "apart-f32-groups", "apart-tokens"])
def test_rows_before_the_first_sequence_are_left_alone(name):
    """Offsets that start behind a few rows: those stay as they were, in `out` and in the joins' view of the groups."""
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths, groups, prefix, _ = ALL[name]
    rng = np.random.default_rng(27)
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    offs = 5 + np.concatenate([[0], np.cumsum(counts)])
    q, q64 = normal(rng, (int(offs[-1]) + 2, heads * group, dh), "bf16")
    out = torch.full_like(q, 9)
    p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), ints(offs), ints(table), ints(groups), out=out)
    assert (out[:5] == 9).all() and (out[-2:] == 9).all()
    check(p, table, ptable, q64[5:], counts, lengths, groups, prefix, True, "bf16", out[5:], name)


def test_captured_steps_replay():
    """A graph of answers about one video, whose own places grow: each replay equals the eager call."""
    torch = require_gpu()
    heads, group, dh, pt, n = 2, 4, 128, 64, 6
    rng = np.random.default_rng(16)
    p, table, ptable = build(heads, dh, pt, [300] * n, [4000], rng)
    t, pt_, lengths, prefix = ints(table), ints(ptable), ints([1, 50, 100, 150, 0, 64]), ints([3900])
    q = torch.randn(n, heads * group, dh, device="cuda").bfloat16()
    p.c.attention_shared(q, lengths, prefix, pt_, None, t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = p.c.attention_shared(q, lengths, prefix, pt_, None, t)
    for _ in range(5):
        lengths += 21
        prefix += 13
        q.copy_(torch.randn(q.shape, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, p.c.attention_shared(q, lengths, prefix, pt_, None, t))
        torch.randn(1 << 16, device="cuda").sum().item()


def test_groups_out_of_range_do_no_harm():
    """Groups that no caller should give: past the sequences, descending, negative.  Sequences of a group that is as it should be are right."""
    torch = require_gpu()
    heads, group, dh, pt = 2, 2, 64, 16
    rng = np.random.default_rng(25)
    counts, lengths, prefix = [2, 1, 3], [10, 20, 3], [40, 30]
    p, table, ptable = build(heads, dh, pt, lengths, prefix, rng)
    q, q64 = normal(rng, (6, heads * group, dh), "bf16")
    for groups in ([0, 3, 1 << 30], [-5, 3, 3], [3, 0, 2], [0, 1 << 30, 2], [-1, -1, 1 << 30]):
        got = p.c.attention_shared(q, ints(lengths), ints(prefix), ints(ptable), ints([0, 2, 3, 6]), ints(table), ints(groups))
        assert got.shape == q.shape and torch.isfinite(got).all()
        if groups[0] <= 0 and groups[1] == 3:
            check(p, table, ptable, q64, counts, lengths, [0, 3, 3], prefix, True, "bf16", got, str(groups))
