"""Writes of batches whose sequences differ: what the kernel is chosen by is their mean, and a sequence far longer than that takes many
passes of it.  Bit for bit as written alone."""
import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from .gpu_util import require_gpu
from .test_gpu_cache import ints, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("heads,dh,pt", [(16, 80, 64), (8, 128, 128), (16, 64, 16), (3, 112, 32)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_long_sequence_among_single_tokens(dtype, heads, dh, pt, norms):
    torch = require_gpu()
    rng = np.random.default_rng(5)
    n, long = 60, 300
    counts = [1] * n
    counts[17], counts[30] = long, 0
    offs = np.concatenate([[0], np.cumsum(counts)])
    rows, tp = int(offs[-1]), -(-(long + 21) // pt)
    k, v, q = (normal(rng, (rows, h, dh), dtype)[0] for h in (heads, heads, 2 * heads))
    held = [normal(rng, (21 * n, heads, dh), dtype)[0] for _ in range(2)]
    pos, rot = ints(rng.integers(0, 5000, (rows, 3))), dj.Rotary((4, 6, 6))
    table = ints(rng.permutation(n * tp).reshape(n, tp))
    kw = dict(k_norm=True, q_norm=True) if norms else {}
    starts = ints([21] * n)
    got = []
    for alone in (False, True):
        c = dj.TokenCache(n * tp, heads, dh, pt)
        for t in (c.k, c.v):
            t.view(torch.uint8).zero_()
        for t in (c.k_scale, c.v_scale):
            t.fill_(1.0)
        c.write(held[0], held[1], ints([0] * n), ints(21 * np.arange(n + 1)), table)
        if not alone:
            q_out = c.write(k, v, starts, ints(offs), table, rot, pos, q, **kw)
        else:
            q_out = torch.empty_like(q)
            for s in range(n):
                a, b = int(offs[s]), int(offs[s + 1])
                if a < b:
                    c.write(k[a:b], v[a:b], starts[s:s + 1], ints([0, b - a]), table[s:s + 1], rot, pos[a:b].contiguous(), q[a:b], q_out[a:b], **kw)
        got.append([t.clone() for t in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale, q_out)])
    for name, a, b in zip(("keys", "values", "scales of keys", "scales of values", "queries"), *got):
        assert torch.equal(a, b), name
