"""Attention with a window: pages that no row sees may hold anything, their scales too, where the table still names them."""
import numpy as np
import pytest

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import close, filled, ints, normal, values
from .test_gpu_window import seen

pytestmark = pytest.mark.gpu

# kv heads, group, dh, page, rows of each sequence, lengths: hidden pages lie in a step of 64 keys with seen ones
CASES = {
    "tokens-16": (2, 4, 128, 16, [1] * 4, [100, 333, 47, 200]),
    "rows-32": (2, 2, 64, 32, [20, 1, 5], [157, 217, 127]),
    "rows-16": (1, 5, 80, 16, [7, 1, 20], [90, 17, 125]),
    "large-16": (64, 2, 64, 16, [80, 80, 80], [150, 290, 205]),
    "large-32": (122, 1, 32, 32, [300], [409]),
    "both-32": (46, 4, 64, 32, [1, 120, 17, 0, 16, 3], [900, 183, 127, 40, 600, 60]),
}


NAN, INF = float("nan"), float("inf")
# (fp32 takes small tiles alone; scales that are numbers tell less than those that are none)
RUNS = [(name, dtype, causal, what) for name in CASES for dtype in (("bf16",) if CASES[name][0] > 2 else ("f32", "bf16"))
        for causal in (True, False) for what in ((NAN, INF, 3e38, -1.0) if name == "rows-32" else (NAN, INF))]


@pytest.mark.parametrize("name,dtype,causal,what", RUNS)
def test_pages_that_no_row_sees_may_hold_anything(name, dtype, causal, what):
    torch = require_gpu()
    heads, group, dh, pt, counts, lengths = CASES[name]
    rng = np.random.default_rng(41)
    offs = np.concatenate([[0], np.cumsum(counts)])
    q, q64 = normal(rng, (int(offs[-1]), heads * group, dh), dtype)
    spoilt = 0
    for window, sinks in ((5, 3), (15, 0), (20, 17)):
        p, table = filled(rng, heads, dh, pt, lengths)
        k8, v8 = p.c.k.view(torch.uint8), p.c.v.view(torch.uint8)
        for s, (n, length) in enumerate(zip(counts, lengths)):
            used = seen(length, n, causal, window, sinks).any(0) if n else np.zeros(length, bool)
            for j in range(-(-length // pt)):
                if used[j * pt:(j + 1) * pt].any():
                    continue
                page = int(table[s, j])
                p.c.k_scale[page] = p.c.v_scale[page] = what
                for x in (k8, v8):
                    x[page] = torch.randint(0, 256, x[page].shape, device="cuda", dtype=torch.uint8)
                near = used[j * pt // 64 * 64:(j * pt // 64 + 1) * 64]
                spoilt += bool(near.any())
        got = values(p.c.attention(q, ints(lengths), ints(offs), ints(table), causal=causal, window=window, sinks=sinks))
        for s, length in enumerate(lengths):
            a, b = offs[s], offs[s + 1]
            if a == b:
                continue
            k, v, _ = p.m.history(table.tolist(), s, length)
            want, mass, size = ref.attention(q64[a:b], k, v, seen(length, b - a, causal, window, sinks), dh ** -0.5)
            tol = ref.attention_tolerance(want, mass, size, dtype, dh, max(1, min(length, window + sinks)))
            close(got[a:b], want, tol, f"{name} {window} {sinks}, sequence {s}")
    assert spoilt      # in steps of 64 keys that a tile takes
