"""Norms of heads at either end of fp32: magnitudes up to 2^60 in every channel of heads of any width, and the least eps."""
import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from .gpu_util import require_gpu
from .test_gpu_cache import Pair, close, ints, normal
from .test_gpu_norm import norm, rounded, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [2, 16, 40, 128, 130, 144, 202, 256, 258, 272, 1024, 8192, 8194, 16384, 70000])
def test_heads_of_the_largest_magnitudes(dh, dtype):
    """Every channel 2^60 or its negative, and one head of channels from 2^58 on."""
    torch = require_gpu()
    rng = np.random.default_rng(dh)
    x64 = np.where(rng.random((3, 2, dh)) < 0.5, -1.0, 1.0) * 2.0 ** 60
    x64[1, 1] *= rng.choice([0.25, 0.5, 0.75, 1.0], dh)
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    x = torch.tensor(x64).to(types[dtype]).cuda()
    w, w64 = normal(rng, (dh,), dtype)
    for weight, weight64 in ((None, None), (w, w64)):
        want, err = norm(x64, weight64, 1e-6, dh)
        close(dj.norm_rotary(x, weight), want, rounded(want, err, dtype), f"{dh} channels")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sec,layout,first", [((8, 12, 12), "halves", 0), ((4, 4, 4), "pairs", 0), ((5, 3, 3), "halves", 0), ((8, 12, 12), "pairs", 4),
                                              ((8, 12, 12), "halves", 1), (None, "halves", 0)])
@pytest.mark.parametrize("dh", [144, 256, 1040])
def test_wide_heads_normed_and_turned(dh, sec, layout, first, dtype):
    """Heads of more than 128 channels by eights, fours and ones, rows aligned and not."""
    rng = np.random.default_rng(6)
    flat, flat64 = normal(rng, first + 9 * 3 * dh, dtype, 3.0)
    x, x64 = flat[first:].view(9, 3, dh), flat64[first:].reshape(9, 3, dh)
    w, w64 = normal(rng, (3, dh), dtype)
    pos = rng.integers(-1000, 1000, (9, 3))
    y, err = norm(x64, w64, 1e-6, dh)
    want, err = turned(y, err, pos, sec, layout, 1000)
    got = dj.norm_rotary(x, w, 1e-6, *((ints(pos), dj.Rotary(sec, layout)) if sec else ()))
    close(got, want, rounded(want, err, dtype), f"{dh} {sec}")


@pytest.mark.parametrize("eps", [1e-6, 1e-37, 1e-40, 2.0 ** -149])
@pytest.mark.parametrize("dh", [64, 40, 256])
def test_zeros_stay_zeros_at_any_eps(dh, eps):
    torch = require_gpu()
    x = torch.zeros(5, 3, dh, device="cuda")
    x[1, 1] = 1.0
    want = torch.zeros_like(x)
    want[1, 1] = 1.0
    got = dj.norm_rotary(x, None, eps)
    assert (got[want == 0] == 0).all() and ((got - want).abs() <= 2.0 ** -20).all()


def test_keys_of_the_largest_magnitudes_into_the_cache():
    """128 channels of 2^60, their sum of squares 2^127: ones and their negatives, exact in 8 bits."""
    torch = require_gpu()
    rng = np.random.default_rng(3)
    k = torch.tensor(np.where(rng.random((9, 2, 128)) < 0.5, -1.0, 1.0) * 2.0 ** 60).float().cuda()
    c = Pair(1, 2, 128, 16).c
    c.write(k, torch.zeros_like(k), ints([0]), ints([0, 9]), k_norm=True)
    got = c.read(ints([0]), ints([0, 9]), rows=9, dtype=torch.float32)[0]
    assert torch.equal(got, torch.sign(k))
