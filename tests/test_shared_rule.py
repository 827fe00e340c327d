"""Which shared calls take their prefix in tiles of the sequences and which in a pass of its own: what was measured as the faster."""
import ctypes

import pytest

from .test_window import lib  # noqa: F401 (a fixture)


def behind(lib, bf16, seqs, rows, heads, group, dh, keys, groups=1, own=64):
    out = (ctypes.c_longlong * 19)()
    lib.t_shared_plan(bf16, seqs, seqs * rows, 1, rows, -(-own // 64), groups, -(-keys // 64), 64, heads, heads * group, dh, 256, out)
    return bool(out[18])


@pytest.mark.parametrize("seqs,rows,keys,want", [
    (1, 1, 100000, True), (2, 1, 100000, False), (3, 1, 100000, False), (2, 1, 200000, False), (2, 1, 70000, False), (3, 1, 40000, False),
    (2, 1, 4000, True), (3, 1, 4000, True), (4, 1, 100000, False), (8, 1, 100000, False), (2, 4, 100000, False), (2, 64, 20000, False), (2, 64, 2000, True),
    (64, 1, 128, True), (64, 1, 2048, False), (64, 1, 8192, False), (64, 40, 512, True), (12, 33, 128, True), (12, 33, 50000, False)])
def test_calls_that_were_measured(lib, seqs, rows, keys, want):  # noqa: F811
    """8 heads of 128 with 4 queries each, in bf16."""
    assert behind(lib, 1, seqs, rows, 8, 4, 128, keys) == want


def test_a_prefix_is_never_read_faster_than_the_memory_has_it(lib):  # noqa: F811
    """Tiles that repeat a long prefix are chosen less and less as they get more: never again, once not."""
    for keys in (1000, 20000, 100000, 500000):
        for rows in (1, 4, 33):
            took = [behind(lib, 1, n, rows, 8, 4, 128, keys) for n in range(1, 40)]
            assert took == sorted(took, reverse=True)
