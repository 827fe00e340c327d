"""Pages taken back by several blocks over several chunks of sequences (1024 at once): each counts the pages of those before it."""
import numpy as np
import pytest

from .gpu_util import require_gpu  # noqa: F401
from .test_gpu_extend import batch, check

pytestmark = pytest.mark.gpu


def parts(n, table_pages):
    """Blocks that take pages back in a call of these sizes, as the launch cuts it."""
    return min(16, (n * table_pages + 32767) // 32768)


@pytest.mark.parametrize("n,pages,share", [(2500, 60, 0.5), (1025, 64, 0.9), (2049, 300, 0.2), (3100, 40, 0.02), (1100, 90, 1.0)])
def test_pages_come_back_in_order_over_blocks_and_chunks(n, pages, share):
    """Many of each chunk's sequences end, with entries that are no pages among theirs; others take pages in the same call."""
    rng = np.random.default_rng(n)
    assert parts(n, pages) > 1 and n > 1024
    counts = np.where(rng.random(n) < share, -1, rng.choice([0, 1, 1, 17], n))
    held = rng.integers(0, 16 * pages - 20, n)
    rows = int(np.maximum(counts, 0).sum())
    for gone, start in ((0.0, 0), (0.2, 12345)):
        check(batch(rng, n, 16, pages, 2 * n, counts, held, gone=gone, start=start), 16, rows)


def test_sequences_that_end_in_one_chunk_alone():
    """None of the first chunk's, all of the second's, one of the third's."""
    rng = np.random.default_rng(8)
    n, pages = 2100, 50
    counts = np.concatenate([np.ones(1024), np.full(1024, -1), [-1], np.zeros(51)]).astype(int)
    assert parts(n, pages) > 1
    check(batch(rng, n, 16, pages, 100, counts, rng.integers(0, 780, n), gone=0.1, start=7), 16, 1024)


def test_a_ring_without_room_takes_no_more_than_it_holds():
    """A cursor that says more pages are free than are not: what comes back stops where the ring is full."""
    rng = np.random.default_rng(9)
    n, pages = 1500, 64
    counts = np.full(n, -1)
    table, lengths, counts, ring, cursor = batch(rng, n, 16, pages, 500, counts, rng.integers(500, 1000, n))
    for room in (len(ring) - 3000, len(ring) - 1, len(ring)):
        check((table, lengths, counts, ring, np.array([11, 11 + room, 0])), 16, 0)
