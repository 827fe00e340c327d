"""Pages handed out and taken back on the GPU, against the rule spelt out sequence by sequence.  Everything is whole numbers:
equal or wrong."""
import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from . import cache_ref as ref
from .gpu_util import require_gpu
from .test_gpu_cache import ints, values

pytestmark = pytest.mark.gpu


def model(table, lengths, counts, ring, cursor, pt, rows, positions, slots):
    """The rule; table, ring, positions and slots in place.  Returns offsets, starts, lengths, cursor."""
    n, P = table.shape
    pages = len(ring)
    taken, given = int(cursor[0]), int(cursor[1])
    room = min(max(given - taken, 0), pages)
    free = [int(ring[(taken + i) % pages]) for i in range(room)]
    offsets, starts, after, used, lack, back, row = [0], [], [], 0, 0, 0, 0
    short = False
    for s in range(n):
        length, new = max(int(lengths[s]), 0), max(int(counts[s]), 0)
        held, need = -(-length // pt), -(-(length + new) // pt) - -(-length // pt)
        fits = new == 0 or held + need <= P
        if fits and need:
            short = short or used + need > room
        got = fits and not (need and short)
        if got:
            table[s, held:held + need] = free[used:used + need]
            used += need
        elif fits:
            lack += need
        if counts[s] < 0:
            for page in table[s, :min(held, P)]:
                if 0 <= page < pages and back < pages - room:
                    ring[(given + back) % pages] = page
                    back += 1
        starts.append(length if got and counts[s] >= 0 else -1)
        after.append(0 if counts[s] < 0 else length + new if got else length)
        for i in range(new):
            if row + i >= rows:
                break
            p = length + i
            page = int(table[s, p // pt]) if got else -1
            positions[row + i] = p
            slots[row + i] = page * pt + p % pt if 0 <= page < pages else -1
        row += new
        offsets.append(row)
    return offsets, starts, after, [taken + used, given + back, lack]


def batch(rng, n, pt, P, spare, counts, held, gone=0.0, start=0):
    """A batch whose sequences hold pages of their own; the ring holds the others."""
    lengths = np.asarray(held)
    own = -(-lengths // pt)
    total = int(own.sum()) + spare
    order = rng.permutation(total)
    table = np.full((n, P), -1)
    at = 0
    for s in range(n):
        table[s, :own[s]] = order[at:at + own[s]]
        at += own[s]
    table[rng.random(table.shape) < gone] = -1
    ring = np.full(total, -7)
    ring[(start + np.arange(spare)) % total] = order[at:]
    return table, lengths, np.asarray(counts), ring, np.array([start, start + spare, 0])


def check(case, pt, rows, new=False):
    torch = require_gpu()
    table, lengths, counts, ring, cursor = case
    n = len(lengths)
    t = [ints(table), ints(lengths), ints(counts), ints(ring), torch.tensor(cursor, device="cuda")]
    keep = [t[1].clone(), t[2].clone(), t[4].clone()]
    out = None
    if not new:
        out = [torch.full(s, -9, dtype=d, device="cuda") for s, d in (
            ((n + 1,), torch.int32), ((n,), torch.int32), ((n,), torch.int32), ((3,), torch.int64),
            ((rows, 3), torch.int32), ((rows,), torch.int64))]
    if len(ring) == 0:      # no cache is that small
        with pytest.raises(dj.DejaVuError):
            dj.extend(*t, pt, rows, out=out)
        return None
    got = dj.extend(*t, pt, rows, out=out)
    assert out is None or got is out
    table, ring = table.copy(), ring.copy()
    positions, slots = np.full((rows, 3), -9), np.full(rows, -9)
    want = model(table, lengths, counts, ring, cursor, pt, rows, positions, slots)
    live = min(rows, want[0][-1]) if new else rows
    for name, g, w in (("table", t[0], table), ("ring", t[3], ring), *zip(("offsets", "starts", "lengths", "cursor"), got, want),
                       ("positions", got[4][:live], positions[:live]), ("slots", got[5][:live], slots[:live])):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert all(torch.equal(a, b) for a, b in zip(keep, (t[1], t[2], t[4])))
    return got, want


@pytest.mark.parametrize("pt", [16, 32, 64, 128])
def test_random_batches(pt):
    rng = np.random.default_rng(pt)
    for n in (1, 2, 7, 64, 300):
        for spare in (0, 1, 5, 3 * n, 20 * n):
            counts = rng.choice([-1, 0, 1, 1, 2, pt - 1, pt, pt + 1, 3 * pt], n)
            held = rng.choice([0, 1, pt - 1, pt, pt + 1, 5 * pt + 3], n)
            case = batch(rng, n, pt, int(rng.choice([7, 9, 12])), spare, counts, held, gone=rng.choice([0, 0.2]),
                         start=int(rng.integers(0, 1 << 33)))
            check(case, pt, int(np.maximum(counts, 0).sum()) + int(rng.choice([0, 3])), new=bool(rng.random() < 0.3))


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2500])
def test_more_sequences_than_a_block_sums_at_once(n):
    rng = np.random.default_rng(n)
    for spare in (n // 2, 8 * n):
        counts = rng.choice([-1, 0, 1, 1, 1, 40], n)
        case = batch(rng, n, 16, 9, spare, counts, rng.integers(0, 90, n), start=11)
        check(case, 16, int(np.maximum(counts, 0).sum()) + 1)


def test_all_end_and_all_stay():
    rng = np.random.default_rng(1)
    held = rng.integers(0, 200, 500)
    check(batch(rng, 500, 16, 13, 3, [-1] * 500, held, gone=0.1, start=5), 16, 0)
    check(batch(rng, 500, 16, 13, 3, [-5] * 500, held), 16, 4)
    check(batch(rng, 500, 16, 13, 3, [0] * 500, held), 16, 4)


def test_long_tables_go_back_in_parts():
    """Pages of sequences that end, more than a block takes back at once."""
    rng = np.random.default_rng(2)
    counts = rng.choice([-1, 1], 40)
    check(batch(rng, 40, 16, 2100, 100, counts, rng.integers(0, 33000, 40), gone=0.3, start=123), 16, 40)


def test_a_prompt_over_many_blocks():
    rng = np.random.default_rng(3)
    check(batch(rng, 3, 16, 20000, 19000, [250000, -1, 33333], [5, 100, 16], start=18999), 16, 283333)


def test_rows_past_the_call_have_no_place():
    """Pages are handed out by counts, rows cut to those there are."""
    rng = np.random.default_rng(4)
    check(batch(rng, 5, 16, 9, 50, [20, 0, 50, 7, 1], [3, 0, 16, 31, 15]), 16, 33)
    check(batch(rng, 5, 16, 9, 50, [20, 0, 50, 7, 1], [3, 0, 16, 31, 15]), 16, 0)


def test_a_sequence_that_passes_its_table_takes_nothing():
    rng = np.random.default_rng(5)
    got, want = check(batch(rng, 4, 16, 4, 30, [10, 40, 32, 5], [60, 30, 32, 60]), 16, 87)
    assert want[1] == [-1, -1, 32, -1] and want[3][2] == 0


def test_a_ring_that_holds_no_more_than_there_are():
    """Cursors that no sequence of calls leads to, and entries that are no pages, do no harm."""
    rng = np.random.default_rng(6)
    table, lengths, counts, ring, _ = batch(rng, 6, 16, 9, 30, [20, 3, -1, 50, -1, 1], [3, 0, 16, 31, 15, 80])
    ring[::3] = rng.choice([-1, 1 << 30, len(ring)], len(ring[::3]))
    for cursor in ([5, 5 + 10 * len(ring), 0], [9, 2, 0], [-40, -20, 7], [1 << 40, (1 << 40) + 9, 0]):
        check((table, lengths, counts, ring, np.array(cursor)), 16, 80)
    check((table, np.array([-4, 0, 300, 0, 1000, -1]), counts, ring, np.array([0, 30, 0])), 16, 80)


def test_positions_and_slots_are_not_asked_for():
    torch = require_gpu()
    rng = np.random.default_rng(7)
    case = batch(rng, 6, 16, 9, 30, [20, 3, -1, 50, -1, 1], [3, 0, 16, 31, 15, 80])
    want, _ = check(case, 16, 80)
    t = [ints(case[0]), *map(ints, case[1:4]), torch.tensor(case[4], device="cuda")]
    new = [torch.empty_like(x) for x in want[:4]] + [None, None]
    dj.extend(*t, 16, 80, out=new)
    assert all(torch.equal(a, b) for a, b in zip(new[:4], want[:4]))


def serving(steps, n):
    """The counts of a few serving steps' sequences."""
    rng = np.random.default_rng(9)
    return [rng.choice([1, 1, 1, 0, 20, -1], n) if i else rng.integers(1, 40, n) for i in range(steps)]


@pytest.mark.parametrize("pages", [40, 14])
def test_serving_steps(pages):
    """Steps of a server: pages handed out, keys and queries normed, turned and written, attention over what each
    sequence holds; sequences that end give their pages to those that start.  Checked against the rows themselves, read
    back."""
    torch = require_gpu()
    heads, group, dh, pt, n, P = 2, 4, 64, 16, 9, 12
    steps = serving(12, n)
    c = dj.TokenCache(pages, heads, dh, pt)
    rot = dj.Rotary((8, 12, 12))
    table, ring = torch.full((n, P), -1, dtype=torch.int32, device="cuda"), torch.arange(pages, dtype=torch.int32, device="cuda")
    lengths, cursor = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.tensor([0, pages, 0], device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    m = [np.full((n, P), -1), np.zeros(n, int), np.arange(pages), np.array([0, pages, 0])]
    lacked = 0
    for counts in steps:
        rows = int(np.maximum(counts, 0).sum()) + 3
        offsets, starts, lengths, cursor, pos, slots = dj.extend(table, lengths, ints(counts), ring, cursor, pt, rows)
        want = model(m[0], m[1], counts, m[2], m[3], pt, rows, np.zeros((rows, 3)), np.zeros(rows))
        m[1], m[3] = np.array(want[2]), np.array(want[3])
        lacked += want[3][2]
        assert np.array_equal(lengths.cpu(), m[1]) and np.array_equal(table.cpu(), m[0])
        held = [p for s in range(n) for p in m[0][s][:-(-m[1][s] // pt)]]
        assert len(set(held)) == len(held)      # no page has two owners
        pos[want[0][-1]:] = 0
        k, v, q = (torch.randn(rows, h, dh, generator=g, device="cuda") for h in (heads, heads, heads * group))
        q = c.write(k, v, starts, offsets, table, rot, pos, q, k_norm=True, q_norm=True)
        got = values(c.attention(q, lengths, offsets, table))
        for s in range(n):
            if counts[s] <= 0 or want[1][s] < 0:
                continue
            length, a = int(m[1][s]), want[0][s]
            out = [x.double().cpu().numpy() for x in c.read(ints([0]), ints([0, length]), table[s:s + 1].contiguous(), rows=length,
                                                            dtype=torch.float32)]
            sees = np.arange(length)[None] <= (length - counts[s] + np.arange(counts[s]))[:, None]
            q64 = values(q)[a:a + counts[s]]
            o, mass, size = ref.attention(q64, *out, sees, dh ** -0.5)
            d = np.abs(got[a:a + counts[s]] - o)
            assert (d <= ref.attention_tolerance(o, mass, size, "f32", dh, length)).all()
    assert (lacked > 0) == (pages < 40)      # the smaller cache runs short


def test_streams_and_answers_about_one_video():
    """Used together: a video's tokens written as a shared prefix; answers whose pages come from the ring, normed, turned and written,
    attending over the prefix and their own places; and streams that see a window of theirs.  Against attention over one table
    of both (whole pages), and against the rows read back."""
    torch = require_gpu()
    heads, group, dh, pt, n, P, pages = 2, 4, 64, 16, 7, 12, 90
    c = dj.TokenCache(pages, heads, dh, pt)
    rot = dj.Rotary((8, 12, 12))
    g = torch.Generator("cuda").manual_seed(2)
    rng = np.random.default_rng(12)
    normal = lambda rows, h: torch.randn(rows, h, dh, generator=g, device="cuda")  # noqa: E731
    ring = torch.arange(pages, dtype=torch.int32, device="cuda")
    table = torch.full((n + 1, P), -1, dtype=torch.int32, device="cuda")
    lengths, cursor = torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.tensor([0, pages, 0], device="cuda")
    video = 9 * pt
    kw, qw = normal(1, heads)[0], normal(1, heads * group)[0]

    def step(counts):
        nonlocal lengths, cursor
        rows = int(np.maximum(counts, 0).sum())
        offsets, starts, lengths, cursor, pos, _ = dj.extend(table, lengths, ints(counts), ring, cursor, pt, rows)
        q = c.write(normal(rows, heads), normal(rows, heads), starts, offsets, table, rot, pos, normal(rows, heads * group), k_norm=kw,
                    q_norm=qw)
        return offsets, q

    step([video] + [0] * n)                       # the video is sequence 0
    prefix, ptable = ints([video]), table[:1].clone()
    for k in range(9):
        counts = np.concatenate([[0], rng.choice([0, 1, 1, 5], n)])
        offsets, q = step(counts)
        assert cursor[2].item() == 0
        if not len(q):
            continue
        own, offs = lengths[1:].contiguous(), offsets[1:].contiguous()
        got = c.attention_shared(q, own, prefix, ptable, offs, table[1:].contiguous())
        both = torch.cat([ptable[:, :9].expand(n, 9), table[1:]], 1).contiguous()
        want = c.attention(q, own + video, offs, both)
        seen = c.attention(q, own, offs, table[1:].contiguous(), window=17, sinks=3)
        for s in range(n):
            a, b, length = offs[s].item(), offs[s + 1].item(), own[s].item()
            if a == b:
                continue
            keys, vals = [values(x) for x in c.read(ints([0]), ints([0, video + length]), both[s:s + 1], rows=video + length,
                                                    dtype=torch.float32)]
            e = (length - (b - a) + np.arange(b - a) + 1)[:, None]
            j = np.arange(length)[None]
            q64 = values(q)[a:b]
            sees = np.concatenate([np.ones((b - a, video), bool), j < e], 1)
            o, mass, size = ref.attention(q64, keys, vals, sees, dh ** -0.5)
            tol = ref.attention_tolerance(o, mass, size, "f32", dh, video + length)
            assert (np.abs(values(got)[a:b] - o) <= tol).all() and (np.abs(values(want)[a:b] - o) <= tol).all()
            o, mass, size = ref.attention(q64, keys[video:], vals[video:], (j < e) & ((j < 3) | (j >= e - 17)), dh ** -0.5)
            assert (np.abs(values(seen)[a:b] - o) <= ref.attention_tolerance(o, mass, size, "f32", dh, length)).all()
    counts = np.full(n + 1, -1)
    counts[0] = 0
    step(counts)                                  # all answers end: the ring holds all but the video's pages
    assert (cursor[1] - cursor[0]).item() == pages - 9 and lengths.tolist() == [video] + [0] * n


def test_captured_steps_replay():
    """A graph of two steps whose lengths and cursor alternate: replayed, it goes on where it stood."""
    torch = require_gpu()
    n, P, pt, pages, rows = 70, 30, 16, 1500, 200
    rng = np.random.default_rng(11)
    counts = [ints(rng.choice([0, 1, 3], n)) for _ in range(2)]
    new = [torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2)]
    cur = [torch.zeros(3, dtype=torch.int64, device="cuda") for _ in range(2)]
    table, ring = torch.full((n, P), -1, dtype=torch.int32, device="cuda"), torch.arange(pages, dtype=torch.int32, device="cuda")
    outs = [(torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), new[1 - i],
             cur[1 - i], torch.zeros(rows, 3, dtype=torch.int32, device="cuda"),
             torch.zeros(rows, dtype=torch.int64, device="cuda")) for i in range(2)]

    def two():
        for i in range(2):
            dj.extend(table, new[i], counts[i], ring, cur[i], pt, rows, out=outs[i])

    def clear():
        table.fill_(-1)
        ring.copy_(torch.arange(pages))
        new[0].zero_()
        cur[0].copy_(torch.tensor([0, pages, 0]))

    clear()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two()
    clear()
    m = [np.full((n, P), -1), np.zeros(n, int), np.arange(pages), np.array([0, pages, 0])]
    for _ in range(5):
        graph.replay()
        for i in range(2):
            w = model(m[0], m[1], counts[i].cpu().numpy(), m[2], m[3], pt, rows, np.zeros((rows, 3)), np.zeros(rows))
            m[1], m[3] = np.array(w[2]), np.array(w[3])
        assert np.array_equal(table.cpu(), m[0]) and np.array_equal(new[0].cpu(), m[1])
        assert np.array_equal(cur[0].cpu(), m[3])
        torch.randn(1000, device="cuda").sum()
