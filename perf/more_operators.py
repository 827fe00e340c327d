"""Performance cases of the operators around the 8-bit cache of keys and values: heads normed and turned
in one pass, on rows and on their way into the cache; attention with a sliding window and first tokens
that stay visible; attention of a batch whose sequences share a long prefix; pages handed out and taken
back on the card, with the maps of a batch's rows.

Definitions (``exact`` computes them in 64 bits):
  norm    every head x of a row becomes x / sqrt(mean(x^2) + eps) * weight (one weight for all heads, or
          one for each) and is then turned: pair i of its ``rot`` leading channels (i and i + rot/2, or 2i
          and 2i + 1) by pos[row, axis(i)] * 10000^(-2i/rot).
  write   keys are normed and turned, then keys and values go to the places start[s] .. of their sequence.
          A page and head has one scale, the least power of two >= 2^-126 with |x| <= 448 scale for what it
          holds; tokens that a page held before are rescaled when the scale grows.  Codes are
          e4m3(x / scale).  Queries are normed and turned beside them.
  window  softmax(q k / sqrt(dh)) v over what a row sees: with e the places up to its own (causal: its
          sequence's rows are the last places) or all of them, place j < e where j < sinks or
          j >= e - window.  A row that sees no key gives 0.
  shared  softmax(q k / sqrt(dh)) v over the places of a prefix that several sequences share, and then the
          sequence's own (causal: its rows are the last of these, and see their own places up to theirs).
  extend  sequence s holds lengths[s] places and gets counts[s] more rows (fewer than 0: it ends).  Rows lie
          one sequence behind the other.  Pages that the new places need come from a ring of free pages,
          cursor = (taken so far, given so far), in order of sequences and places; the pages of
          sequences that end go back to it in the same order.  From the first sequence on that the ring
          does not hold enough for, those that need pages get none: their start is -1 and their length
          stays.  cursor[2] is how many pages were lacking.  Positions are (p, p, p) for place p,
          slots page * page_tokens + p % page_tokens, or -1.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6


def listed():
    return [
        # Queries and keys of a batch of 64 frames of 257 tokens (16 heads of 80 each, one weight for every
        # head), where they lie in the packed rows of a projection.
        dict(name="norm_frames", op="norm", dtype="bf16", rows=16448, heads=32, head_dim=80, rot=80,
             layout="halves", per_head=True, far=64, packed=3840),
        # A few query rows in fp32, one weight for all heads, half of a head turned.
        dict(name="norm_query_f32", op="norm", dtype="f32", rows=5, heads=12, head_dim=64, rot=32,
             layout="pairs", per_head=False, far=100000, packed=0),
        # One new token of each of 48 answers in progress: queries and keys normed and turned, keys and
        # values quantised.
        dict(name="write_norm_tokens", op="write", dtype="bf16", seqs=48, rows=48, pad=0,
             ragged=False, start=6000, kv_heads=8, group=4, head_dim=128, page=64, rot=128,
             per_head=False, lens=1),
        # The tokens of 16 frames of 577, in six clips of different lengths.
        dict(name="write_norm_clips", op="write", dtype="bf16", seqs=6, rows=9232, pad=3, ragged=True,
             start=3000, kv_heads=16, group=1, head_dim=80, page=64, rot=80, per_head=True, lens=2),
        # A serving step of 64 streams of very different lengths: each sees the 257 tokens of its first
        # frame and its last 2048; the pages between are gone.
        dict(name="window_tokens", op="window", dtype="bf16", seqs=64, rows=64, pad=0, ragged=False,
             shortest=1, longest=12000, window=2048, sinks=257, gone=True, causal=True, kv_heads=8,
             group=4, head_dim=128, page=64, lens=3),
        # Prompts of two requests behind long histories.
        dict(name="window_prompt", op="window", dtype="bf16", seqs=2, rows=4096, pad=0, ragged=False,
             shortest=5000, longest=6144, window=1024, sinks=64, gone=False, causal=True, kv_heads=8,
             group=4, head_dim=128, page=64, lens=4),
        # Questions of different lengths in fp32 with short pages and padding, one sequence empty.
        dict(name="window_question_f32", op="window", dtype="f32", seqs=4, rows=333, pad=7, ragged=True,
             shortest=0, longest=1801, window=300, sinks=5, gone=False, causal=True, kv_heads=16,
             group=1, head_dim=80, page=16, lens=5),
        # One token of each of 64 answers about one long video.
        dict(name="shared_tokens", op="shared", dtype="bf16", seqs=64, rows=64, pad=0, ragged=False,
             groups=1, prefix_shortest=50001, prefix_longest=50001, shortest=1, longest=700,
             causal=True, kv_heads=8, group=4, head_dim=128, page=64, lens=6),
        # A few answers about one video: too few rows to fill a large tile.
        dict(name="shared_few", op="shared", dtype="bf16", seqs=8, rows=8, pad=0, ragged=False,
             groups=1, prefix_shortest=100003, prefix_longest=100003, shortest=1, longest=300,
             causal=True, kv_heads=8, group=4, head_dim=128, page=64, lens=7),
        # Questions in fp32 about three clips, one of them empty.
        dict(name="shared_questions_f32", op="shared", dtype="f32", seqs=12, rows=401, pad=5, ragged=True,
             groups=3, prefix_shortest=0, prefix_longest=2056, shortest=0, longest=60, causal=True,
             kv_heads=16, group=1, head_dim=64, page=16, lens=8),
        # A serving step of 256 answers, a few of which have ended.
        dict(name="extend_step", op="extend", seqs=256, rows=256, ended=0.05, held=4000, spare=1.2,
             page=64, lens=9),
        # The prompts of a thousand requests.
        dict(name="extend_prompts", op="extend", seqs=1000, rows=100003, ended=0.1, held=1500, spare=1.1,
             page=16, lens=10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges that the listed ones stand for."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["norm", "write", "window", "window", "shared", "shared", "extend"])
        if op == "extend":
            seqs = _log_int(rng, 1, 4000)
            return dict(op=op, seqs=seqs, rows=max(1, _log_int(rng, seqs, 100000)),
                        ended=rng.choice([0.0, 0.05, 0.3]), held=_log_int(rng, 1, 5000),
                        spare=rng.choice([0.5, 1.0, 1.5]), page=rng.choice([16, 32, 64, 128]),
                        lens=rng.randrange(1 << 30))
        f32 = rng.random() < 0.25
        dh = rng.choice([16, 32, 48, 64, 64, 80, 96, 112, 128, 128])
        c = dict(op=op, dtype="f32" if f32 else "bf16", head_dim=dh)
        if op == "norm":
            c.update(rows=_log_int(rng, 1, 20000), heads=rng.choice([1, 8, 12, 16, 24, 32, 40]),
                     rot=rng.choice([0, dh, dh, max(2, dh // 4 * 2)]),
                     layout=rng.choice(["halves", "pairs"]), per_head=rng.random() < 0.5,
                     far=_log_int(rng, 2, 1 << 30), packed=0)
            if rng.random() < 0.5:
                c["packed"] = c["heads"] * dh + rng.choice([dh, 8, 1024])
        else:
            seqs = _log_int(rng, 1, 128)
            c.update(seqs=seqs, kv_heads=rng.choice([1, 2, 3, 4, 8, 12, 16]),
                     page=rng.choice([16, 32, 64, 64, 128]), pad=rng.choice([0, 0, 5]),
                     ragged=rng.random() < 0.6, group=rng.choice([1, 1, 2, 4, 5, 8, 16]),
                     lens=rng.randrange(1 << 30))
            single = rng.random() < 0.5
            if single:
                c["ragged"] = False
            rows = seqs if single else max(seqs, _log_int(rng, seqs, 20000))
            if op != "write" and not single:
                rows = max(seqs, min(rows, 4096))
            c["rows"] = rows if c["ragged"] else rows // seqs * seqs
            if op == "write":
                c.update(start=_log_int(rng, 1, 20000), rot=rng.choice([0, dh, dh // 4 * 2]),
                         per_head=rng.random() < 0.5)
            least = 1 if rng.random() < 0.2 else -(-2 * rows // seqs)   # mostly, every row sees something
            if op == "window":
                longest = max(least, _log_int(rng, 1, 50000 if seqs < 4 else 12000))
                c.update(longest=longest, shortest=rng.choice([0, 1, longest // 2, longest]),
                         window=_log_int(rng, 1, 5000), sinks=rng.choice([0, 1, 4, 64, 257, 1000]),
                         causal=rng.random() < 0.7, gone=rng.random() < 0.5)
            elif op == "shared":
                prefix, longest = _log_int(rng, 1, 100000), max(least, _log_int(rng, 1, 2000))
                c.update(groups=min(seqs, rng.choice([1, 1, 2, 5])), prefix_longest=prefix,
                         prefix_shortest=rng.choice([0, prefix // 2, prefix]), longest=longest,
                         shortest=rng.choice([0, 1, longest]), causal=rng.random() < 0.7)
        if _cost(c) <= most and _room(c):
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 5e14)


def _room(c):
    """Whether the plain form's padded tensors stay small enough."""
    if c["op"] in ("norm", "extend"):
        return True
    s = _sizes(c)
    wide = c["kv_heads"] * c["head_dim"]
    pool = c["seqs"] * s["table_pages"] * c["page"] * wide
    if c["op"] == "write":
        return pool <= 1 << 29
    scores = c["seqs"] * c["kv_heads"] * c["group"] * max(s["counts"]) * s["table_pages"] * c["page"]
    if c["op"] == "shared":
        pool += c["groups"] * s["prefix_pages"] * c["page"] * wide
        scores += c["groups"] * c["kv_heads"] * c["group"] * max(s["group_rows"]) * s["prefix_pages"] * c["page"]
    return pool <= 1 << 30 and scores <= 1 << 31 and 4 * scores * c["head_dim"] <= 4e12 and \
        (c["dtype"] == "bf16" or work(c)["flops"] <= 1e11)


# ---- sizes ---------------------------------------------------------------------------------------
def _cuts(rng, total, n, least):
    """n numbers of at least `least` that add up to `total`."""
    cuts = sorted(rng.randint(0, total - least * n) for _ in range(n - 1))
    return [b - a + least for a, b in zip([0] + cuts, cuts + [total - least * n])]


def _sizes(c):
    """Rows of each sequence, where they start, and how long it is after them."""
    rng = random.Random(c["lens"])
    n, rows = c["seqs"], c["rows"]
    if c["op"] == "extend":
        ended = [rng.random() < c["ended"] for _ in range(n)]
        ended[rng.randrange(n)] = False
        cuts = _cuts(rng, rows, n, rows // (2 * n))
        counts = [-1 if e else k for e, k in zip(ended, cuts)]
        lengths = [rng.randint(0, c["held"]) for _ in range(n)]
        after = [a + max(k, 0) for a, k in zip(lengths, counts)]
        pages = [-(-x // c["page"]) for x in after]
        held = [-(-x // c["page"]) for x in lengths]
        return dict(counts=counts, lengths=lengths, held=held, table_pages=max(1, max(pages)),
                    need=sum(pages) - sum(held))
    counts = _cuts(rng, rows, n, 1) if c["ragged"] else [rows // n] * n
    if c["op"] == "write":
        starts = [rng.randint(0, c["start"]) for _ in range(n)]
        lengths = [a + k for a, k in zip(starts, counts)]
    else:
        lengths = [rng.randint(c["shortest"], c["longest"]) for _ in range(n)]
        if n > 1 and c["shortest"] < c["longest"]:
            lengths[rng.randrange(n)] = c["longest"]
            if c["shortest"] == 0:
                lengths[(lengths.index(c["longest"]) + 1) % n] = 0
        starts = [length - k for length, k in zip(lengths, counts)]
    s = dict(counts=counts, starts=starts, lengths=lengths,
             table_pages=max(1, max(-(-x // c["page"]) for x in lengths)))
    if c["op"] == "shared":
        members = _cuts(rng, n, c["groups"], 1)
        first = [sum(members[:g]) for g in range(c["groups"] + 1)]
        prefix = [rng.randint(c["prefix_shortest"], c["prefix_longest"]) for _ in members]
        prefix[0] = c["prefix_longest"]
        if c["prefix_shortest"] == 0 and len(prefix) > 1:
            prefix[-1] = 0
        s.update(groups=first, prefix=prefix, prefix_pages=max(1, max(-(-x // c["page"]) for x in prefix)),
                 group_rows=[sum(counts[a:b]) for a, b in zip(first, first[1:])])
    return s


def _pairs(count, length, causal):
    """Query rows times keys that they see, of a sequence."""
    if not causal:
        return count * length
    first = max(length - count + 1, 1)
    return (first + length) * (length - first + 1) // 2


def work(case):
    c = case
    if c["op"] == "extend":
        s = _sizes(c)
        return {"bytes": 20 * c["seqs"] + 8 * s["need"] + 20 * sum(max(k, 0) for k in s["counts"]),
                "flops": 4 * c["rows"]}
    el, dh = SIZE[c["dtype"]], c["head_dim"]
    if c["op"] == "norm":
        n = c["rows"] * c["heads"]
        return {"bytes": 2 * n * dh * el + (12 * c["rows"] if c["rot"] else 0),
                "flops": 4 * n * dh + 3 * n * c["rot"]}
    s = _sizes(c)
    rows, hd = c["rows"], c["kv_heads"] * dh
    if c["op"] == "write":
        return {"bytes": rows * (2 * hd * (el + 1) + 2 * c["group"] * hd * el) + (12 * rows if c["rot"] else 0),
                "flops": rows * hd * (4 + 4 * (c["group"] + 1) + (3 * (c["group"] + 1) if c["rot"] else 0))}
    heads = c["kv_heads"] * c["group"]
    pairs, keys = 0, 0
    for k, length in zip(s["counts"], s["lengths"]):
        if c["op"] == "shared":
            keys += length
            pairs += _pairs(k, length, c["causal"])
            continue
        for i in range(k):
            e = max(0, length - k + i + 1) if c["causal"] else length
            pairs += min(e, min(e, c["sinks"]) + min(c["window"], max(0, e - c["sinks"])))
        first = max(0, length - k + 1) if c["causal"] else length
        low = max(0, first - c["window"])
        keys += min(length, min(c["sinks"], low) + length - low)
    if c["op"] == "shared":
        keys += sum(s["prefix"])
        pairs += sum(a * b for a, b in zip(s["prefix"], s["group_rows"]))
    return {"bytes": keys * 2 * hd + 2 * rows * heads * dh * el, "flops": 4 * dh * heads * pairs}


# ---- inputs --------------------------------------------------------------------------------------
def _sections(rot):
    pairs = rot // 2
    h = pairs // 3
    return [pairs - 2 * h, h, h]


def _layout(c):
    return c.get("layout", "halves")


def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(dev).manual_seed(seed)
    if c["op"] == "extend":
        return _prepare_extend(c, g, dev)
    dt, dh = TYPES[c["dtype"]], c["head_dim"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev).to(dt)

    def weight(heads):
        shape = (heads, dh) if c["per_head"] else (dh,)
        return (1 + 0.3 * torch.randn(*shape, generator=g, device=dev)).to(dt)

    st = {"case": dict(c)}
    if c["op"] == "norm":
        rows, wide = c["rows"], c["heads"] * dh
        x = normal(rows, max(wide, c["packed"]))
        x *= torch.exp(torch.randn(rows, 1, generator=g, device=dev)).to(dt)
        st["x"] = x[:, :wide].unflatten(1, (c["heads"], dh))
        st["weight"] = weight(c["heads"])
        st["pos"] = torch.randint(0, c["far"], (rows, 3), generator=g, device=dev, dtype=torch.int32)
        return st

    s = _sizes(c)
    n, H, pt, P = c["seqs"], c["kv_heads"], c["page"], s["table_pages"]
    PP = s["prefix_pages"] if c["op"] == "shared" else 0
    shared = c["groups"] * PP if PP else 0
    total = n * P + shared + 3
    for name in ("k", "v"):
        shape = (total, H, pt, dh) if name == "k" else (total, H, dh, pt)
        codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device=dev)
        for a in range(0, total, 4096):     # a part at a time: the fp32 values are larger
            part = codes[a:a + 4096]
            part.copy_((torch.randn(part.shape, generator=g, device=dev) * 100).clamp_(-448, 448))
        st[name + "_pages"] = codes
        st[name + "_scale"] = torch.exp2(torch.randint(-9, -5, (total, H), generator=g,
                                                       device=dev).float())
    # pages in no order; places past a sequence's last page hold no page
    order = torch.randperm(total, generator=g, device=dev)
    used = torch.tensor([-(-x // pt) for x in s["lengths"]], device=dev)[:, None]
    page = torch.arange(P, device=dev)[None]
    there = page < used
    if c.get("gone"):   # nor do those that no row sees any more
        length = torch.tensor(s["lengths"], device=dev)[:, None]
        count = torch.tensor(s["counts"], device=dev)[:, None]
        low = (length - count + 1 if c["causal"] else length) - c["window"]
        there &= (page * pt < c["sinks"]) | ((page + 1) * pt > low)
    st["table"] = torch.where(there, order[:n * P].view(n, P), -1).to(torch.int32)
    offs = [0]
    for k in s["counts"]:
        offs.append(offs[-1] + k)
    st["offsets"] = torch.tensor(offs, dtype=torch.int32, device=dev)
    st["starts"] = torch.tensor(s["starts"], dtype=torch.int32, device=dev)
    st["lengths"] = torch.tensor(s["lengths"], dtype=torch.int32, device=dev)
    rows = c["rows"] + c["pad"]
    st["rows"], st["most"] = rows, max(s["counts"])
    # the plain forms' index lists: sequence of each row, its place among the sequence's rows
    st["seq"] = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(s["counts"], device=dev))
    st["rank"] = torch.arange(c["rows"], device=dev) - st["offsets"][st["seq"]]
    if c["op"] != "write":
        st["q"] = normal(rows, H * c["group"], dh)
        st["out"] = torch.zeros(rows, H * c["group"], dh, dtype=dt, device=dev)
        if PP:
            st["groups"] = torch.tensor(s["groups"], dtype=torch.int32, device=dev)
            st["prefix_lengths"] = torch.tensor(s["prefix"], dtype=torch.int32, device=dev)
            used = torch.tensor([-(-x // pt) for x in s["prefix"]], device=dev)[:, None]
            st["prefix_table"] = torch.where(torch.arange(PP, device=dev)[None] < used,
                                             order[n * P:n * P + shared].view(-1, PP), -1).to(torch.int32)
            st["group_offsets"] = st["offsets"][st["groups"].long()]
            st["row_group"] = torch.repeat_interleave(torch.arange(c["groups"], device=dev),
                                                      torch.tensor(s["group_rows"], device=dev))
            st["group_rank"] = torch.arange(c["rows"], device=dev) - st["group_offsets"][st["row_group"]]
            st["group_most"] = max(s["group_rows"])
        return st
    # write: queries, keys and values lie side by side in the rows of one projection
    heads = c["group"] * H
    qkv = normal(rows, (heads + 2 * H) * dh)
    qkv[:, heads * dh:] *= torch.exp(torch.randn(1, 2 * H * dh, generator=g, device=dev)).to(dt)
    q, k, v = qkv.split([heads * dh, H * dh, H * dh], 1)
    st["q"], st["k_new"], st["v_new"] = (x.unflatten(1, (-1, dh)) for x in (q, k, v))
    st["q_out"] = torch.zeros(rows, heads, dh, dtype=dt, device=dev)
    st["k_weight"], st["q_weight"] = weight(H), weight(heads)
    # tokens that follow one another in a clip of 16 x 16 patches a frame
    at = int(torch.randint(0, 100000, (1,), generator=g, device=dev)) + torch.arange(rows, device=dev)
    st["pos"] = torch.stack([at // 256, at // 16 % 16, at % 16], 1).to(torch.int32)
    st["at"] = st["rank"] + st["starts"][st["seq"]]
    # the pages written, in order of the rows, and what each held before
    unit, keep, pages = {}, [], []
    for q_, (k_, a) in enumerate(zip(s["counts"], s["starts"])):
        for p in range(a // pt, (a + k_ - 1) // pt + 1):
            unit[q_, p] = len(keep)
            keep.append(max(0, a - p * pt))
            pages.append((q_, p))
    first_unit = torch.tensor([unit[q_, a // pt] for q_, a in enumerate(s["starts"])], device=dev)
    st["unit"] = first_unit[st["seq"]] + st["at"] // pt - (st["starts"] // pt)[st["seq"]]
    st["keep"] = torch.tensor(keep, device=dev)
    pq = torch.tensor(pages, device=dev)
    st["unit_page"] = st["table"][pq[:, 0], pq[:, 1]].long()
    return st


def _prepare_extend(c, g, dev):
    s = _sizes(c)
    n, P = c["seqs"], s["table_pages"]
    spare = max(1, int(s["need"] * c["spare"]))
    total = sum(s["held"]) + spare
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)
    held = torch.tensor(s["held"], device=dev)
    page = torch.arange(P, device=dev)[None]
    at = (torch.cumsum(held, 0) - held)[:, None] + page
    st = {"case": dict(c), "pages": total}
    st["table"] = torch.where(page < held[:, None], order[at.clamp(max=total - 1)], -1)
    # free pages stand somewhere in the ring, round its end
    taken = int(torch.randint(0, 1 << 20, (1,), generator=g, device=dev))
    ring = torch.full((total,), -1, dtype=torch.int32, device=dev)
    ring[(taken + torch.arange(spare, device=dev)) % total] = order[total - spare:]
    st["ring"] = ring
    st["cursor"] = torch.tensor([taken, taken + spare, 0], dtype=torch.int64, device=dev)
    st["counts"] = torch.tensor(s["counts"], dtype=torch.int32, device=dev)
    st["lengths"] = torch.tensor(s["lengths"], dtype=torch.int32, device=dev)
    rows = c["rows"]
    st["out"] = {"offsets": torch.zeros(n + 1, dtype=torch.int32, device=dev),
                 "starts": torch.zeros(n, dtype=torch.int32, device=dev),
                 "lengths": torch.zeros(n, dtype=torch.int32, device=dev),
                 "cursor": torch.zeros(3, dtype=torch.int64, device=dev),
                 "positions": torch.zeros(rows, 3, dtype=torch.int32, device=dev),
                 "slots": torch.zeros(rows, dtype=torch.int64, device=dev)}
    return st


# ---- plain forms ---------------------------------------------------------------------------------
def _turn(x, pos, rot, layout):
    """Rotary positions of fp32 rows [T, H, dh] (angles in 64 bits)."""
    if not rot:
        return x
    i = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    axis = torch.repeat_interleave(torch.arange(3, device=x.device),
                                   torch.tensor(_sections(rot), device=x.device), output_size=rot // 2)
    angle = pos.double()[:, axis] * 10000.0 ** (-2 * i / rot)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if layout == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2),
                      x[..., rot:]], -1)


def _norm(x, weight):
    """Rows [T, H, dh] normed in fp32."""
    y = x.float()
    return y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()


def _norm_turn(x, weight, pos, c):
    return _turn(_norm(x, weight), pos, c["rot"], _layout(c))


def _scale_of(most):
    """The least power of two >= 2^-126 whose 448-fold is at least `most`."""
    m, e = torch.frexp(most)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
    return torch.ldexp(torch.ones_like(most), torch.where(most > 0, e, -126))


def _put(x, pages, scale, st, tokens_first):
    """Quantises rows x [T, H, dh] into pages in place."""
    pt = st["case"]["page"]
    unit, upage, keep = st["unit"], st["unit_page"], st["keep"]
    most = torch.zeros(len(keep), x.shape[1], device=x.device)
    most.index_reduce_(0, unit, x.abs().amax(-1), "amax")
    old = torch.where(keep[:, None] > 0, scale[upage], 0.0)
    new = torch.maximum(old, _scale_of(most))
    held = torch.arange(pt, device=x.device) < keep[:, None]
    held = held[:, None, :, None] if tokens_first else held[:, None, None, :]
    bytes_ = pages.view(torch.uint8)
    before = bytes_[upage]
    grown = before.view(torch.float8_e4m3fn).float() * (old / new)[:, :, None, None]
    bytes_[upage] = torch.where(held, grown.to(torch.float8_e4m3fn).view(torch.uint8), before)
    codes = (x / new[unit][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    if tokens_first:
        bytes_[upage[unit], :, st["at"] % pt] = codes
    else:
        bytes_[upage[unit], :, :, st["at"] % pt] = codes
    scale[upage] = new


def _write(st):
    c, n = st["case"], st["case"]["rows"]
    pos = st["pos"][:n]
    st["q_out"][:n] = _norm_turn(st["q"][:n], st["q_weight"], pos, c).to(st["q"].dtype)
    _put(_norm_turn(st["k_new"][:n], st["k_weight"], pos, c), st["k_pages"], st["k_scale"], st, True)
    _put(st["v_new"][:n].float(), st["v_pages"], st["v_scale"], st, False)


def _history(st, table):
    """Keys and values [n, H, places, dh] of the table's sequences in fp32."""
    c = st["case"]
    n, P = table.shape
    table = table.clamp(min=0).long()
    shape = (n, c["kv_heads"], P * c["page"], c["head_dim"])
    k = st["k_pages"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()
    k = (k * st["k_scale"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(shape)
    v = st["v_pages"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()
    v = (v * st["v_scale"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(shape)
    return k, v


def _softmax_part(st, table, offsets, most, sees, seq, rank):
    """Maxima [rows, H, G, 1], sums and products with the values of rows that lie together: `most` at most
    from offsets[s] on; sees(i, key) says which keys the i-th of them does not see."""
    c = st["case"]
    n, H, G, dh = len(table), c["kv_heads"], c["group"], c["head_dim"]
    k, v = _history(st, table)
    i = torch.arange(most, device=k.device)[None]
    row = (offsets[:-1, None] + i).clamp(max=st["rows"] - 1).long()
    q = st["q"][row].float().unflatten(2, (H, G))                  # n, most, H, G, dh
    q = q.permute(0, 2, 3, 1, 4).reshape(n, H, G * most, dh)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1 / math.sqrt(dh))
    key = torch.arange(k.shape[2], device=k.device)
    s = s.unflatten(2, (G, most)).masked_fill(~sees(i[:, :, None], key)[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = (s - top.where(top > -math.inf, torch.zeros_like(top))).exp()
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, most))
    return [x.permute(0, 3, 1, 2, 4)[seq, rank] for x in (top, p.sum(-1, keepdim=True), o)]


def _sees(st, i, length):
    """Places that the i-th row of each sequence sees, were there no window."""
    count = (st["offsets"][1:] - st["offsets"][:-1])[:, None, None]
    length = length[:, None, None]
    return length - count + i + 1 if st["case"]["causal"] else length + 0 * i


def _rows_out(st, o, total):
    n = st["case"]["rows"]
    st["out"][:n] = (o / total.where(total > 0, torch.ones_like(total))).flatten(1, 2).to(st["q"].dtype)
    return st["out"]


def _window(st):
    c = st["case"]

    def sees(i, key):
        e = _sees(st, i, st["lengths"])
        return (key < e) & ((key < c["sinks"]) | (key >= e - c["window"]))

    _, total, o = _softmax_part(st, st["table"], st["offsets"], st["most"], sees, st["seq"], st["rank"])
    return _rows_out(st, o, total)


def _shared(st):
    m0, l0, o0 = _softmax_part(st, st["prefix_table"], st["group_offsets"], st["group_most"],
                               lambda i, key: key < st["prefix_lengths"][:, None, None] + 0 * i,
                               st["row_group"], st["group_rank"])
    m1, l1, o1 = _softmax_part(st, st["table"], st["offsets"], st["most"],
                               lambda i, key: key < _sees(st, i, st["lengths"]), st["seq"], st["rank"])
    top = torch.maximum(m0, m1)
    top = top.where(top > -math.inf, torch.zeros_like(top))
    a, b = (m0 - top).exp(), (m1 - top).exp()
    return _rows_out(st, o0 * a + o1 * b, l0 * a + l1 * b)


def _extend(st):
    c, out, dev = st["case"], st["out"], st["table"].device
    pt, pages, rows, P = c["page"], st["pages"], c["rows"], st["table"].shape[1]
    counts, lengths = st["counts"].long(), st["lengths"].long()
    taken, given = st["cursor"][0], st["cursor"][1]
    room = given - taken
    new = counts.clamp(min=0)
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(new, 0)])
    held, after = (lengths + pt - 1) // pt, (lengths + new + pt - 1) // pt
    want = after - held
    upto = torch.cumsum(want, 0)
    served = (want == 0) | (upto <= room)
    ends = counts < 0
    page = torch.arange(P, device=dev)[None]
    # pages that go back: those of the sequences that end
    back = ends[:, None] & (page < held[:, None]) & (st["table"] >= 0) & (st["table"] < pages)
    place = torch.cumsum(back.flatten().long(), 0) - 1
    count_back = torch.minimum(place[-1] + 1, pages - room)
    goes = back.flatten() & (place < pages - room)
    ring = st["ring"].clone()
    at = torch.where(goes, (given + place) % pages, pages)
    st["ring"] = torch.cat([ring, ring.new_zeros(1)]).scatter(0, at, st["table"].flatten())[:pages]
    # pages handed out
    gets = served[:, None] & (page >= held[:, None]) & (page < after[:, None])
    source = (taken + (upto - want)[:, None] + page - held[:, None]) % pages
    st["table"].copy_(torch.where(gets, ring[source], st["table"]))
    out["offsets"].copy_(offsets)
    out["starts"].copy_(torch.where(served & ~ends, lengths, -1))
    out["lengths"].copy_(torch.where(ends, 0, torch.where(served, lengths + new, lengths)))
    got = torch.where(served, want, 0).sum()
    out["cursor"].copy_(torch.stack([taken + got, given + count_back, want.sum() - got]))
    row = torch.arange(rows, device=dev)
    seq = torch.searchsorted(offsets[1:], row, right=True)
    inside = seq < len(counts)
    seq = seq.clamp(max=len(counts) - 1)
    p = lengths[seq] + row - offsets[seq]
    entry = st["table"][seq, (p // pt).clamp(max=P - 1)].long()
    slot = torch.where(served[seq] & (entry >= 0) & (entry < pages), entry * pt + p % pt, -1)
    out["positions"].copy_(torch.where(inside, p, out["positions"][:, 0])[:, None].expand(-1, 3))
    out["slots"].copy_(torch.where(inside, slot, out["slots"]))
    return {"table": st["table"], "ring": st["ring"], **out}


# ---- one pass ------------------------------------------------------------------------------------
def _kept(st):
    """What a program keeps between calls: the cache over its pages, the rotary positions' rates."""
    from paper_2506_14107_amd import dejavu
    c = st["case"]
    if c["op"] == "extend":
        st["call"] = dejavu
        return
    if c["op"] != "norm":
        st["cache"] = dejavu.TokenCache(
            st["k_pages"].shape[0], c["kv_heads"], c["head_dim"], c["page"],
            buffers=(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"]))
    rot = c.get("rot", 0)
    st["rotary"] = dejavu.Rotary(_sections(rot), layout=_layout(c)) if rot else None
    st["call"] = dejavu


def run(state):
    st, c = state, state["case"]
    if not own:
        if c["op"] == "norm":
            return _norm_turn(st["x"], st["weight"], st["pos"], c).to(st["x"].dtype)
        if c["op"] == "window":
            return _window(st)
        if c["op"] == "shared":
            return _shared(st)
        if c["op"] == "extend":
            return _extend(st)
        _write(st)
    else:
        if "call" not in st:
            _kept(st)
        if c["op"] == "extend":
            out = st["out"]
            st["call"].extend(st["table"], st["lengths"], st["counts"], st["ring"], st["cursor"],
                              c["page"], c["rows"], out=(out["offsets"], out["starts"], out["lengths"],
                                                         out["cursor"], out["positions"], out["slots"]))
            return {"table": st["table"], "ring": st["ring"], **out}
        pos = st["pos"] if st.get("rotary") else None
        if c["op"] == "norm":
            return st["call"].norm_rotary(st["x"], st["weight"], EPS, pos, st["rotary"])
        if c["op"] == "window":
            return st["cache"].attention(st["q"], st["lengths"], st["offsets"], st["table"],
                                         causal=c["causal"], max_rows=st["most"], out=st["out"],
                                         window=c["window"], sinks=c["sinks"])
        if c["op"] == "shared":
            return st["cache"].attention_shared(
                st["q"], st["lengths"], st["prefix_lengths"], st["prefix_table"], st["offsets"],
                st["table"], st["groups"], causal=c["causal"], max_rows=st["most"], out=st["out"])
        st["cache"].write(st["k_new"], st["v_new"], st["starts"], st["offsets"], st["table"],
                          rotary=st["rotary"], positions=pos, q=st["q"], q_out=st["q_out"],
                          k_norm=st["k_weight"], q_norm=st["q_weight"], eps=EPS)
    return {"q": st["q_out"], "k": st["k_pages"], "v": st["v_pages"], "k_scale": st["k_scale"],
            "v_scale": st["v_scale"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _e4m3(x):
    """Nearest value of one sign, four exponent and three fraction bits, ties to even (|x| <= 448)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_norm(x, weight, pos, c):
    x = x.double()
    x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    y, rot, pair = x.clone(), c["rot"], 0
    for axis, size in enumerate(_sections(rot)):
        for _ in range(size):
            a = pos[:, axis].double()[:, None] * 10000.0 ** (-2 * pair / rot)
            i0, i1 = (pair, pair + rot // 2) if _layout(c) == "halves" else (2 * pair, 2 * pair + 1)
            y[..., i0] = x[..., i0] * a.cos() - x[..., i1] * a.sin()
            y[..., i1] = x[..., i1] * a.cos() + x[..., i0] * a.sin()
            pair += 1
    return y


def _exact_pages(st, name, x):
    """Pages and scales after the write of rows x, sequence by sequence."""
    c, s = st["case"], _sizes(st["case"])
    pages = st[name + "_pages"].double()
    if name == "v":
        pages = pages.transpose(2, 3).contiguous()
    scale, pt = st[name + "_scale"].double(), c["page"]
    table, row = st["table"].tolist(), 0
    for q, (count, start) in enumerate(zip(s["counts"], s["starts"])):
        done = 0
        while done < count:
            at = start + done
            page, slot = table[q][at // pt], at % pt
            k = min(count - done, pt - slot)
            new = x[row:row + k].transpose(0, 1)                       # H, k, dh
            most = new.abs().amax((1, 2)).clamp(min=1e-300) / 448
            size = torch.exp2(torch.ceil(torch.log2(most)).clamp(min=-126))
            if slot:
                size = torch.maximum(size, scale[page])
                pages[page, :, :slot] = _e4m3(pages[page, :, :slot] *
                                              (scale[page] / size)[:, None, None])
            pages[page, :, slot:slot + k] = _e4m3(new / size[:, None, None])
            scale[page] = size
            done, row = done + k, row + k
    return (pages if name == "k" else pages.transpose(2, 3).contiguous()), scale


def _exact_extend(st):
    """Sequence by sequence, page by page."""
    c, s, pages = st["case"], _sizes(st["case"]), st["pages"]
    pt = c["page"]
    table, ring = st["table"].cpu().numpy().copy(), st["ring"].cpu().numpy().copy()
    taken, given, _ = st["cursor"].tolist()
    free = [int(ring[i % pages]) for i in range(taken, given)]
    lack, short, row, room = 0, False, 0, given - taken
    offsets, starts, lengths = [0], [], []
    positions, slots = st["out"]["positions"].cpu().numpy().copy(), st["out"]["slots"].cpu().numpy().copy()
    for q, (k, a) in enumerate(zip(s["counts"], s["lengths"])):
        held, new = -(-a // pt), max(k, 0)
        need = -(-(a + new) // pt) - held
        short = short or need > len(free)
        if k < 0:
            for page in table[q, :held]:
                if 0 <= page < pages and given - taken < pages:
                    ring[given % pages] = page
                    given += 1
        got = not (short and need)
        if got:
            table[q, held:held + need] = free[:need]
            free = free[need:]
        else:
            lack += need
        starts.append(a if got and k >= 0 else -1)
        lengths.append(0 if k < 0 else a + new if got else a)
        for i in range(new):
            page = int(table[q, (a + i) // pt]) if got else -1
            positions[row + i] = a + i
            slots[row + i] = page * pt + (a + i) % pt if page >= 0 else -1
        row += new
        offsets.append(row)
    return {"table": table, "ring": ring, "offsets": offsets, "starts": starts, "lengths": lengths,
            "cursor": [taken + room - len(free), given, lack], "positions": positions, "slots": slots}


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    dev = "cuda"
    if c["op"] == "extend":
        of = {k: v.dtype for k, v in st["out"].items()}
        return {k: torch.as_tensor(v, dtype=of.get(k, torch.int32), device=dev)
                for k, v in _exact_extend(st).items()}
    if c["op"] == "norm":
        return _exact_norm(st["x"], st["weight"], st["pos"], c)
    n, s = c["rows"], _sizes(c)
    if c["op"] == "write":
        q = torch.zeros(st["q_out"].shape, dtype=torch.float64, device=dev)
        q[:n] = _exact_norm(st["q"], st["q_weight"], st["pos"], c)[:n]
        k = _exact_norm(st["k_new"], st["k_weight"], st["pos"], c)
        (kp, ks), (vp, vs) = _exact_pages(st, "k", k), _exact_pages(st, "v", st["v_new"].double())
        return {"q": q, "k": kp, "v": vp, "k_scale": ks, "v_scale": vs}
    H, G, dh, pt = c["kv_heads"], c["group"], c["head_dim"], c["page"]

    def history(table, length):
        """Keys and values [H, length, dh] of one sequence."""
        pages = table[:-(-length // pt)].long().clamp(min=0)
        k = st["k_pages"][pages].double() * st["k_scale"][pages].double()[:, :, None, None]
        v = st["v_pages"][pages].double() * st["v_scale"][pages].double()[:, :, None, None]
        return [x.reshape(H, -1, dh)[:, :length] for x in
                (k.permute(1, 0, 2, 3), v.permute(1, 0, 3, 2))]

    o = torch.zeros(st["out"].shape, dtype=torch.float64, device=dev)
    row, group = 0, -1
    for q, (count, length) in enumerate(zip(s["counts"], s["lengths"])):
        k, v = history(st["table"][q], length)
        P = 0
        if c["op"] == "shared":
            g = max(i for i in range(c["groups"]) if s["groups"][i] <= q)
            if g != group:
                group, prefix = g, history(st["prefix_table"][g], s["prefix"][g])
            P = s["prefix"][g]
            k, v = torch.cat([prefix[0], k], 1), torch.cat([prefix[1], v], 1)
        key = torch.arange(P + length, device=dev) - P       # places; those of the prefix below 0
        for a in range(0, count, 512):
            b = min(count, a + 512)
            qs = st["q"][row + a:row + b].double().unflatten(1, (H, G)).permute(1, 2, 0, 3)
            logits = torch.matmul(qs.flatten(1, 2), k.transpose(1, 2)) / math.sqrt(dh)
            logits = logits.unflatten(1, (G, b - a))
            e = torch.arange(a, b, device=dev)[:, None] + length - count + 1 if c["causal"] else \
                torch.full((b - a, 1), length, device=dev)
            hidden = (key >= e) & (key >= 0)
            if c["op"] == "window":
                hidden |= (key >= c["sinks"]) & (key < e - c["window"])
            p = torch.softmax(logits.masked_fill_(hidden, -math.inf), -1).nan_to_num(0.0)
            o[row + a:row + b] = torch.matmul(p.flatten(1, 2), v).unflatten(1, (G, b - a)) \
                .permute(2, 0, 1, 3).flatten(1, 2)
        row += count
    return o
