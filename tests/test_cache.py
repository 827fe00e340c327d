"""Rotary positions and the 8-bit cache on the CPU: what the entry points refuse, before any GPU
work, and where rows, pages and tiles go."""
import ctypes
import math
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from paper_2506_14107_amd import dejavu as dj

from . import test_gpu_cache as on_gpu

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2506_14107_amd", "csrc")
FAKE = 1 << 20   # an aligned address that nothing may touch


# ---- rates ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("sections,per_axis,base", [((8, 12, 12), False, 1e4), ((0, 16, 16), True, 100.0),
                                                    ((64, 0, 0), False, 5e5), ((1, 0, 0), True, 1.0)])
def test_rotary_rates(sections, per_axis, base):
    """2^64 / (2 pi) times the rate, rounded to a whole number (half a unit) after a few roundings in
    more than 53 bits; the expected value has a few in 53."""
    plan = dj.Rotary(sections, per_axis=per_axis, base=base).plan
    assert plan.dim == 2 * sum(sections) and tuple(plan.section) == sections
    i = 0
    for s in sections:
        for j in range(s):
            rate = base ** (-j / s) if per_axis else base ** (-2 * i / plan.dim)
            want = rate / (2 * math.pi) * 2.0 ** 64
            assert abs(plan.turn[i] - want) <= want * 2.0 ** -50 + 0.5, (i, plan.turn[i], want)
            i += 1
    assert all(t == 0 for t in plan.turn[i:])


@pytest.mark.parametrize("kw", [dict(sections=(0, 0, 0)), dict(sections=(65, 0, 0)),
                                dict(sections=(-1, 2, 2)), dict(base=0.5), dict(base=math.nan),
                                dict(base=math.inf)])
def test_rotary_init_refuses(kw):
    with pytest.raises(dj.DejaVuError) as e:
        dj.Rotary(**dict(dict(sections=(4, 4, 4)), **kw))
    assert e.value.code == dj.DV_EINVAL


def test_rotary_init_refuses_unknown_layouts_and_nulls():
    lib = dj.load()
    sec = (ctypes.c_int * 3)(4, 4, 4)
    plan = dj.dv_rotary_plan()
    assert lib.dv_rotary_init(ctypes.byref(plan), ctypes.byref(sec), 2, 0, 1e4) == dj.DV_EINVAL
    assert lib.dv_rotary_init(None, ctypes.byref(sec), 0, 0, 1e4) == dj.DV_EINVAL
    assert lib.dv_rotary_init(ctypes.byref(plan), None, 0, 0, 1e4) == dj.DV_EINVAL
    with pytest.raises(ValueError):
        dj.Rotary((4, 4, 4), layout="other")
    with pytest.raises(ValueError):
        dj.Rotary((4, 4))


# ---- refusals ------------------------------------------------------------------------------------
ROT = dj.Rotary((8, 12, 12))
WIDE_ROT = dj.Rotary((16, 24, 24))
BLANK = dj.dv_rotary_plan()


def call_rotary(**kw):
    a = dict(plan=ROT.address, dtype=dj.DV_BF16, x=FAKE, x_stride=256, rows=5, heads=4, head_dim=64,
             positions=FAKE, out=2 * FAKE, out_stride=256)
    a.update(kw)
    return dj.load().dv_rotary(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(plan=None), dict(plan=ctypes.addressof(BLANK)), dict(dtype=2), dict(x=None), dict(positions=None),
    dict(out=None), dict(rows=-1), dict(heads=0), dict(head_dim=0), dict(head_dim=62),
    dict(head_dim=65, x_stride=512, out_stride=512), dict(x_stride=255), dict(out_stride=255),
    dict(out=FAKE, x_stride=512), dict(rows=1 << 30, heads=32, x_stride=2048, out_stride=2048)])
def test_rotary_refuses(kw):
    assert call_rotary(**kw) == dj.DV_EINVAL and dj.dv_last_error()


def test_launches_past_2_to_32_threads_are_refused():
    tiny = dj.Rotary((1, 0, 0))
    assert call_rotary(plan=tiny.address, heads=1, head_dim=2, x_stride=2, out_stride=2,
                       rows=(1 << 27) + 1) == dj.DV_EINVAL
    # a page of 128 tokens of 128 channels takes blocks of 512 threads
    big = dict(c=dict(page_tokens=128, head_dim=128), wide=1 << 14, n_seqs=600000, rows=600000, offsets=None)
    assert refused("dv_cache_write", WRITE, big) == dj.DV_EINVAL and "600000" in dj.dv_last_error()


def test_rotary_of_no_rows():
    assert call_rotary(rows=0) == dj.DV_OK


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, pages=64, page_tokens=64, kv_heads=8, head_dim=64)
    a.update(kw)
    return dj.dv_cache(*a.values())


COMMON = [
    dict(cache=None), dict(c=dict(k=None)), dict(c=dict(v=None)), dict(c=dict(k_scale=None)),
    dict(c=dict(v_scale=None)), dict(c=dict(k=FAKE + 8)), dict(c=dict(v=FAKE + 4)), dict(c=dict(pages=0)),
    dict(c=dict(page_tokens=48)), dict(c=dict(page_tokens=256)), dict(c=dict(kv_heads=0)),
    dict(c=dict(head_dim=8)), dict(c=dict(head_dim=72)), dict(c=dict(head_dim=144)), dict(n_seqs=0),
    dict(table_pages=0), dict(table_pages=(1 << 24) + 1), dict(table=None, table_pages=17),
    dict(rows=-1), dict(offsets=None, rows=3), dict(rows=(1 << 31) - 1, c=dict(kv_heads=64), wide=1 << 14),
    dict(dtype=3), dict(at=None)]


def refused(fn, base, kw):
    a = dict(base)
    desc = cache(**kw.get("c", {}))
    wide = kw.get("wide")
    if wide:
        a.update({k: wide for k in a if k.endswith("stride")})
    a["cache"] = ctypes.addressof(desc)
    a.update({k: v for k, v in kw.items() if k not in ("c", "wide")})
    return getattr(dj.load(), fn)(*a.values())


WRITE = dict(cache=0, n_seqs=4, table=FAKE, table_pages=8, offsets=FAKE, at=FAKE, dtype=dj.DV_BF16, k=FAKE,
             k_stride=512, v=FAKE, v_stride=512, rows=9, plan=None, positions=None, q=None, q_stride=0,
             q_heads=0, q_out=None, q_out_stride=0, stream=None)
QUERY = dict(plan=ROT.address, positions=FAKE, q=FAKE, q_stride=1024, q_heads=16, q_out=FAKE,
             q_out_stride=1024)


@pytest.mark.parametrize("kw", COMMON + [
    dict(k=None), dict(v=None), dict(k_stride=511), dict(v_stride=511), dict(plan=ROT.address),
    dict(plan=WIDE_ROT.address, positions=FAKE), dict(plan=ctypes.addressof(BLANK), positions=FAKE),
    dict(QUERY, plan=None), dict(QUERY, positions=None), dict(QUERY, q_out=None), dict(QUERY, q_heads=0),
    dict(QUERY, q_stride=1023), dict(QUERY, q_out_stride=1000), dict(QUERY, q_stride=2048)])
def test_write_refuses(kw):
    assert refused("dv_cache_write", WRITE, kw) == dj.DV_EINVAL and dj.dv_last_error()


READ = dict(cache=0, n_seqs=4, table=FAKE, table_pages=8, offsets=FAKE, at=FAKE, dtype=dj.DV_F32, k=FAKE,
            k_stride=512, v=FAKE, v_stride=512, rows=9, stream=None)


@pytest.mark.parametrize("kw", COMMON + [dict(k=None), dict(v=None), dict(k_stride=511), dict(v_stride=0)])
def test_read_refuses(kw):
    assert refused("dv_cache_read", READ, kw) == dj.DV_EINVAL and dj.dv_last_error()


ATTEND = dict(cache=0, n_seqs=4, table=FAKE, table_pages=8, offsets=FAKE, at=FAKE, dtype=dj.DV_BF16, q=FAKE,
              q_stride=1024, rows=9, q_heads=16, max_rows=0, scale=0.125, causal=1, out=FAKE, out_stride=1024,
              workspace=FAKE, workspace_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("kw", COMMON + [
    dict(q=None), dict(out=None), dict(q_stride=1023), dict(out_stride=1020), dict(out_stride=1026),
    dict(out=FAKE + 4), dict(q_heads=0), dict(q_heads=12), dict(max_rows=-1), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(rows=1 << 28, wide=1024),
    dict(dtype=dj.DV_F32, out=FAKE + 8), dict(out_stride=2048)])
def test_attention_refuses(kw):
    assert refused("dv_cache_attention", ATTEND, kw) == dj.DV_EINVAL and dj.dv_last_error()


def test_attention_refuses_a_workspace_that_is_too_small():
    """A long table splits its keys over blocks, which meet in the workspace."""
    desc = cache(pages=4096)
    at = ctypes.addressof(desc)
    need = dj.dv_cache_attention_workspace(at, 4, 1024, True, dj.DV_BF16, 4, 16, 1)
    assert need > 0
    kw = dict(c=dict(pages=4096), rows=4, table_pages=1024, max_rows=1)
    for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=FAKE + 4)):
        assert refused("dv_cache_attention", ATTEND, dict(kw, **bad)) == dj.DV_EINVAL
        assert "workspace" in dj.dv_last_error()


def test_calls_without_rows_do_nothing():
    assert refused("dv_cache_write", WRITE, dict(rows=0)) == dj.DV_OK
    assert refused("dv_cache_read", READ, dict(rows=0)) == dj.DV_OK
    assert refused("dv_cache_attention", ATTEND, dict(rows=0)) == dj.DV_OK


def test_workspace_refuses():
    desc = cache()
    at, lib, n = ctypes.addressof(desc), dj.load(), ctypes.c_size_t(7)
    assert lib.dv_cache_attention_workspace(at, 4, 8, 1, 1, 9, 16, 0, None) == dj.DV_EINVAL
    assert lib.dv_cache_attention_workspace(at, 4, 8, 1, 1, 9, 12, 0, ctypes.byref(n)) == dj.DV_EINVAL
    assert lib.dv_cache_attention_workspace(None, 4, 8, 1, 1, 9, 16, 0, ctypes.byref(n)) == dj.DV_EINVAL
    assert lib.dv_cache_attention_workspace(at, 4, 8, 1, 2, 9, 16, 0, ctypes.byref(n)) == dj.DV_EINVAL
    assert n.value == 0


def test_wrapper_refuses_tensors_off_the_device():
    import torch
    x = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError):
        dj.rotary(x, torch.zeros(3, 3, dtype=torch.int32), ROT)
    c = dj.TokenCache(4, 2, 64, 16, device="cpu")
    with pytest.raises(ValueError):
        c.write(x, x, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        dj.TokenCache(4, 2, 64, 16, buffers=(c.v, c.k, c.k_scale, c.v_scale))


# ---- where rows go -------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plans") / "cache_plans.so")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
                    "-I", os.path.join(rocm, "include"), "-I", CSRC, os.path.join(HERE, "cache_plans.cpp"), "-o",
                    so], check=True)
    return ctypes.CDLL(so)


def ints(a):
    a = np.ascontiguousarray(a, np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def ragged(rng, n):
    counts = [rng.choice([0, 0, 1, 1, 2, 15, 16, 17, 63, 64, 65, 130, 300]) for _ in range(n)]
    return counts, np.concatenate([[0], np.cumsum(counts)])


@pytest.mark.parametrize("pt", [16, 32, 64, 128])
def test_every_row_has_one_place(lib, pt):
    """Ragged batches from any start, with padding behind them: the slots' parts cover every row of
    every sequence once, at its place, in the page the table names -- or in none where the table ends,
    names no page of the cache, or the start is negative."""
    rng = random.Random(pt)
    for n in (1, 2, 5, 64, 65, 130):
        counts, offs = ragged(rng, n)
        starts = [rng.choice([-3, 0, 1, pt - 1, pt, 5 * pt + 7]) for _ in range(n)]
        rows, tp, pages = int(offs[-1]) + rng.choice([0, 3]), 9, 7 * n
        table = np.array([[rng.choice([-1, pages, 1 << 30, rng.randrange(pages)]) for _ in range(tp)]
                          for _ in range(n)])
        (o, op), (s, sp), (t, tpp) = ints(offs), ints(starts), ints(table)
        out = np.zeros((rows // pt + 2 * n + 8, 5), np.int32)
        slots = lib.t_page_parts(tpp, tp, pages, op, n, rows, sp, pt, out.ctypes.data_as(ctypes.c_void_p))
        assert slots <= len(out)
        seen = {}
        for q, page, row0, slot0, k in out[:slots]:
            assert page < pages and 0 <= slot0 and slot0 + k <= pt
            for i in range(k):
                assert row0 + i not in seen
                seen[row0 + i] = (q, page, slot0 + i)
        want = {}
        for q in range(n):
            for i in range(counts[q] if starts[q] >= 0 else 0):
                p = starts[q] + i
                page = table[q][p // pt] if p // pt < tp else -1
                want[int(offs[q]) + i] = (q, page if 0 <= page < pages else -1, p % pt)
        assert seen == want


def test_places_without_offsets_and_table(lib):
    starts, sp = ints([0, 17, 31, 32])
    out = np.zeros((4, 5), np.int32)
    assert lib.t_page_parts(None, 2, 8, None, 4, 4, sp, 16, out.ctypes.data_as(ctypes.c_void_p)) == 4
    assert out.tolist() == [[0, 0, 0, 0, 1], [1, 3, 1, 1, 1], [2, 5, 2, 15, 1], [3, -1, 3, 0, 1]]


def test_rows_before_the_first_offset_have_no_place(lib):
    (o, op), (s, sp) = ints([5, 40, 40, 57]), ints([3, 0, 20])
    out = np.zeros((64, 5), np.int32)
    slots = lib.t_page_parts(None, 8, 24, op, 3, 60, sp, 16, out.ctypes.data_as(ctypes.c_void_p))
    assert sorted(r0 + i for _, _, r0, _, k in out[:slots] for i in range(k)) == list(range(5, 57))
    tiles = np.zeros((64, 6), np.int32)
    slots = lib.t_tiles(8, op, 3, 60, sp, 16, 3, 4, 1, tiles.ctypes.data_as(ctypes.c_void_p))
    rows = sorted((q, first + i) for q, _, first, n, _, _ in tiles[:slots] if q >= 0 for i in range(n))
    assert rows == [(0, i) for i in range(35 * 3)] + [(2, i) for i in range(17 * 3)]


def test_offsets_past_the_rows_are_cut(lib):
    """Rows that a call does not have are not touched, whatever its offsets say."""
    (o, op), (s, sp) = ints([0, 40, 90, 1 << 30]), ints([0, 0, 0])
    out = np.zeros((64, 5), np.int32)
    slots = lib.t_page_parts(None, 8, 24, op, 3, 60, sp, 16, out.ctypes.data_as(ctypes.c_void_p))
    assert all(r0 + k <= 60 for _, _, r0, _, k in out[:slots])


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("group", [1, 3, 4, 16, 20])
@pytest.mark.parametrize("shift", [4, 7])
def test_every_packed_row_has_one_tile(lib, shift, group, causal):
    rng = random.Random(group)
    for n in (1, 3, 64, 70):
        counts, offs = ragged(rng, n)
        lengths = [rng.choice([-1, 0, 1, 5, 100, 1000, 1 << 30]) for _ in range(n)]
        rows, tp, pt = int(offs[-1]) + 2, 40, 16
        (o, op), (s, sp) = ints(offs), ints(lengths)
        out = np.zeros((rows * group // (1 << shift) + n + 8, 6), np.int32)
        slots = lib.t_tiles(tp, op, n, rows, sp, pt, group, shift, causal, out.ctypes.data_as(ctypes.c_void_p))
        assert slots <= len(out)
        seen = set()
        for q, row0, first, k, length, end in out[:slots]:
            if q < 0:
                continue
            assert row0 == offs[q] and length == max(0, min(lengths[q], tp * pt))
            last = (first + k - 1) // group
            assert end == (max(0, length - counts[q] + last + 1) if causal else length)
            for i in range(first, first + k):
                assert (q, i) not in seen
                seen.add((q, i))
        assert seen == {(q, i) for q in range(n) for i in range(counts[q] * group)}
    out = np.zeros((64, 6), np.int32)
    (s, sp) = ints([5] * 6)
    slots = lib.t_tiles(4, None, 6, 6, sp, 16, group, shift, causal, out.ctypes.data_as(ctypes.c_void_p))
    assert sorted((q, i) for q, _, f, k, _, _ in out[:slots] for i in range(f, f + k)) == \
        [(q, i) for q in range(6) for i in range(group)]


# ---- how attention is cut ------------------------------------------------------------------------
FEW, MANY, BOTH = range(3)


def plan(lib, bf16, n, rows, offsets, max_rows, table_pages, pt, heads, q_heads, dh, cus=256):
    out = (ctypes.c_longlong * 7)()
    route = lib.t_attn_plan(bf16, n, rows, offsets, max_rows, table_pages, pt, heads, q_heads, dh, cus, out)
    return (route, *out)


def test_attention_routes_of_the_gpu_tests(lib):
    """The cases that test large tiles take them, alone or for the longer sequences; the others small
    ones; some batches of each split their keys."""
    split = set()
    for cases, large in ((on_gpu.ATTENTION, False), (on_gpu.LARGE, True)):
        for name, (heads, group, dh, pt, counts, lengths, pad) in cases.items():
            tp = max(1, max(-(-x // pt) for x in lengths))
            for most in (0, max(counts)):
                p = plan(lib, 1, len(counts), sum(counts) + pad, 1, most, tp, pt, heads, heads * group, dh)
                if not large:
                    assert p[0] == FEW, name
                elif len(counts) > 1 and not (most and len(set(counts)) == 1 and pad == 0):
                    assert p[0] == BOTH, name
                else:
                    assert p[0] == MANY, name
                split |= {(w, p[i] > 1) for w, i in (("few", 2), ("many", 5)) if p[i]}
            assert plan(lib, 0, len(counts), sum(counts) + pad, 1, 0, tp, pt, heads, heads * group, dh)[0] == FEW
    assert plan(lib, 1, 3, 240, 1, 0, 10, 16, 64, 128, 64)[0] == BOTH      # of test_attention_extremes
    assert split == {(w, s) for w in ("few", "many") for s in (False, True)}, split


@pytest.mark.parametrize("bf16", [0, 1])
def test_attention_cuts_cover_the_table(lib, bf16):
    """Splits cover every key that a table can hold, in the range the kernels take; the workspace holds a
    partial result for every tile, head and split; launches stay within 2^32 threads."""
    rng = random.Random(4)
    for _ in range(3000):
        n, heads, group = rng.choice([1, 2, 3, 64, 300]), rng.choice([1, 2, 8, 40]), rng.choice([1, 4, 7, 16])
        pt, dh = rng.choice([16, 32, 64, 128]), rng.choice([16, 64, 128])
        tp = min((1 << 30) // pt, int(2 ** rng.uniform(0, 26)))
        offsets = rng.random() < 0.7
        rows = n if not offsets else rng.choice([n, 5 * n, int(2 ** rng.uniform(0, 18))])
        most = rng.choice([0, 1, rows])
        p = plan(lib, bf16, n, rows, int(offsets), most, tp, pt, heads, heads * group, dh, rng.choice([0, 256, 304]))
        need = 0
        for chunk, splits, slots, rows_a_tile in ((*p[1:4], 16), (*p[4:7], 128)):
            if not splits:
                continue
            assert chunk % 256 == 0 and 1 <= splits <= 512
            assert chunk * splits >= tp * pt > chunk * (splits - 1)
            assert slots * heads * splits * 256 < 1 << 32
            if splits > 1:
                need += slots * heads * splits * rows_a_tile * (dh + 2) * 4
        # 64 blocks a unit of 16 rows; splits of large tiles only where two blocks a unit leave room
        assert p[7] == need and need <= 304 * (64 * 16 + 4 * 128) * (dh + 2) * 4 + (1 << 24)
