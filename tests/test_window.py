"""Attention with a window and over shared prefixes on the CPU: what is refused, which keys tiles take, how calls are cut."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest
import torch

from paper_2506_14107_amd import dejavu as dj

from . import test_gpu_shared as on_gpu
from .test_cache import ATTEND, COMMON, FAKE, cache, refused
from .test_cache_operators import on_device

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2506_14107_amd", "csrc")
EINVAL = dj.DV_EINVAL


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plans") / "window_plans.so")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(rocm, "include"), "-I", CSRC, os.path.join(HERE, "window_plans.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


# ---- which keys a tile takes ---------------------------------------------------------------------------
def tiles(lib, *a):
    out = (ctypes.c_int * 4000)()
    n = lib.t_window_tiles(*a, out)
    return [tuple(out[5 * i:5 * i + 5]) for i in range(n)]


def plan(lib, *a):
    out = (ctypes.c_longlong * 7)()
    return (lib.t_window_plan(*a, out), *out)


@pytest.mark.parametrize("shift", [4, 7])
def test_tiles_take_every_key_that_a_row_sees(lib, shift):
    """... in whole steps of 64 but for the last one, and within the splits that the call launches, whatever bound of rows
    it was given."""
    rng = random.Random(shift)
    big = 1 << 30
    for _ in range(4000):
        n, group, causal = rng.choice([1, 2, 9, 100]), rng.choice([1, 3, 4, 16]), rng.choice([0, 1])
        length = rng.choice([-1, 0, 1, 63, 64, 65, 300, 1000, 3000])
        window, sinks = rng.choice([1, 2, 63, 64, 65, 200, 1000, big]), rng.choice([0, 1, 63, 64, 65, 300, 5000, big])
        tp, pt = rng.choice([1, 30, 200]), 16
        length = min(length, tp * pt)
        p = plan(lib, 1, 1, n, 1, rng.choice([0, 1, n]), tp, pt, 2, 2 * group, 64, 256, window, sinks)
        for first, rows, end, skip0, left_out in tiles(lib, n, length, tp, pt, group, shift, causal, window, sinks):
            assert skip0 % 64 == 0 and left_out % 64 == 0 and (left_out == 0 or skip0 + left_out < end)
            for i in range(first // group, (first + rows - 1) // group + 1):
                e = max(0, length - n + i + 1) if causal else max(0, length)
                assert e <= end
                if left_out:      # what is left out lies between the sinks and the row's window
                    assert skip0 >= min(sinks, e) and skip0 + left_out <= e - window
            chunk, splits = p[1:3] if shift == 4 else p[4:6]
            if splits:
                assert end - left_out <= chunk * splits


def test_windows_are_cut_by_what_they_see(lib):
    """Splits and workspaces follow the window, not the table."""
    short = plan(lib, 1, 64, 64, 1, 1, 200, 64, 8, 32, 128, 256, 2048, 257)
    long = plan(lib, 1, 64, 64, 1, 1, 200000, 64, 8, 32, 128, 256, 2048, 257)
    assert short == long
    assert plan(lib, 1, 64, 64, 1, 1, 200, 64, 8, 32, 128, 256, 1 << 30, 0) == \
        plan(lib, 1, 64, 64, 1, 1, 200, 64, 8, 32, 128, 256, 0, 0)


@pytest.mark.parametrize("bf16", [0, 1])
def test_shared_calls_are_cut(lib, bf16):
    """Splits cover every key that a table can hold, slots every row whichever way it falls into groups, the workspace a
    partial result for every tile, head and split."""
    rng, seen = random.Random(5), set()
    for _ in range(3000):
        n, heads, group = rng.choice([1, 2, 64, 300]), rng.choice([1, 2, 8, 40]), rng.choice([1, 4, 16])
        pt, dh, ng = rng.choice([16, 64, 128]), rng.choice([16, 64, 128]), rng.choice([1, 1, 2, 30])
        tables = [min((1 << 30) // pt, int(2 ** rng.uniform(0, 22))) for _ in range(2)]
        offsets = rng.random() < 0.7
        rows = rng.choice([n, 5 * n, int(2 ** rng.uniform(0, 16))]) if offsets else n
        out = (ctypes.c_longlong * 19)()
        lib.t_shared_plan(bf16, n, rows, int(offsets), rng.choice([0, rows]), tables[0], ng, tables[1], pt, heads, heads * group, dh,
                          256, out)
        total = blocks = 0
        if out[18]:      # one plan, whose splits cover the prefix in whole steps and the sequence
            route, *cuts, size = out[:8]
            need = 0
            for (chunk, splits, slots), tile in ((cuts[:3], 16), (cuts[3:], 128)):
                assert not splits or chunk % 64 == 0 and chunk * splits >= -(-tables[1] * pt // 64) * 64 + tables[0] * pt
                need += slots * heads * splits * tile * (dh + 2) * 4 * (splits > 1)
            assert size == need == out[16] and chunk * splits < 1 << 31
            seen.add("behind")
            continue
        seen.add("apart")
        for i, (k, seqs) in enumerate(((tables[0], n), (tables[1], ng))):
            route, *cuts, size = out[8 * i:8 * i + 8]
            need = 0
            for (chunk, splits, slots), tile, off in ((cuts[:3], 16, 1), (cuts[3:], 128, 0)):
                assert bool(splits) == (route != off) and (bf16 or tile == 16 or not splits)
                if not splits:
                    continue
                assert chunk % 64 == 0 and chunk * splits >= k * pt > chunk * (splits - 1) and splits <= 512
                if seqs == 1:
                    assert slots >= -(-rows * group // tile)
                elif i or offsets:      # each sequence may end with a part of a tile
                    assert slots >= rows * group // tile + min(seqs, rows * group % tile + rows * group // tile)
                else:
                    assert slots == seqs * -(-group // tile)
                need += slots * heads * splits * tile * (dh + 2) * 4
                blocks += slots * heads * splits
            assert size == need
            total += need
        assert out[16] == total and out[17] == blocks
    assert seen == {"behind", "apart"}


def test_shared_calls_of_the_gpu_tests(lib):
    """Their long prefixes take large tiles, small ones or either by group, under sequences in small tiles or by sequence; the
    short ones go with the sequences' own keys, in small tiles, large ones and either."""
    def plans(cases):
        out, r = (ctypes.c_longlong * 19)(), {}
        for name, (heads, group, dh, pt, counts, lengths, groups, prefix, pad) in cases.items():
            tp, ptp = (max(1, max(-(-x // pt) for x in y)) for y in (lengths, prefix))
            lib.t_shared_plan(1, len(counts), sum(counts) + pad, 1, 0, tp, len(prefix), ptp, pt, heads, heads * group, dh, 256, out)
            r[name] = ("behind", out[0]) if out[18] else (out[8], out[0])
        return r

    assert plans(on_gpu.LONG) == {"tokens": (1, 0), "groups": (2, 0), "prompts": (1, 2), "prompts-16": (2, 2), "few": (0, 0)}
    assert set(plans(on_gpu.BEHIND).values()) == {("behind", 0), ("behind", 1), ("behind", 2)}
    assert set(plans(on_gpu.APART).values()) == {(0, 0)}


# ---- refusals ------------------------------------------------------------------------------------------
def insert(base, before, **kw):
    out = {}
    for k, v in base.items():
        if k == before:
            out.update(kw)
        out[k] = v
    return out


WINDOW = insert(ATTEND, "out", window=100, sinks=4)
SHARED = insert(ATTEND, "dtype", n_groups=2, groups=FAKE, prefix_table=FAKE, prefix_table_pages=8, prefix_lengths=FAKE)
ATTENTION = COMMON + [
    dict(q=None), dict(out=None), dict(q_stride=1023), dict(out_stride=1020), dict(out_stride=1026), dict(out=FAKE + 4),
    dict(q_heads=0), dict(q_heads=12), dict(max_rows=-1), dict(scale=0.0), dict(scale=float("nan")), dict(rows=1 << 28, wide=1024),
    dict(dtype=dj.DV_F32, out=FAKE + 8), dict(out_stride=2048)]


@pytest.mark.parametrize("kw", ATTENTION + [dict(window=0), dict(window=-1), dict(sinks=-1)])
def test_window_refuses(kw):
    assert refused("dv_cache_attention_window", WINDOW, kw) == EINVAL and dj.dv_last_error()


@pytest.mark.parametrize("kw", ATTENTION + [
    dict(n_groups=0), dict(prefix_table=None), dict(prefix_lengths=None), dict(prefix_table_pages=0),
    dict(prefix_table_pages=(1 << 24) + 1), dict(groups=None), dict(n_groups=(1 << 31) - 1)])
def test_shared_refuses(kw):
    assert refused("dv_cache_attention_shared", SHARED, kw) == EINVAL and dj.dv_last_error()


def test_shared_refuses_a_workspace_that_is_too_small():
    """Prefixes and sequences in one pass, whose splits meet in it, and in one each."""
    desc = cache(pages=1 << 20)
    for n, pages in ((4, 40), (64, 2000)):
        need = dj.dv_cache_attention_shared_workspace(ctypes.addressof(desc), n, 1024, True, 2, pages, dj.DV_BF16, n, 16, 1)
        assert need > 0
        kw = dict(c=dict(pages=1 << 20), n_seqs=n, rows=n, table_pages=1024, max_rows=1, prefix_table_pages=pages)
        for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=FAKE + 4)):
            assert refused("dv_cache_attention_shared", SHARED, dict(kw, **bad)) == EINVAL and "workspace" in dj.dv_last_error()


def test_window_refuses_a_workspace_that_is_too_small():
    desc = cache(pages=4096)
    need = dj.dv_cache_attention_window_workspace(ctypes.addressof(desc), 4, 1024, True, dj.DV_BF16, 4, 16, 1, 30000, 0)
    assert need > 0
    kw = dict(c=dict(pages=4096), rows=4, table_pages=1024, max_rows=1, window=30000, sinks=0)
    for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=FAKE + 4)):
        assert refused("dv_cache_attention_window", WINDOW, dict(kw, **bad)) == EINVAL and "workspace" in dj.dv_last_error()


def test_calls_without_rows_do_nothing():
    assert refused("dv_cache_attention_window", WINDOW, dict(rows=0)) == dj.DV_OK
    assert refused("dv_cache_attention_shared", SHARED, dict(rows=0)) == dj.DV_OK


def test_workspaces_refuse():
    desc = cache()
    at, l, n = ctypes.addressof(desc), dj.load(), ctypes.c_size_t(7)
    for a in ((4, 8, 1, 1, 9, 16, 0, 0, 4), (4, 8, 1, 1, 9, 16, 0, 5, -1), (4, 8, 1, 1, 9, 12, 0, 5, 0), (4, 8, 1, 2, 9, 16, 0, 5, 0)):
        assert l.dv_cache_attention_window_workspace(at, *a, ctypes.byref(n)) == EINVAL
    for a in ((4, 8, 1, 0, 8, 1, 9, 16, 0), (4, 8, 1, 2, 0, 1, 9, 16, 0), (4, 8, 1, 2, 8, 1, 9, 12, 0), (4, 8, 1, 2, 8, 2, 9, 16, 0)):
        assert l.dv_cache_attention_shared_workspace(at, *a, ctypes.byref(n)) == EINVAL
    assert n.value == 0
    assert l.dv_cache_attention_window_workspace(at, 4, 8, 1, 1, 9, 16, 0, 5, 0, None) == EINVAL
    assert l.dv_cache_attention_shared_workspace(at, 4, 8, 1, 2, 8, 1, 9, 16, 0, None) == EINVAL


def test_wrappers_refuse_what_does_not_fit(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    c = dj.TokenCache(8, 2, 64, 16, device="cpu")
    c.index = 0
    i32 = torch.int32
    q, lengths, offs, table = on_device(5, 4, 64), on_device(2, dtype=i32), on_device(3, dtype=i32), on_device(2, 4, dtype=i32)
    for kw in (dict(window=-1), dict(sinks=4), dict(window=5, sinks=-1)):
        with pytest.raises(ValueError):
            c.attention(q, lengths, offs, table, out=q, **kw)
        with pytest.raises(ValueError):
            c.attention_workspace(2, 5, 4, **kw)
    good = dict(prefix_lengths=on_device(2, dtype=i32), prefix_table=on_device(2, 3, dtype=i32), groups=on_device(3, dtype=i32))
    for kw in (dict(prefix_lengths=on_device(1, dtype=i32)), dict(prefix_lengths=on_device(2, 1, dtype=i32)), dict(groups=None),
               dict(prefix_table=on_device(6, dtype=i32)), dict(groups=on_device(2, dtype=i32)),
               dict(groups=on_device(3, dtype=torch.int64)), dict(prefix_table=on_device(2, 3, dtype=i32, index=1))):
        with pytest.raises(ValueError):
            c.attention_shared(q, lengths, offsets=offs, table=table, out=q, **dict(good, **kw))
    import types
    x = types.SimpleNamespace(get_device=lambda: 0)
    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="cuda:1"):
        c.attention_shared(x, x, x, x, stream=stream)
