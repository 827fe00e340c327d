"""What the operators around the 8-bit cache refuse, before any GPU work."""
import ctypes
import math
import types

import pytest
import torch

from paper_2506_14107_amd import dejavu as dj

from .test_cache import BLANK, COMMON, FAKE, QUERY, ROT, WIDE_ROT, WRITE, refused


def head_norm(weight=FAKE, per_head=0, eps=1e-6):
    return dj.dv_head_norm(weight, per_head, eps)


NORM = head_norm()
BAD = [head_norm(eps=e) for e in (0.0, -1.0, math.nan, math.inf)]


# ---- norms ---------------------------------------------------------------------------------------------
def call_norm(**kw):
    a = dict(norm=ctypes.addressof(NORM), plan=ROT.address, dtype=dj.DV_BF16, x=FAKE, x_stride=256, rows=5, heads=4,
             head_dim=64, positions=FAKE, out=2 * FAKE, out_stride=256)
    a.update(kw)
    return dj.load().dv_norm_rotary(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(norm=None), *(dict(norm=ctypes.addressof(b)) for b in BAD), dict(plan=ctypes.addressof(BLANK)), dict(dtype=2),
    dict(x=None), dict(positions=None), dict(out=None), dict(rows=-1), dict(heads=0), dict(head_dim=0), dict(head_dim=62),
    dict(head_dim=63, plan=None), dict(x_stride=255), dict(out_stride=255), dict(out=FAKE, x_stride=512),
    dict(rows=1 << 30, heads=32, x_stride=2048, out_stride=2048)])
def test_norm_rotary_refuses(kw):
    assert call_norm(**kw) == dj.DV_EINVAL and dj.dv_last_error()


def test_norm_rotary_of_no_rows():
    assert call_norm(rows=0) == dj.DV_OK and call_norm(rows=0, plan=None, positions=None, x=None) == dj.DV_OK


WRITE_NORM = dict(list(WRITE.items())[:-1], k_norm=ctypes.addressof(NORM), q_norm=None, stream=None)


@pytest.mark.parametrize("kw", COMMON + [
    dict(k=None), dict(v=None), dict(k_stride=511), dict(plan=ROT.address), dict(plan=WIDE_ROT.address, positions=FAKE),
    *(dict(k_norm=ctypes.addressof(b)) for b in BAD), *(dict(QUERY, q_norm=ctypes.addressof(b)) for b in BAD),
    dict(q_norm=ctypes.addressof(NORM)), dict(QUERY, plan=None), dict(QUERY, q_out=None, q_norm=ctypes.addressof(NORM)),
    dict(QUERY, q_heads=0, q_norm=ctypes.addressof(NORM)), dict(QUERY, q_stride=1023, plan=None, q_norm=ctypes.addressof(NORM))])
def test_write_with_norms_refuses(kw):
    assert refused("dv_cache_write_norm", WRITE_NORM, kw) == dj.DV_EINVAL and dj.dv_last_error()


def test_write_with_norms_of_no_rows():
    assert refused("dv_cache_write_norm", WRITE_NORM, dict(rows=0)) == dj.DV_OK
    assert refused("dv_cache_write_norm", WRITE_NORM, dict(QUERY, rows=0, plan=None, q_norm=ctypes.addressof(NORM))) == dj.DV_OK


# ---- pages handed out ---------------------------------------------------------------------------------
EXTEND = dict(n_seqs=4, table=FAKE, table_pages=8, page_tokens=64, lengths=2 * FAKE, counts=3 * FAKE, ring=4 * FAKE, pages=100,
              cursor=5 * FAKE, rows=9, offsets=6 * FAKE, starts=7 * FAKE, lengths_out=8 * FAKE, cursor_out=9 * FAKE, positions=None,
              slots=None, stream=None)


@pytest.mark.parametrize("kw", [dict([(name, None)]) for name in (
    "table", "lengths", "counts", "ring", "cursor", "offsets", "starts", "lengths_out", "cursor_out")] + [
    dict(n_seqs=0), dict(table_pages=0), dict(pages=0), dict(pages=(1 << 30) + 1), dict(rows=-1), dict(page_tokens=48),
    dict(page_tokens=256), dict(table_pages=(1 << 24) + 1), dict(n_seqs=1 << 15, table_pages=1 << 16),
    dict(n_seqs=(1 << 30) + 1, table_pages=1)])
def test_extend_refuses(kw):
    assert dj.load().dv_cache_extend(*dict(EXTEND, **kw).values()) == dj.DV_EINVAL and dj.dv_last_error()


@pytest.mark.parametrize("out,at", [(out, EXTEND[x] + d) for out, size in (
    ("offsets", 20), ("starts", 16), ("lengths_out", 16), ("cursor_out", 24), ("positions", 108), ("slots", 72))
    for x, held in (("lengths", 16), ("counts", 16), ("cursor", 24)) for d in (0, held - 4, 4 - size)])
def test_extend_refuses_outputs_over_what_it_reads(out, at):
    assert dj.load().dv_cache_extend(*dict(EXTEND, **{out: at}).values()) == dj.DV_EINVAL and "overlap" in dj.dv_last_error()


# ---- tensors -------------------------------------------------------------------------------------------
def test_wrappers_refuse_tensors_off_the_device():
    x, at = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        dj.norm_rotary(x)
    with pytest.raises(ValueError):
        dj.extend(torch.zeros(3, 4, dtype=torch.int32), at, at, at, torch.zeros(3, dtype=torch.int64), 16, 3)


def on_device(*shape, dtype=torch.bfloat16, index=0):
    """A tensor that claims to be on a device."""
    t = torch.empty(shape, dtype=dtype, device="meta")
    return types.SimpleNamespace(shape=t.shape, dtype=dtype, stride=t.stride, dim=t.dim, get_device=lambda: index, device="cuda:0",
                                 is_contiguous=t.is_contiguous, data_ptr=lambda: FAKE)


def test_wrappers_refuse_what_does_not_fit(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(dj, "_raw_stream", lambda index: 0)
    x, i32, i64 = on_device(5, 2, 64), torch.int32, torch.int64
    pos = on_device(5, 3, dtype=i32)
    for a in ((x, on_device(63)), (x, on_device(3, 64)), (x, on_device(64, dtype=torch.float32)), (x, on_device(64, index=1)),
              (x, None, 1e-6, pos), (x, None, 1e-6, None, ROT), (x, None, 1e-6, on_device(4, 3, dtype=i32), ROT),
              (x, None, 1e-6, on_device(5, 3, dtype=i64), ROT), (on_device(5, 2, 64, dtype=torch.float16),), (on_device(5, 64),)):
        with pytest.raises(ValueError):
            dj.norm_rotary(*a, out=x)
    with pytest.raises(dj.DejaVuError):
        dj.norm_rotary(x, None, 0.0, out=x)
    c = dj.TokenCache(4, 2, 64, 16, device="cpu")
    c.index = 0
    starts = on_device(1, dtype=i32)
    offs = on_device(2, dtype=i32)
    for kw in (dict(k_norm=on_device(3, 64)), dict(k_norm=on_device(64, dtype=torch.float32)), dict(q_norm=True),
               dict(q=x, q_out=x, q_norm=on_device(3, 64))):
        with pytest.raises(ValueError):
            c.write(x, x, starts, offs, **kw)
    n, P, pages, rows = 3, 4, 20, 7
    good = dict(table=on_device(n, P, dtype=i32), lengths=on_device(n, dtype=i32), counts=on_device(n, dtype=i32),
                ring=on_device(pages, dtype=i32), cursor=on_device(3, dtype=i64), page_tokens=16, rows=rows)
    out = [on_device(n + 1, dtype=i32), on_device(n, dtype=i32), on_device(n, dtype=i32), on_device(3, dtype=i64),
           on_device(rows, 3, dtype=i32), on_device(rows, dtype=i64)]
    for kw in (dict(table=on_device(n, dtype=i32)), dict(table=on_device(n, P, dtype=i64)), dict(lengths=on_device(n + 1, dtype=i32)),
               dict(counts=on_device(n, dtype=i64)), dict(ring=on_device(2, 10, dtype=i32)), dict(cursor=on_device(3, dtype=i32)),
               dict(cursor=on_device(2, dtype=i64)), dict(rows=1 << 32), dict(lengths=on_device(n, dtype=i32, index=1))):
        with pytest.raises(ValueError):
            dj.extend(**dict(good, **kw), out=out)
    for i, bad in enumerate((on_device(n, dtype=i32), on_device(n, dtype=i64), on_device(n + 1, dtype=i32), on_device(2, dtype=i64),
                             on_device(rows, dtype=i32), on_device(rows, dtype=i32))):
        with pytest.raises(ValueError):
            dj.extend(**good, out=out[:i] + [bad] + out[i + 1:])


def test_streams_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = types.SimpleNamespace(get_device=lambda: 0)
    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    for call in (lambda: dj.norm_rotary(x, stream=stream), lambda: dj.extend(x, x, x, x, x, 16, 1, stream=stream)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()
