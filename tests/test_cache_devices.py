"""Which device, stream and sizes the operators on token rows take, with tensors stood in for."""
import types

import pytest
import torch

from paper_2506_14107_amd import dejavu as dj


def test_device_zero_is_a_device(monkeypatch):
    """A cache asked for on device 0 lies there, whatever device is current."""
    seen, empty = [], torch.empty
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: seen.append(device) or empty(*a, device="cpu", **k))
    dj.TokenCache(4, 2, 64, 16, device=0)
    assert [torch.device("cuda", d) if isinstance(d, int) else d for d in seen] == [torch.device("cuda", 0)] * 4
    seen.clear()
    dj.TokenCache(4, 2, 64, 16)
    assert seen == [torch.device("cuda", 1)] * 4


def test_streams_of_another_device_are_refused(monkeypatch):
    """Work asked for on a stream that is not of the tensors' device would run on another than the one given."""
    rot = dj.Rotary((8, 12, 12))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = types.SimpleNamespace(get_device=lambda: 0)
    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="cuda:1"):
        dj.rotary(x, x, rot, stream=stream)
    c = dj.TokenCache(4, 2, 64, 16, device="cpu")
    c.index = 0
    for call in (lambda: c.write(x, x, x, stream=stream), lambda: c.read(x, stream=stream),
                 lambda: c.attention(x, x, stream=stream)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()


def test_counts_past_a_c_int_are_refused(monkeypatch):
    """2^32 rows or sequences would be cut to 0, and the call do nothing without an error."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def big(*shape, dtype=torch.bfloat16):
        t = torch.empty(shape, dtype=dtype, device="meta")
        return types.SimpleNamespace(shape=t.shape, dtype=dtype, stride=t.stride, dim=t.dim, get_device=lambda: 0,
                                     is_contiguous=lambda: True, data_ptr=lambda: 0)

    n = 1 << 32
    rot = dj.Rotary((4, 2, 2))
    with pytest.raises(ValueError, match="too many"):
        dj.rotary(big(n, 1, 16), big(n, 3, dtype=torch.int32), rot)
    c = dj.TokenCache(4, 1, 16, 16, device="cpu")
    c.index = 0
    x, at = big(n, 1, 16), big(1, dtype=torch.int32)
    for call in (lambda: c.write(x, x, at), lambda: c.read(at, out=(x, x)), lambda: c.attention(x, at),
                 lambda: c.read(big(n, dtype=torch.int32), out=(x, x))):
        with pytest.raises(ValueError, match="too many"):
            call()
