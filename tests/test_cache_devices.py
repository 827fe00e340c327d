"""Which device and stream the operators on token rows take, with devices stood in for."""
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
