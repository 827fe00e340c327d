"""Which device and stream the operators on token rows take, with devices stood in for."""
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
