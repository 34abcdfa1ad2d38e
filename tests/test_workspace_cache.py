"""The binding's workspaces: one cached buffer per stream for eager calls, memory of the graph's own for captured ones."""
import torch

from paper_2509_23472_amd import api


def test_captured_calls_take_no_cached_buffer(monkeypatch):
    capturing = [False]
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: capturing[0], raising=False)
    monkeypatch.setattr(api, "_stream_ptr", lambda: 11)
    monkeypatch.setattr(api, "_workspaces", {})
    device = torch.device("cpu", 0)
    eager = api._workspace(1000, device)
    assert api._workspace(800, device) is eager
    capturing[0] = True
    held = api._workspace(1000, device)
    assert held.numel() >= 1000 and held.data_ptr() != eager.data_ptr()
    grown = api._workspace(5000, device)
    assert grown.numel() >= 5000 and all(w is eager for w in api._workspaces.values())
    capturing[0] = False
    assert api._workspace(1000, device) is eager                                  # what was captured is not handed to eager calls
    assert api._workspace(5000, device).data_ptr() not in (held.data_ptr(), grown.data_ptr())
