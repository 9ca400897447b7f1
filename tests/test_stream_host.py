"""The stream that calls are enqueued on: torch's current one, by its public interface where the
private one for its pointer is not there.  No GPU is needed: the handle and torch are stand-ins."""
import types

import pytest


@pytest.mark.parametrize("private", [False, True])
def test_current_stream(private, monkeypatch):
    import paper_2206_08369_amd as pm
    seen, asked = [], []
    monkeypatch.setattr(pm, "pmlp_set_stream", lambda h, s: seen.append((h, s)))
    device = types.SimpleNamespace(index=3)

    def current_stream(d):
        asked.append(d)
        return types.SimpleNamespace(cuda_stream=0xABC0)

    c = types.SimpleNamespace()
    if private:
        c._cuda_getCurrentRawStream = lambda i: 0xABC0 if i == 3 else None
    net = pm.PackedMLP.__new__(pm.PackedMLP)
    net._torch = types.SimpleNamespace(_C=c, cuda=types.SimpleNamespace(current_stream=current_stream))
    net.device, net.handle = device, 77
    try:
        net._stream()
    finally:
        net.handle = None
    assert seen == [(77, 0xABC0)] and asked == ([] if private else [device])
