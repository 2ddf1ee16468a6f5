"""Attention's entry points make the tensor's device current for their call, and only then ask for the stream.  Without a GPU: torch's
device functions and the library are stood in for."""
import contextlib

import torch

from paper_2202_04305_amd import binding


class _Pattern:
    _h, device, _sizes, _workspaces = 7, torch.device("cuda", 3), (2, 0, 0), {}


def test_the_inspector_runs_on_the_tensors_device(monkeypatch):
    now, calls = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d.index
        yield
        now[0] = before

    class library:
        @staticmethod
        def sp_prepare_attention(h, grad, stream):
            calls.append((h, grad, stream))
            return 0
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(binding, "load_library", lambda: library)
    monkeypatch.setattr(binding, "_stream_ptr", lambda: 1000 + now[0])
    S = _Pattern()
    assert binding.sp_prepare_attention(S, grad=True) is S
    assert calls == [(7, 1, 1003)] and now == [0]
    now[0] = 3
    binding.sp_prepare_attention(S)
    assert calls[1:] == [(7, 0, 1003)]
