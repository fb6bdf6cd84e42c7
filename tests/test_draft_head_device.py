"""A DraftHead's library calls are made with its device current: a device's default stream reaches the
library as NULL, which names the current device.  (On the CPU: the library's calls are recorded.)"""
import contextlib

import pytest
import torch

from paper_2608_12913_amd import dcd, runner


@pytest.fixture
def calls(monkeypatch):
    current, made = [], []

    @contextlib.contextmanager
    def device(d):
        current.append(d)
        yield
        current.pop()

    class Default:
        cuda_stream = 0

        def synchronize(self):
            pass

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Default())
    monkeypatch.setattr(torch.cuda, "synchronize", lambda d=None: None)
    for name in ("quantize_fp8", "logits_fp8", "sample"):
        monkeypatch.setattr(dcd, name, lambda *a, name=name, **kw: made.append((name, current[-1] if current else None)))
    return made


def test_calls_are_made_on_the_heads_device(calls):
    head = runner.DraftHead(torch.randn(300, 64), max_rows=3, device="cpu")
    h, u, tokens = torch.randn(2, 64), torch.rand(2), torch.zeros(2, dtype=torch.int32)
    head.launch(h, u, tokens)
    head.launch(h, u, tokens, stream=0)
    head.propose(h, u)
    assert [n for n, _ in calls] == ["quantize_fp8"] + 3 * ["quantize_fp8", "logits_fp8", "sample"]
    assert all(d is not None and torch.device(d) == head.device for _, d in calls)


def test_device_is_the_tensors_own(calls):
    head = runner.DraftHead(torch.randn(300, 64), max_rows=3, device="cpu")
    assert head.device == head.w.device == head.logits.device == head.workspace.device
