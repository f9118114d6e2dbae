"""examples/train_encoder.py: a step waits for nothing on the host."""
import pytest
import torch

import examples.train_encoder as ex

pytestmark = pytest.mark.gpu


def test_a_step_does_not_synchronise(monkeypatch):
    """torch raises at any of its calls that waits for the device, for one whole step and the windows of the next."""
    real, calls = ex.windows, []

    def windows(*args, **kw):
        calls.append(torch.cuda.get_sync_debug_mode())
        if len(calls) == 2:
            torch.cuda.set_sync_debug_mode("error")
        x = real(*args, **kw)
        if len(calls) == 3:
            torch.cuda.set_sync_debug_mode("default")
        return x

    monkeypatch.setattr(ex, "windows", windows)
    try:
        ex.train(steps=4)
    finally:
        torch.cuda.set_sync_debug_mode("default")
    assert calls == [0, 0, 2, 0]
