"""Calls on tensors of a device that is not the current one."""
from __future__ import annotations

import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2606_11357_amd import tilefuse as tf  # noqa: E402


class Machine:
    """Two devices, and a library that notes which was current at each call."""

    def __init__(self, monkeypatch):
        self.current, self.calls = 0, []
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.current)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index)
        monkeypatch.setattr(torch.cuda, "device", self.made_current)
        monkeypatch.setattr(tf, "load", lambda: self)

    @contextlib.contextmanager
    def made_current(self, device):
        before, self.current = self.current, torch.device(device).index
        yield
        self.current = before

    def tf_silu_mul(self, *args):
        self.calls.append((self.current, args[-1].value))      # the stream comes last
        return self.status

    status = 0


class On:
    """A tensor, as far as a call asks, of some device."""
    is_cuda, dtype, shape = True, torch.float16, (4, 32)

    def __init__(self, device):
        self.device = torch.device(device)

    def is_contiguous(self):
        return True

    def dim(self):
        return 2

    def data_ptr(self):
        return 0x10000


@pytest.mark.parametrize("device,index", [("cuda:0", 0), ("cuda:1", 1)])
def test_the_tensors_device_is_current_at_the_launch(monkeypatch, device, index):
    m = Machine(monkeypatch)
    tf.silu_mul(On(device), out=On(device))
    assert m.calls == [(index, 100 + index)] and m.current == 0
    m.status = tf.TF_ERR_ALIGN
    m.tf_status_str = lambda status: b"misaligned"
    with pytest.raises(tf.TileFuseError):
        tf.silu_mul(On(device), out=On(device))
