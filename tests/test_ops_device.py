"""Which device and stream the operators' Python calls run on, where the current device is another one: without a GPU, with torch's state and the library replaced."""
import contextlib
import types

import pytest
import torch

from paper_2012_15469_amd import ops


class Machine:
    """Two GPUs' current streams, the current device, and what the library is called with while which of them is current."""

    def __init__(self, monkeypatch, device, streams):
        self.device, self.streams, self.calls = device, dict(streams), []
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.device, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: self.streams[i], raising=False)
        monkeypatch.setattr(torch.cuda, "stream", self.on_stream)
        monkeypatch.setattr(torch.cuda, "device", lambda d: self.on_device(d.index if isinstance(d, torch.device) else d))
        library = types.SimpleNamespace(**{name: self.recorded(name) for name in ("cada_adamw_step", "cada_adamw_moments", "cada_adamw_destroy")})
        monkeypatch.setattr(ops, "_lib", library)

    def recorded(self, name):
        def call(*args):
            self.calls.append((name, self.device, self.streams[self.device]))
            return 0
        return call

    @contextlib.contextmanager
    def on_device(self, index):
        before, self.device = self.device, index
        yield
        self.device = before

    @contextlib.contextmanager
    def on_stream(self, s):
        with self.on_device(s.device.index):
            before, self.streams[self.device] = self.streams[self.device], s.cuda_stream
            yield
            self.streams[self.device] = before


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("streams", [{0: 7, 1: 7}, {0: 5, 1: 7}, {0: 7, 1: 5}], ids=str)
@pytest.mark.parametrize("bits", [8, 32])
def test_moments_and_steps_of_a_plan_on_another_device(monkeypatch, bits, streams, current):
    m = Machine(monkeypatch, current, streams)
    opt = ops.AdamW.__new__(ops.AdamW)
    opt.plan, opt.device, opt.stream, opt.state_bits, opt.lr, opt.t = 1, torch.device("cuda", 1), types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=7), bits, 1e-3, 0
    opt.m = opt.v = (torch.zeros(256, dtype=torch.int8), torch.zeros(1)) if bits == 8 else torch.zeros(256)
    try:
        values = opt.moments()
        assert all(x.dtype == torch.float32 and x.shape == (256,) for x in values)
        assert m.calls == ([("cada_adamw_moments", 1, 7)] if bits == 8 else []) and m.device == current and m.streams == streams
        opt.step()
        assert m.calls[-1][:2] == ("cada_adamw_step", 1) and opt.t == 1 and m.device == current
    finally:
        opt.plan = None          # (no plan of the library's)
