"""Calls with tensors of several devices, with stand-ins for the devices (no GPU needed)."""
import contextlib
import types

import pytest
import torch


class On(torch.Tensor):
    """A CPU tensor that says it lies on the CUDA device `at`."""

    def get_device(self):
        return self.at


def tensor(at):
    t = torch.zeros(2).as_subclass(On)
    t.at = at
    return t


@pytest.fixture
def vmb(monkeypatch):
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    state = vmb.vmb
    now = types.SimpleNamespace(device=0, stream=0)

    @contextlib.contextmanager
    def device(index):
        before, now.device = now.device, index
        yield
        now.device = before

    @contextlib.contextmanager
    def stream(s):
        before, now.stream = now.stream, s.cuda_stream
        yield
        now.stream = before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(state, "_current_device", lambda: now.device)
    monkeypatch.setattr(state, "_several_devices", lambda: True)
    state.now = now
    yield state
    del state.now


def test_a_call_runs_on_the_device_of_its_tensors(vmb):
    call = vmb._on_its_stream(lambda *a, stream=None, **k: (vmb.now.device, vmb.now.stream))
    assert call(tensor(0)) == (0, 0) and call(tensor(1)) == (1, 0) and call(x=tensor(2)) == (2, 0) and call(None, 3.0) == (0, 0)
    s = types.SimpleNamespace(cuda_stream=9, device_index=1)
    assert call(tensor(1), stream=s) == (1, 9) and (vmb.now.device, vmb.now.stream) == (0, 0)
    with pytest.raises(ValueError):
        call(tensor(0), stream=s)


def test_tensors_of_two_devices_are_refused(vmb):
    vmb._one_device(tensor(1), tensor(1), None)
    for other in (tensor(0), tensor(2)):
        with pytest.raises(ValueError):
            vmb._one_device(tensor(1), None, other)


def test_one_device_alone_is_not_asked_for(vmb, monkeypatch):
    monkeypatch.setattr(vmb, "_several_devices", lambda: False)
    monkeypatch.setattr(vmb, "_current_device", None)
    call = vmb._on_its_stream(lambda *a, stream=None: vmb.now.stream)
    assert call(tensor(0)) == 0
    vmb._one_device(tensor(0), None)
