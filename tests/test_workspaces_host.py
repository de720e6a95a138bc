"""Which default workspace a call gets, with the device calls replaced by stand-ins (no GPU needed)."""
import contextlib
import threading
import types

import pytest
import torch


@pytest.fixture
def fake(monkeypatch):
    """The current stream as a number, buffers on the CPU, and a log of the stream that each was made on."""
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    state = types.SimpleNamespace(stream=1, capturing=False, made=[])

    @contextlib.contextmanager
    def on(stream):
        before, state.stream = state.stream, stream.cuda_stream
        yield
        state.stream = before

    zeros = torch.zeros

    def make(n, dtype, device):
        state.made.append(state.stream)
        return zeros(n, dtype=dtype)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state.capturing)
    monkeypatch.setattr(torch, "zeros", make)
    monkeypatch.setattr(vmb.vmb, "_raw_stream", lambda index: state.stream)
    monkeypatch.setattr(vmb.vmb, "_delta_ws", vmb.vmb.Workspace())
    state.get = lambda stream=None: vmb.delta_workspace(torch.device("cuda", 0), stream=stream)
    return state


def test_one_buffer_per_stream_made_on_it(fake):
    a, b = (types.SimpleNamespace(cuda_stream=n) for n in (5, 6))
    x, y, z = fake.get(a), fake.get(b), fake.get()
    assert len({t.data_ptr() for t in (x, y, z)}) == 3 and fake.made == [5, 6, 1]
    assert fake.get(a) is x and fake.get(b) is y and fake.get() is z and fake.stream == 1


def test_one_buffer_per_thread(fake):
    mine, others = fake.get(), []
    t = threading.Thread(target=lambda: others.append(fake.get()))
    t.start()
    t.join()
    assert others[0].data_ptr() != mine.data_ptr()


def test_a_captured_call_keeps_its_buffer_to_itself(fake):
    warm = fake.get()
    fake.capturing = True
    one, two = fake.get(), fake.get()
    fake.capturing = False
    assert len({t.data_ptr() for t in (warm, one, two)}) == 3 and fake.get() is warm


def test_growth_zero_fills_a_new_buffer_on_the_same_stream(fake):
    import paper_2412_16602_gb300 as vmb
    ws = vmb.vmb._delta_ws
    small = ws.get(300, torch.device("cuda", 0))
    small.fill_(7)
    large = ws.get(5000, torch.device("cuda", 0))
    assert small.numel() == 512 and large.numel() == 5120 and int(large.sum()) == 0
    assert ws.get(300, torch.device("cuda", 0)) is large and fake.made == [1, 1]
