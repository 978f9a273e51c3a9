"""What the experts' products of an EPBuffer wait for and what waits for them, with streams and events that only record it: no GPU."""
import contextlib
import threading

import pytest
import torch

from paper_2603_13606_amd import buffer


class Stream:
    def __init__(self, address, torchs=True, device=0):
        self.cuda_stream, self.stream_id, self.device_index = address, address + 100 if torchs else address, device
        self.log, self.capturing = [], False

    def wait_event(self, event):
        self.log.append(("waits for", event))

    def wait_stream(self, other):
        self.log.append(("waits for stream", other.cuda_stream))


class Event:
    def __init__(self):
        self.stream = None

    def record(self, stream):
        self.stream = stream.cuda_stream
        stream.log.append(("event", self))

    def synchronize(self):
        waited.append(self)


waited = []


@pytest.fixture
def buf(monkeypatch):
    """A buffer whose last call ran on the communication stream, with a handle."""
    b = buffer.EPBuffer.__new__(buffer.EPBuffer)
    b.compute, b._comm, b._lock, b._comm_given = Stream(1), Stream(2), threading.Lock(), False
    b._order_event, b._order_streams, b._last_event = "last call", (2,), None
    b.handle = buffer.EPHandle("raw", None, 4)
    current = [b.compute]
    waited.clear()

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def product(*args, handle=None, stream=None, **kw):
        assert handle == "raw"
        (current[-1] if stream is None else stream).log.append("product")

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: current[-1])
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: current[-1].capturing)
    monkeypatch.setattr(buffer.ep, "ep_expert_product", product)
    monkeypatch.setattr(buffer.ep, "ep_expert_product_backward", product)
    monkeypatch.setattr(buffer.ep, "ep_handle_destroy", lambda raw: waited.append("destroyed"))
    return b


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def forward(b):
    return b.expert_product(bf(6, 16), bf(2, 8, 16), b.handle)


def backward(b):
    return b.expert_product_backward(bf(6, 8), b.handle, bf(2, 8, 16))


@pytest.mark.parametrize("call", [forward, backward])
def test_products_run_on_the_compute_stream_behind_the_calls_made(buf, call):
    call(buf)
    assert [e if isinstance(e, str) else e[0] for e in buf.compute.log] == ["waits for", "product", "event"]
    assert buf.compute.log[0][1] == "last call" and buf._comm.log == []
    assert buf._order_event == "last call" and buf._order_streams == (2,), "nothing that was not told to waits for a product"


@pytest.mark.parametrize("call", [forward, backward])
def test_a_handle_is_destroyed_behind_its_products(buf, call):
    """Of every stream they ran on, whatever other calls the handle has had since."""
    call(buf)
    side = Stream(3)
    with torch.cuda.stream(side):
        call(buf)
        call(buf)
    buf._last_event = Event()      # a combine on the communication stream
    buf.destroy_handle(buf.handle)
    last = [[e[1] for e in s.log if e[0] == "event"][-1] for s in (buf.compute, side)]
    assert waited[-1] == "destroyed" and all(e in waited for e in last + [buf._last_event]) and not buf.handle.alive


def test_products_under_capture_leave_no_event(buf):
    """An event of a capture can't be waited for outside of it, and the capture can't wait for calls made before."""
    buf.compute.capturing = True
    forward(buf)
    assert buf.compute.log == ["product"]
    buf.compute.capturing = False
    buf.destroy_handle(buf.handle)
    assert waited == ["destroyed"]


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("capturing", [False, True])
def test_a_stream_of_somebody_else_is_not_remembered(buf, call, capturing):
    """Its owner may destroy it while the handle lives: the product runs on the communication stream, in its place."""
    theirs = Stream(7, torchs=False)
    theirs.capturing = capturing
    with torch.cuda.stream(theirs):
        call(buf)
    assert [e if isinstance(e, str) else e[0] for e in buf._comm.log] == ["waits for stream", "product", "event"]
    assert buf._comm.log[0][1] == 7 and theirs.log == [("waits for", buf._comm.log[-1][1])]
    assert list(buf.handle.products) == ([] if capturing else [2])


@pytest.mark.parametrize("call", [forward, backward])
def test_products_of_a_destroyed_handle_are_refused(buf, call):
    """As in a backward pass that comes too late: the library has freed what the handle points to."""
    buf.destroy_handle(buf.handle)
    with pytest.raises(ValueError):
        call(buf)
    assert "product" not in buf.compute.log
