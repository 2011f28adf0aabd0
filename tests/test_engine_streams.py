"""One engine on several streams: what its calls queue on which stream, and in what order (CPU: streams, events
and the library are stand-ins that write down what is asked of them)."""

from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import BatchPlan, engine  # noqa: E402
from paper_2606_21238_amd.engine import DeviceBatch, PrefillEngine  # noqa: E402

HQ, HKV, D = 4, 2, 64


class Tensor:
    """A contiguous device tensor, as far as the engine looks."""
    is_cuda = True

    def __init__(self, *shape, size=2, at=0x1000):
        self.shape, self.size, self.at = shape, size, at

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.size

    def is_floating_point(self):
        return True

    def dim(self):
        return len(self.shape)

    def data_ptr(self):
        return self.at


@pytest.fixture
def world(monkeypatch):
    """(engine, batch, log): calls of the library go to the log as ("call", name, stream), events as
    ("record", event, stream) and ("wait", stream, event); world.current is torch's current stream."""
    log = []
    w = SimpleNamespace(log=log, current=0, capturing=set())

    class Event:
        n = 0

        def __init__(self):
            Event.n += 1
            self.n = Event.n

        def record(self, stream):
            log.append(("record", self.n, stream.cuda_stream))

    class Stream:
        def __init__(self, handle, device=None):
            self.cuda_stream = handle

        def synchronize(self):
            log.append(("host waits", self.cuda_stream))

        def wait_event(self, ev):
            log.append(("wait", self.cuda_stream, ev.n))

    class Use:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.before, w.current = w.current, self.stream.cuda_stream

        def __exit__(self, *exc):
            w.current = self.before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                log.append(("call", name, args[-1]))
                return 0
            return call

    for name, x in (("Event", Event), ("Stream", Stream), ("ExternalStream", Stream), ("stream", Use),
                    ("default_stream", lambda device=None: Stream(0)), ("current_stream", lambda device=None: Stream(w.current)),
                    ("is_current_stream_capturing", lambda: w.current in w.capturing)):
        monkeypatch.setattr(torch.cuda, name, x)
    monkeypatch.setattr(engine, "_current_stream", lambda index=None: w.current)
    monkeypatch.setattr(engine, "lib", lambda: Lib())
    w.eng = PrefillEngine(HQ, HKV, D, 8, 12, 2, device="cpu", num_cus=4)
    w.eng._ws = torch.zeros(4096, dtype=torch.uint8)
    plan = BatchPlan(np.array([[3]], np.int32), np.array([0, 5], np.int32), np.array([5], np.int32),
                     np.zeros(1, np.int32), np.zeros(1, np.int32), np.arange(5, dtype=np.int32), 5, 5)
    t = Tensor(1, 1, size=4)
    w.db = DeviceBatch(plan, t, t, t, t, t, 8, 1, 1024, 128, 5, 0x2000)
    return w


def attend(w, stream):
    """stream: None, a number (of a torch stream), or "raw" and a handle."""
    if isinstance(stream, tuple):
        stream = stream[1]
    elif stream is not None:
        stream = torch.cuda.Stream(stream)
    w.eng.attention(w.db, Tensor(5, HQ, D), Tensor(5, HQ, D), stream=stream)


def test_calls_on_one_stream_queue_nothing_between(world):
    for _ in range(3):
        attend(world, 11)
    assert world.log == [("call", "arckv_prefill_attention", 11)] * 3


def test_a_call_on_another_stream_waits_for_the_one_before(world):
    attend(world, 11)
    attend(world, 22)
    attend(world, None)            # torch's current stream, the default one
    attend(world, None)
    call = "arckv_prefill_attention"
    assert world.log == [("call", call, 11), ("record", 1, 11), ("wait", 22, 1), ("call", call, 22),
                                ("record", 2, 22), ("wait", 0, 2), ("call", call, 0), ("call", call, 0)]


def test_every_kind_of_call_takes_part(world):
    eng, db = world.eng, world.db
    rows, q, lse = Tensor(5, HKV, D), Tensor(5, HQ, D), Tensor(5, HQ, size=4)
    calls = [lambda s: eng.scatter(db, rows, rows, stream=s), lambda s: eng.attention(db, q, q, stream=s),
             lambda s: eng.attention(db, q, q, stream=s, lse=lse),
             lambda s: eng.attention_weights(db, q, lse, Tensor(1, HKV, 5, size=4), stream=s),
             lambda s: eng.project(db, Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32), q, rows, rows, 1e4, stream=s),
             lambda s: eng.project_to_pool(db, Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32), q, 1e4, stream=s)]
    for n, call in enumerate(calls):
        attend(world, 100 + n)
        world.log.clear()
        call(torch.cuda.Stream(200 + n))
        (kind, ev, old), wait, rest = world.log[0], world.log[1], world.log[2:]
        assert (kind, old) == ("record", 100 + n) and wait == ("wait", 200 + n, ev)
        assert [e[2] for e in rest] == [200 + n]


def test_a_buffer_is_replaced_once_every_stream_is_done_with_it(world):
    """Its memory goes back to the order of the stream that it was allocated on, which may not be the last user's:
    the host waits first.  With one stream alone that order is enough."""
    eng = world.eng
    on = {n: torch.cuda.Stream(n) for n in (11, 22, 33)}
    attend(world, 11)
    eng._ensure_ws(8192, eng._torch_stream(on[11]))
    eng._ensure_ws(8193, eng._torch_stream(on[11]))
    assert eng._ws.numel() == 8193 and ("host waits", 11) not in world.log
    attend(world, 22)
    eng._ensure_ws(9000, eng._torch_stream(on[22]))
    assert eng._ws.numel() == 9000 and world.log[-1] == ("host waits", 22)
    attend(world, 11)
    eng._ensure_ws(9001, eng._torch_stream(on[22]))                     # 22 waits for 11 in its own order
    assert ("host waits", 22) not in world.log[-3:]
    rows, q = Tensor(5, HKV, D), Tensor(5, HQ, D)
    for _ in range(2):
        eng.project(world.db, Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32), q, rows, rows, 1e4, stream=on[33])
    assert ("host waits", 33) not in world.log               # the first table replaces none
    eng._y = eng._y[:1]                                      # too small now
    eng.project_to_pool(world.db, Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32), q, 1e4, stream=on[22])
    assert ("host waits", 22) in world.log


def test_a_capturing_stream_waits_for_nothing(world):
    """An event from outside would end the capture; what follows goes on from the last stream that ran."""
    attend(world, 11)
    world.capturing.add(22)
    world.log.clear()
    attend(world, 22)
    assert world.log == [("call", "arckv_prefill_attention", 22)]
    attend(world, 11)
    assert world.log[1:] == [("call", "arckv_prefill_attention", 11)]


def test_a_stream_that_is_captured_meanwhile_is_not_waited_for(world):
    attend(world, 11)
    world.capturing.add(11)
    world.log.clear()
    attend(world, 22)
    assert world.log == [("call", "arckv_prefill_attention", 22)]


def test_a_raw_handle_is_not_touched_after_its_call(world):
    """Its owner may have destroyed it: the event is there already when the stream changes."""
    call = "arckv_prefill_attention"
    attend(world, ("raw", 11))
    attend(world, ("raw", 11))
    attend(world, 22)
    assert world.log == [("call", call, 11), ("record", 1, 11), ("call", call, 11), ("record", 2, 11), ("wait", 22, 2), ("call", call, 22)]
    world.log.clear()
    attend(world, ("raw", 22))           # the same stream by its handle
    attend(world, 22)                    # what follows has no event yet
    attend(world, 33)
    assert world.log == [("call", call, 22), ("record", 3, 22), ("call", call, 22), ("record", 4, 22), ("wait", 33, 4), ("call", call, 33)]
    world.capturing.add(44)
    world.log.clear()
    attend(world, ("raw", 44))           # an event of a capture is of no use outside it
    assert world.log == [("call", call, 44)]
