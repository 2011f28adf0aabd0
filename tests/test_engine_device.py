"""The engine's calls run on its own device, whichever is torch's current one (CPU: devices, streams and the library are
stand-ins)."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import engine  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.test_engine_streams import D, HKV, HQ, Tensor, world  # noqa: E402,F401


@pytest.fixture
def on(world, monkeypatch):
    """The library's calls as (name, the device that was current); the engine's is 1, torch's current one 0."""
    got, now = [], [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            now.append(self.index)

        def __exit__(self, *exc):
            now.pop()

    class Lib:
        def __getattr__(self, name):
            return lambda *args: got.append((name, now[-1], args)) or 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(engine, "lib", lambda: Lib())
    world.eng.device = torch.device("cuda", 1)
    world.eng._y = torch.zeros(1 << 16, dtype=torch.uint8)
    return got


class Event:
    def __init__(self, handle):
        self.cuda_event = handle


def test_every_call_makes_the_engines_device_the_current_one(world, on):
    eng, db = world.eng, world.db
    rows, q, lse, x, w = Tensor(5, HKV, D), Tensor(5, HQ, D), Tensor(5, HQ, size=4), Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32)
    eng.scatter(db, rows, rows)
    eng.attention(db, q, q)
    eng.attention(db, q, q, lse=lse)
    eng.attention(db, q, q, events=[Event(71), Event(72), Event(73)])
    eng.attention_weights(db, q, lse, Tensor(1, HKV, 5, size=4))
    eng.project(db, x, w, q, rows, rows, 1e4)
    eng.project_to_pool(db, x, w, q, 1e4)
    assert [(name, device) for name, device, _ in on] == [(f"arckv_{name}", 1) for name in (
        "kv_scatter", "prefill_attention", "prefill_attention_lse", "prefill_attention_timed", "attention_weights", "qkv_rope",
        "qkv_rope_to_pool")]
    assert on[3][2][-4:] == (0, 71, 72, 73)              # the stream, then its events


def test_a_device_without_an_index_is_the_one_that_is_current(monkeypatch):
    """cuda: the device of the day the engine is made, not of each later call."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert PrefillEngine._device_of("cuda") == torch.device("cuda", 3)
    assert PrefillEngine._device_of("cuda:1") == torch.device("cuda", 1)
    assert PrefillEngine._device_of("cpu") == torch.device("cpu")
