"""What the engine's calls leave in a graph that captures them (CPU: streams and the library are stand-ins): a
replay must read and write memory that the engine's later calls do not use."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import engine  # noqa: E402
from tests.test_engine_streams import D, HKV, HQ, Tensor, attend, world  # noqa: E402,F401


@pytest.fixture
def calls(world, monkeypatch):
    """The arguments of the library's calls; the batch's arrays lie in slot 2 of the metadata ring."""
    got = []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: got.append((name, args)) or 0

    monkeypatch.setattr(engine, "lib", lambda: Lib())
    eng = world.eng
    eng._dev_meta = [torch.zeros(64, dtype=torch.int32) for _ in range(4)]
    eng._stage = [torch.zeros(64, dtype=torch.int32) for _ in range(4)]
    world.db.cu_q = eng._dev_meta[2][8:10]
    return got


def workspace(call):
    return call[1][-3]                 # ..., workspace, ws_bytes, stream


def test_a_captured_attention_has_a_workspace_of_its_own(world, calls):
    eng = world.eng
    attend(world, None)
    assert workspace(calls[0]) == eng._ws.data_ptr()
    world.capturing.add(0)
    keep, real = [], torch.empty

    def empty(*shape, **kw):
        keep.append(real(*shape, **kw))
        return keep[-1]

    with pytest.MonkeyPatch.context() as m:
        m.setattr(torch, "empty", empty)
        attend(world, None)
        attend(world, None)
    assert [workspace(c) for c in calls[1:]] == [t.data_ptr() for t in keep] and all(t.numel() == 1024 for t in keep)
    assert eng._ws.data_ptr() not in [t.data_ptr() for t in keep]


def test_a_captured_producer_has_a_table_of_its_own(world, calls):
    eng = world.eng
    eng._y = torch.zeros(1 << 16, dtype=torch.uint8)
    rows, q, x, w = Tensor(5, HKV, D), Tensor(5, HQ, D), Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32)
    for capture in (False, True):
        if capture:
            world.capturing.add(0)
        calls.clear()
        eng.project(world.db, x, w, q, rows, rows, 1e4)
        eng.project_to_pool(world.db, x, w, q, 1e4)
        assert [eng._y.data_ptr() in c[1] for c in calls] == [not capture] * 2


@pytest.mark.parametrize("call", ["scatter", "attention", "attention_weights", "project", "project_to_pool"])
def test_the_ring_lets_go_of_a_captured_batch(world, calls, call):
    eng, db = world.eng, world.db
    rows, q, x, w = Tensor(5, HKV, D), Tensor(5, HQ, D), Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32)
    args = dict(scatter=(rows, rows), attention=(q, q), attention_weights=(q, Tensor(5, HQ, size=4), Tensor(1, HKV, 5, size=4)),
                project=(x, w, q, rows, rows, 1e4), project_to_pool=(x, w, q, 1e4))[call]
    getattr(eng, call)(db, *args)
    assert all(t is not None for t in eng._dev_meta)
    world.capturing.add(0)
    getattr(eng, call)(db, *args)
    assert [t is None for t in eng._dev_meta] == [t is None for t in eng._stage] == [False, False, True, False]


def test_staging_is_not_captured(world):
    world.capturing.add(0)
    before = world.eng.cache.stats()
    with pytest.raises(ValueError, match="captured"):
        world.eng.prepare([np.arange(20, dtype=np.int32)])
    with pytest.raises(ValueError, match="captured"):
        world.eng.upload(world.db.plan)
    assert world.eng.cache.stats() == before
