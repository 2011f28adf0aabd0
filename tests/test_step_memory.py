"""A StepBatch may be let go of right after any of its calls: its memory is held for the stream that the call went to (CPU: streams,
events and the library are stand-ins)."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import SharedBounds  # noqa: E402
from paper_2606_21238_amd.engine import StepBatch, StepPlan  # noqa: E402
from tests.test_engine_streams import D, HKV, HQ, Tensor, world  # noqa: E402, F401

HOME = 11


class Memory(Tensor):
    """One of the batch's own tensors; `held`: the streams that it was recorded for."""

    def __init__(self, *shape):
        super().__init__(*shape, size=4)
        self.held = []

    def numel(self):
        return 64

    def record_stream(self, stream):
        self.held.append(stream.cuda_stream)


def calls(eng, sb):
    rows, q, x, w = Tensor(5, HKV, D), Tensor(5, HQ, D), Tensor(5, 32), Tensor((HQ + 2 * HKV) * D, 32)
    new, lse = Tensor(1, size=4), Tensor(5, HQ, size=4)
    new.is_floating_point = lambda: False
    return {"advance": lambda s: eng.advance(sb, new, stream=s), "shared_attention": lambda s: eng.shared_attention(sb, q, q, stream=s),
            "scatter": lambda s: eng.scatter(sb, rows, rows, stream=s), "project": lambda s: eng.project(sb, x, w, q, rows, rows, 1e4, stream=s),
            "project_to_pool": lambda s: eng.project_to_pool(sb, x, w, q, 1e4, stream=s),
            "attention_weights": lambda s: eng.attention_weights(sb, q, lse, Tensor(1, HKV, 5, size=4), stream=s)}


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", ["advance", "shared_attention", "scatter", "project", "project_to_pool", "attention_weights"])
def test_every_call_holds_the_memory(world, name, raw):  # noqa: F811
    m = [Memory(1, 1) for _ in range(6)]
    sb = StepBatch(StepPlan(1), *m[:4], None, 0, 0, 1024, 0, 5, 0, None, bounds=SharedBounds(1, 1, 5, 5, 5, 1, HQ, HKV, D, 4), group_start=m[0],
                   prefix_lens=m[0], free_blocks=m[0], free_count=m[0], work_plan=m[4], workspace=m[5], home=HOME, memory=m)
    world.eng._y = torch.zeros(4 * 5 * D, dtype=torch.uint8)
    call = calls(world.eng, sb)[name]
    on = lambda handle: handle if raw else torch.cuda.Stream(handle)  # noqa: E731
    call(on(HOME))
    assert [x.held for x in m] == [[]] * 6               # the stream that it goes back to
    call(on(22))
    assert [x.held for x in m] == [[22]] * 6
    world.capturing.add(33)                              # a captured call: the graph's owner keeps the batch
    call(on(33))
    assert [x.held for x in m] == [[22]] * 6


def test_planned_batches_are_not_asked(world):  # noqa: F811
    """Theirs lies in the engine's ring."""
    rows = Tensor(5, HKV, D)
    world.eng.scatter(world.db, rows, rows, stream=torch.cuda.Stream(22))
    assert world.log[-1] == ("call", "arckv_kv_scatter", 22)
