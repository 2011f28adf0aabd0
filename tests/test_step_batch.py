"""What PrefillEngine.step_batch, advance and shared_attention refuse, before any device work (CPU: streams are stand-ins)."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd.engine import PrefillEngine, StepBatch, StepPlan  # noqa: E402
from tests.test_step_refusals import BOUNDS, Tensor, f32, i32  # noqa: E402

PHYS, PRIVATE = 20, 12


class Passed(Exception):
    pass


@pytest.fixture
def eng(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    e = PrefillEngine(8, 2, 64, 8, PHYS, 2, device="cpu", num_cus=4, private_blocks=PRIVATE)
    monkeypatch.setattr(e, "_torch_stream", lambda stream: (_ for _ in ()).throw(Passed()))
    return e


TABLES = [[3, 4, 5, 20, -1], [3, 4, 5, 21, -1], [7, 22, -1, -1, -1]]
GOOD = dict(tables=TABLES, held=[50, 60, 17], group_sizes=[2, 1], prefix_lens=[48, 0], max_tokens=6, free_blocks=[23, 24, 25])


def call(eng, **kw):
    return eng.step_batch(**{**GOOD, **kw})


def test_what_passes(eng):
    for kw in (dict(), dict(group_sizes=[], prefix_lens=[]), dict(free_blocks=[]), dict(true_lens=[50, 600, 17]), dict(max_new=2),
               dict(prefix_lens=[33, 17]), dict(held=[48, 48, 0], free_blocks=[20, 21, 22]), dict(max_tokens=0),
               dict(tables=np.array(TABLES, np.int64)), dict(prefix_lens=[48, 16])):
        with pytest.raises(Passed):
            call(eng, **kw)


@pytest.mark.parametrize("kw,word", [
    (dict(held=[50, 60]), "tables must be"), (dict(tables=[3, 4]), "tables must be"), (dict(prefix_lens=[48]), "one per group"),
    (dict(true_lens=[50, 60]), "true_lens"), (dict(held=[50.0, 60.0, 17.0]), "integers"), (dict(free_blocks=[23.5]), "integers"),
    (dict(max_tokens=-1), "max_tokens"), (dict(max_new=-1), "max_new"), (dict(held=[-1, 60, 17]), "0 <= held"), (dict(held=[50, 81, 17]), "0 <= held"),
    (dict(true_lens=[49, 60, 17]), "true length"), (dict(true_lens=[50, 60, 1 << 31]), "true length"), (dict(group_sizes=[2, 2]), "groups"),
    (dict(group_sizes=[2, 0], prefix_lens=[0, 0]), "groups"), (dict(group_sizes=[3, 0], prefix_lens=[16, 0]), "groups"),
    (dict(tables=[[3, 4, 5, 20, -1], [3, 4, 5, 32, -1], [7, 22, -1, -1, -1]]), "outside"),
    (dict(tables=[[3, 4, 5, 20, -1], [3, 4, 5, -1, -1], [7, 22, -1, -1, -1]]), "outside"),
    (dict(tables=[[3, 4, 5, (1 << 32) + 20, -1], [3, 4, 5, 21, -1], [7, 22, -1, -1, -1]]), "outside"),
    (dict(free_blocks=[19]), "private"), (dict(free_blocks=[32]), "private"), (dict(free_blocks=[23, 23]), "twice"),
    (dict(free_blocks=[20]), "holds"), (dict(tables=[[3, 4, 5, 20, -1], [3, 4, 5, 20, -1], [7, 22, -1, -1, -1]]), "belongs to two"),
    (dict(prefix_lens=[51, 0]), "holds fewer"), (dict(prefix_lens=[-1, 0]), "holds fewer"),
    (dict(prefix_lens=[49, 0]), "different blocks"), (dict(tables=[[3, 4, 5, 20, -1], [3, 6, 5, 21, -1], [7, 22, -1, -1, -1]]), "different"),
    (dict(group_sizes=[3], prefix_lens=[16]), "different")])
def test_refusals(eng, kw, word):
    with pytest.raises(ValueError, match=word):
        call(eng, **kw)


def test_wrapped_free_blocks_are_refused(eng):
    with pytest.raises(ValueError, match="private"):
        call(eng, free_blocks=np.array([(1 << 32) + 23], np.int64))


def test_other_pools_and_capture_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(ValueError, match="bf16"):
        PrefillEngine(8, 2, 64, 8, PHYS, 2, device="cpu", num_cus=4, kv_format="mx4").step_batch(**GOOD)
    with pytest.raises(ValueError, match="captured"):
        PrefillEngine(8, 2, 64, 8, PHYS, 2, device="cpu", num_cus=4, private_blocks=PRIVATE).step_batch(**GOOD)


def test_calls_of_a_step_refuse(eng):
    sb = StepBatch(StepPlan(3), *[None] * 5, 0, 0, 0, 0, n_tokens=6, bounds=BOUNDS)
    for bad in (i32(2), f32(3), Tensor(3), i32(3, 1)):
        with pytest.raises(ValueError, match="new_tokens"):
            eng.advance(sb, bad)
    q = Tensor(6, 8, 64)
    for kw in (dict(q=Tensor(5, 8, 64)), dict(out=Tensor(6, 8, 32)), dict(lse=f32(6, 2)), dict(lse=i32(6, 8)), dict(q=f32(6, 8, 64))):
        with pytest.raises(ValueError):
            eng.shared_attention(sb, **{**dict(q=q, out=q), **kw})
    with pytest.raises(ValueError, match="shared_attention"):
        eng.attention(sb, q, q)
    with pytest.raises(ValueError, match="StepBatch"):
        eng.evict(sb, f32(3, 2, 80), 16, np.zeros((3, 1), np.int32))
