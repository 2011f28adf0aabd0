"""PrefillEngine.resume: the batch of sessions that were cut, and what it refuses (CPU: the plan that it uploads)."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import BatchPlan  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402

PHYS, PRIVATE = 12, 9


@pytest.fixture
def resume(monkeypatch):
    """resume() that gives its plan."""
    eng = PrefillEngine(4, 2, 64, 8, PHYS, 2, device="cpu", num_cus=4, kv_format="mx4", private_blocks=PRIVATE)
    monkeypatch.setattr(eng, "upload", lambda plan, stream: plan)
    return eng.resume


def test_the_plan():
    eng = PrefillEngine(4, 2, 64, 8, PHYS, 2, device="cpu", num_cus=4, kv_format="mx4", private_blocks=PRIVATE)
    eng.upload = lambda plan, stream: (plan, stream)
    p, stream = eng.resume([[12, 20, 7], [15, 13, 14]], [15, 32], [3, 1], [1000, 33], stream=5)
    assert stream == 5
    assert p.block_tables.tolist() == [[12, 20, -1], [15, 13, 14]]        # (what is behind the blocks needed is not looked at)
    assert p.cu_q.tolist() == [0, 3, 4] and p.seq_lens.tolist() == [18, 33] and p.true_lens.tolist() == [1000, 33]
    assert p.prefix_lens.tolist() == [15, 32] and p.hit_blocks.tolist() == [0, 2]
    assert p.slot_mapping.tolist() == [12 * 16 + 15, 20 * 16, 20 * 16 + 1, 14 * 16]
    assert (p.max_q_len, p.max_seq_len) == (3, 33)
    assert all(x.dtype == np.int32 for x in (p.block_tables, p.cu_q, p.seq_lens, p.prefix_lens, p.hit_blocks, p.slot_mapping,
                                             p.true_lens))


def test_true_lens_are_one_for_each_request():
    eng = PrefillEngine(4, 2, 64, 8, PHYS, 2, device="cpu", num_cus=4, kv_format="mx4", private_blocks=PRIVATE)
    i32 = lambda *x: np.array(x, np.int32)                                        # noqa: E731
    plan = BatchPlan(i32([13]), i32(0, 1), i32(5), i32(4), i32(0), i32(13 * 16 + 4), 1, 5, true_lens=i32(9, 9))
    with pytest.MonkeyPatch.context() as m:
        m.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
        m.setattr(eng, "_torch_stream", lambda s: None)
        with pytest.raises(ValueError, match="true_lens"):
            eng.upload(plan)
    assert eng._turn == 0


def test_empty_batches(resume):
    p = resume(np.zeros((0, 3), int), [], [], [])
    assert p.n_reqs == 0 and p.cu_q.tolist() == [0] and p.slot_mapping.tolist() == []
    p = resume([[13]], [16], [0], [40])
    assert p.cu_q.tolist() == [0, 0] and p.seq_lens.tolist() == [16] and p.max_q_len == 0


@pytest.mark.parametrize("args,word", [
    (([[12, 13]], [20], [1], [20]), "true_lens"), (([[12, 13]], [-1], [2], [20]), "held"), (([[12, 13]], [20], [-1], [20]), "held"),
    (([[12, 13]], [20], [1], [1 << 31]), "true_lens"),
    (([[12]], [16], [1], [99]), "2 blocks"), (([[11, 12]], [16], [1], [99]), "private"), (([[12, 21]], [16], [1], [99]), "private"),
    (([[12, -1]], [16], [1], [99]), "private"), (([[12, (1 << 32) + 13]], [16], [1], [99]), "private"),
    (([12, 13], [16], [1], [99]), "tables"), (([[12, 13]], [16, 1], [1], [99]), "tables"), (([[12, 13]], [16], [1, 1], [99]), "tables"),
    (([[12, 13], [14, 13]], [16, 16], [1, 1], [99, 99]), "one slot"),
    (([[12, 13]], [16], [1], [99, 100]), "tables"), (([[12, 13]], [16.5], [1], [99]), "integers"),
])
def test_refusals(resume, args, word):
    with pytest.raises(ValueError, match=word):
        resume(*args)
