"""What PrefillEngine.evict refuses of its destination blocks, before any device work (CPU: the weights are a
stand-in that has a device tensor's shape)."""

from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import BatchPlan  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402

HKV, PHYS, PRIVATE = 2, 12, 4


class Weights:
    """A contiguous fp32 device tensor, as far as the checks look."""
    is_cuda = True

    def __init__(self, *shape):
        self.shape = shape

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def element_size(self):
        return 4

    def is_floating_point(self):
        return True


@pytest.fixture
def evict(monkeypatch):
    """evict(dst_tables) of a batch of 40 and 20 tokens in blocks 3, 4, 5 and 6, 7, down to 20; destinations that pass
    reach the stream's check, which stops the call."""
    eng = PrefillEngine(4, HKV, 64, 8, PHYS, 2, device="cpu", num_cus=4, kv_format="mx4", private_blocks=PRIVATE)
    plan = BatchPlan(np.array([[3, 4, 5], [6, 7, -1]], np.int32), np.array([0, 40, 60], np.int32),
                     np.array([40, 20], np.int32), np.zeros(2, np.int32), np.zeros(2, np.int32),
                     np.arange(60, dtype=np.int32), 40, 40)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    return lambda dst, keep=20: eng.evict(SimpleNamespace(plan=plan), Weights(2, HKV, 40), keep, dst)


def test_private_blocks_pass(evict):
    for dst in ([[12, 13], [14, 15]], [[15, 12, 0], [13, 14, 99]]):      # (what is behind ceil(keep / 16) is not looked at)
        with pytest.raises(ValueError, match="captured"):
            evict(np.array(dst, np.int32))
    with pytest.raises(ValueError, match="captured"):
        evict(np.array([[12], [14]], np.int64), 16)


@pytest.mark.parametrize("block", [0, 2, 8, 11])       # resident, free or scratch: none in the batch
def test_blocks_of_the_cache_are_refused(evict, block):
    for at in range(4):
        dst = np.array([12, 13, 14, 15], np.int32)
        dst[at] = block
        with pytest.raises(ValueError, match="the block cache"):
            evict(dst.reshape(2, 2))


def test_other_refusals_name_what_is_wrong(evict):
    for dst, word in (([[12, 5], [13, 14]], "of the batch"), ([[12, 16], [13, 14]], "outside"), ([[12, -1], [13, 14]], "outside"),
                      ([[12, 13], [13, 14]], "twice"), ([[12, 13]], "dst_tables"), ([[12], [13]], "dst_tables")):
        with pytest.raises(ValueError, match=word):
            evict(np.array(dst, np.int32))


def test_block_numbers_are_not_wrapped_or_rounded(evict):
    """Numbers of more than 32 bits, whose low halves are private blocks, and numbers that are no integers."""
    with pytest.raises(ValueError, match="outside"):
        evict(np.array([[12, 13], [14, (1 << 32) + 15]], np.int64))
    with pytest.raises(ValueError, match="outside"):
        evict(np.array([[12, 13], [14, 15 - (1 << 32)]], np.int64))
    with pytest.raises(ValueError, match="integers"):
        evict(np.array([[12, 13], [14, 15.5]]))
