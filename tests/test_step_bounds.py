"""The bounds that a step batch fixes, and what they cost: a batch of decodes that names no max_new gets the kernels and the memory of
one token for each request (CPU)."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_21238_amd import SharedBounds, engine, shared_prefix_sizes  # noqa: E402
from tests.test_step_batch import GOOD, Passed, call, eng  # noqa: E402, F401


def bounds(eng, monkeypatch, **kw):  # noqa: F811
    seen = []
    monkeypatch.setattr(engine, "shared_prefix_sizes", lambda b: seen.append(b) or shared_prefix_sizes(b))
    with pytest.raises(Passed):
        call(eng, **kw)
    return seen[-1]


@pytest.mark.parametrize("kw,max_new,max_group_q", [
    (dict(max_tokens=3), 1, 2), (dict(max_tokens=6), 2, 4), (dict(max_tokens=7), 3, 6), (dict(max_tokens=1), 1, 1), (dict(max_tokens=0), 0, 0),
    (dict(max_tokens=6, max_new=6), 6, 6), (dict(max_tokens=6, max_new=9), 6, 6), (dict(max_tokens=6, max_new=1), 1, 2),
    (dict(tables=np.zeros((0, 4), np.int32), held=[], group_sizes=[], prefix_lens=[], free_blocks=[], max_tokens=5), 5, 0)])
def test_max_new(eng, monkeypatch, kw, max_new, max_group_q):  # noqa: F811
    b = bounds(eng, monkeypatch, **kw)
    assert (b.max_q, b.max_new, b.max_group_q) == (kw["max_tokens"], max_new, max_group_q)


def test_decode_batches_reserve_what_a_token_each_needs(eng, monkeypatch):  # noqa: F811
    """1000 requests, tables of 8192 tokens, 32 / 8 heads of 128: 123 MiB, where one request with all of the rows takes 1120."""
    n = 1000
    eng.hq, eng.hkv, eng.d, eng.num_cus = 32, 8, 128, 256
    b = bounds(eng, monkeypatch, tables=np.full((n, 512), -1), held=np.zeros(n, int), group_sizes=[n], prefix_lens=[0], free_blocks=[], max_tokens=n)
    assert b == SharedBounds(n, 1, n, n, 1, 512, 32, 8, 128, 256)
    assert shared_prefix_sizes(b)[1] >> 20 < 130
    whole = SharedBounds(n, 1, n, n, n, 512, 32, 8, 128, 256)
    assert shared_prefix_sizes(whole)[1] >> 20 > 1000
