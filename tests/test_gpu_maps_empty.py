"""Steps without a slot: nobody gets a token, and the call ends well for any number of requests."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.test_gpu_maps import Case, _need_gpu, same  # noqa: E402, F401


@pytest.mark.parametrize("n", [0, 5, 2048, 2049, 3000])
@pytest.mark.parametrize("mean_new", [0, 3])
def test_no_slots(n, mean_new):
    print_case(f"maps without slots: {n} requests, {mean_new} new")
    c = Case(n + mean_new, n, 9, mean_new, 1.0)
    c.slot_cap = 0
    t = c.tensors()
    ak.batch_maps(**t)
    same(t, c.want())


def test_no_slots_captured():
    print_case("maps without slots, captured")
    c = Case(7, 2500, 9, 3, 1.0)
    c.slot_cap = 0
    t = c.tensors()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ak.batch_maps(**t)
    for _ in range(3):
        t["seq_lens"].fill_(-7)
        t["cu_q"].fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        same(t, c.want())
