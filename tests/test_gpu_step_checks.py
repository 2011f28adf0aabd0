"""The device-checked build on the calls of a device-side step: nothing is recorded on valid input, and bad blocks are."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import _lib  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import check_out, reference  # noqa: E402
from tests.test_gpu_checks import checked  # noqa: E402, F401
from tests.test_gpu_maps import Case, same  # noqa: E402
from tests.test_gpu_shared import attend, shared_batch  # noqa: E402

KINDS = [([(1280, [(30, 1)] * 5), (64, [(2000, 1)])], "tail"), ([(256, [(30, 1)] * 3)], "short"),
         ([(512, [(128, 128), (130, 1)])], "wide, apart"), ([(1024, [(128, 128), (9, 1), (9, 1), (9, 1)])], "wide"), ([(704, [(20, 20), (45, 9)])], "narrow")]


@pytest.mark.parametrize("groups,what", KINDS)
def test_shared_attention(checked, groups, what):  # noqa: F811
    print_case(f"checked build: shared prefixes, {what}")
    b = shared_batch(groups, 8, 2, 128, 5)
    ak.device_checks(reset=True)
    want = reference(b)
    out, lse = attend(b)
    check_out(b, out, lse, want, what)
    assert ak.device_checks() == (0, 0)
    bt = b["bt"].copy()
    bt[-1, 1] = len(b["pool"][0]) + 3                     # a block of the last request (and, if it is alone, of its group)
    attend(b, bt=bt)
    kind, count = ak.device_checks()
    # (requests that fill their own tiles are not shared: test_shared's tolerances hold either way)
    if len(groups[-1][1]) == 1 or what in ("short", "wide, apart"):
        assert kind == _lib.CHECK_BLOCK and count >= 1
    else:                                                 # shared keys are read through the group's first table
        assert (kind, count) == (0, 0)


def test_maps(checked):  # noqa: F811
    for mean_new, cap in ((3, None), (300, 20_000)):
        print_case(f"checked build: maps, {mean_new} new")
        c = Case(3, 40, 60, mean_new, 1.0)
        c.slot_cap = cap or c.slot_cap
        t = c.tensors()
        ak.batch_maps(**t)
        same(t, c.want())
        assert ak.device_checks() == (0, 0)
        c.free[:] = np.where(np.arange(len(c.free)) % 2, c.free, -2)
        t = c.tensors()
        ak.batch_maps(**t)
        same(t, c.want())
        kind, count = ak.device_checks()
        assert kind == _lib.CHECK_BLOCK and count >= 1
