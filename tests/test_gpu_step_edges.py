"""Steps whose requests come and go: members of a group that have ended, rows that see no key.  Tolerances of mx4_helpers.reference."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import check_out, reference  # noqa: E402
from tests.test_gpu_shared import attend, bounds_of, shared_batch  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


# (groups, requests that have ended, what): the routes of the own keys, and groups at either end of the batch
ENDED = [([(2048, [(9, 0), (40, 1), (17, 1)])], [0], "tail"),
         ([(2048, [(9, 0), (4, 0), (17, 1)]), (128, [(3, 0), (20, 2), (5, 0)]), (1600, [(8, 0), (1, 1)])], [0, 1, 3, 5, 6], "tail, several"),
         ([(704, [(9, 0), (45, 20), (33, 9)])], [0], "narrow"),
         ([(1024, [(9, 0), (128, 128), (9, 1), (40, 1), (12, 1)])], [0], "wide"),
         ([(256, [(9, 0), (40, 1), (17, 1)])], [0], "one launch")]


@pytest.mark.parametrize("groups,ended,what", ENDED)
def test_the_first_request_of_a_group_has_ended(groups, ended, what):
    """It holds nothing any more and its table names no block: the others go on sharing what their own tables name."""
    print_case(f"ended members: {what}")
    for hq, hkv, d in ((8, 2, 128), (4, 2, 64)):
        b = shared_batch(groups, hq, hkv, d, 61)
        want = reference(b)
        b["seq"][ended] = 0
        b["bt"][ended] = -1
        out, lse = attend(b)
        check_out(b, out, lse, want, what)


@pytest.mark.parametrize("n", [3, 500])
def test_the_first_requests_of_many_groups_have_ended(n):
    """Groups of three whose first has ended (500: the plan does not fit LDS)."""
    print_case(f"ended members of {n} groups")
    rng = np.random.default_rng(n)
    groups = [(128, [(5, 0), (int(rng.integers(1, 40)), 1), (int(rng.integers(1, 40)), 1)]) for _ in range(n)]
    b = shared_batch(groups, 4, 2, 64, 63, room=100)
    want = reference(b)
    b["seq"][::3] = 0
    b["bt"][::3] = -1
    out, lse = attend(b)
    check_out(b, out, lse, want, f"{n} groups")


# (groups, alone, requests without keys, what)
NO_KEYS = [([(256, [(30, 1)] * 3)], [(1, 1), (7, 1), (1, 1)], [3, 5], "one launch"),
           ([(128, [(5, 1)] * 4)] * 128, [(1, 1)] * 5 + [(60, 1)] + [(1, 1)] * 3, [512, 513, 514, 515, 516, 518, 519, 520], "tail, short tables"),
           ([(2048, [(30, 1)] * 3)], [(1, 1), (7, 1), (1, 1)], [3, 5], "tail, long tables"),
           ([(2048, [(30, 1)] * 2), (64, [(5, 1), (1, 1)])], [(7, 1)], [3], "tail, in a group"),
           ([(704, [(20, 20), (45, 9)])], [(3, 3), (9, 9)], [2], "narrow"),
           ([(1024, [(128, 128), (9, 1), (40, 1), (12, 1)])], [(70, 70), (2, 2)], [4, 5], "wide")]


@pytest.mark.parametrize("groups,alone,empty,what", NO_KEYS)
def test_rows_of_requests_without_keys(groups, alone, empty, what):
    """Rows of a request of length 0 (the places of a batch of fixed size that nobody has) see no key: out 0, lse -inf."""
    print_case(f"rows without keys: {what}")
    for hq, hkv, d in ((8, 2, 128), (4, 2, 64)):
        b = shared_batch(groups, hq, hkv, d, 65, alone=alone)
        want = reference(b)
        b["seq"][empty] = 0
        b["bt"][empty] = -1
        out, lse = attend(b)
        for r in range(len(b["reqs"])):
            rows = slice(int(b["cu"][r]), int(b["cu"][r + 1]))
            if r in empty:
                assert (out[rows] == 0).all() and (lse[rows] == -torch.inf).all(), f"{what}: request {r}"
            else:
                sub = dict(b, reqs=[b["reqs"][r]], cu=np.array([0, b["new"][r]]))
                check_out(sub, out[rows], lse[rows], [want[r]], f"{what}: request {r}")


def test_short_tables_take_the_tail_kernel():
    """The case above reaches it: too many (request, head) pairs for one launch, tables of at most 1024 tokens."""
    groups, alone, _, _ = NO_KEYS[1]
    b = shared_batch(groups, 4, 2, 64, 65, alone=alone)
    assert len(b["reqs"]) * 2 > 1024 and b["bt"].shape[1] * 16 <= 1024 and ak.shared_prefix_sizes(bounds_of(b))[1] > 0
