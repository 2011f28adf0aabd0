"""The device-checked build on the slots of a step that is not full: -1 names no slot and is recorded nowhere, others outside the
pool are."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import _lib  # noqa: E402
from tests.gpu_helpers import bits, print_case  # noqa: E402
from tests.mx4_helpers import DEV, i32  # noqa: E402
from tests.test_gpu_checks import checked  # noqa: E402, F401
from tests.test_gpu_parity import randn_bf16  # noqa: E402


@pytest.mark.parametrize("n,live", [(40, 7), (1500, 900)])
@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_slots_of_minus_one(checked, fmt, n, live):  # noqa: F811
    print_case(f"checked build: scatter of {live} of {n} rows, {fmt}")
    hkv, d, nb = 2, 64, 120
    slots = np.full(n, -1, np.int32)
    slots[:live] = np.random.default_rng(n).permutation(16 * nb)[:live]
    k, v = randn_bf16((n, hkv, d), 1), randn_bf16((n, hkv, d), 2)

    def scatter(rows, at):
        if fmt == "bf16":
            pool = torch.full((nb, hkv, 16, d), -1, dtype=torch.int16, device=DEV), torch.full((nb, hkv, d, 16), -1, dtype=torch.int16, device=DEV)
            ak.kv_scatter(*pool, k[:rows], v[:rows], i32(at))
        else:
            pool = (torch.full((nb, hkv, 17 * d), 0xFF, dtype=torch.uint8, device=DEV),)
            ak.kv_scatter_mx4(*pool, k[:rows], v[:rows], i32(at))
        torch.cuda.synchronize()
        return pool

    ak.device_checks(reset=True)
    got, want = scatter(n, slots), scatter(live, slots[:live])
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert ak.device_checks() == (0, 0)
    for bad in (-2, 16 * nb, 1 << 30):
        other = slots.copy()
        other[live + 3] = bad
        again = scatter(n, other)
        assert all(torch.equal(x, y) for x, y in zip(again, want))
        kind, count = ak.device_checks()
        assert kind == _lib.CHECK_SLOT and count >= 1
    if fmt == "bf16":
        assert (bits(got[0]) != 0xFFFF).any()
