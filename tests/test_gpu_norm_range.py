"""The norm of rows whose squares fp32 does not hold: below its smallest and above its largest numbers.  Tolerances of test_gpu_norm:
a power of two scales such a row without rounding it, so the sum's bound stays as it is."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.test_gpu_norm import DEV, _need_gpu, check_bf16, check_e4m3, check_sum, inputs, ref  # noqa: E402, F401

# (factor on a row of ordinary values, eps): squares below the normal numbers, eps of nothing, of the squares' size, far above
# and far below them; squares and their sum beyond the largest number
SCALES = [(2.0 ** e, eps) for e in (-125, -110, -70, -60, -50, -42, -38, -30) for eps in (0.0, 2.0 ** (2 * e) if e > -70 else 0.0, 1e-6, 1e-30)]
SCALES += [(2.0 ** e, eps) for e in (45, 55, 60, 64, 90, 115) for eps in (0.0, 1e-6, 2.0 ** min(2 * e, 126))]


@pytest.mark.parametrize("h", [1, 33, 1000, 4096, 5120, 32768])
@pytest.mark.parametrize("n,with_res", [(3, True), (260, False)])
def test_rows_of_any_size(h, n, with_res):
    n = min(n, (1 << 21) // h)
    x0, res0, w = inputs(n, h, h + n)
    x0[0, 0] = 1                                             # (a row of zeros without eps is 0 / 0)
    wd = w.to(DEV)
    for factor, eps in sorted(set(SCALES)):
        print_case(f"norm {n} x {h}: rows of size {factor:.3g}, eps {eps:.3g}")
        x, res = (x0.double() * factor).to(torch.bfloat16), (res0.double() * factor).to(torch.bfloat16) if with_res else None
        hs, y = ref(x, res, w, eps)
        rows = (hs != 0).any(1)
        assert rows[0]
        xd, rd = x.to(DEV), None if res is None else res.to(DEV)
        rout = None if res is None else torch.empty_like(rd)
        out = torch.full_like(xd, float("nan"))
        ak.add_rms_norm(xd, wd, out, eps, residual=rd, residual_out=rout)
        check_bf16(out.cpu()[rows], y[rows], (n, h))
        if res is not None:
            check_sum(rout, hs)
        codes, scales = torch.full((n, h), 0x7F, dtype=torch.uint8, device=DEV), torch.full((n,), float("nan"), device=DEV)
        ak.add_rms_norm(xd, wd, codes, eps, residual=rd, residual_out=rout, scales=scales)
        if float(y[rows].abs().amax(1).min()) / 448 > 2e-38:          # (below: test_scales_that_are_no_normal_numbers)
            check_e4m3(codes.cpu()[rows], scales.cpu()[rows], y[rows])


def test_a_row_of_other_sizes_beside_it_and_special_values():
    """Large and small values in one row, the largest number, infinities, NaN and zeros."""
    print_case("norm: special rows of any size")
    x = torch.zeros(8, 256, dtype=torch.bfloat16)
    x[0, 0], x[0, 1], x[0, 2] = 3e38, 1.0, 1e-3
    x[1, 5] = 1e-38
    x[2] = 2.0 ** -70
    x[2, 9] = float("nan")
    x[3] = 2.0 ** 70
    x[3, 9] = float("inf")
    x[5] = 2.0 ** -133                                       # the smallest number of bf16
    x[6] = 2.0 ** -133
    x[6, 7] = 2.0 ** -41                                     # the others are 2^-92 of it
    x[7] = 2.0 ** -60
    x[7, 7] = 2.0 ** 55
    w = torch.ones(256, dtype=torch.bfloat16)
    out = torch.empty(8, 256, dtype=torch.bfloat16, device=DEV)
    ak.add_rms_norm(x.to(DEV), w.to(DEV), out, 0.0)
    got, (_, y) = out.cpu(), ref(x, None, w, 0.0)
    for r in (0, 1, 5, 6, 7):
        check_bf16(got[r:r + 1], y[r:r + 1], r)
    assert torch.isnan(got[2]).all() and torch.isnan(got[4]).all()                                  # NaN; 0 / 0
    assert torch.isnan(got[3, 9]) and (got[3, :9] == 0).all() and (got[3, 10:] == 0).all()          # inf / inf, and finite / inf
