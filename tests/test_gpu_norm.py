"""Residual addition and root-mean-square norm, to bf16 and to 8 bits, against the formula in 64 bits.

Tolerances.  A row's squares are added in fp32: at most 40 in a thread, then a tree of 6 lane and 16 wave steps, so the
sum is off by at most 70 * 2^-24 of itself and its root by half of that; the mean, the sum with eps, the root, the quotient and
two products add 6 * 2^-24, h itself 2^-24: y is off by less than 60 * 2^-24 < 4e-6 of itself, SLACK with room for products
of those.  bf16 rounds by at most 2^-8 of the value, E4M3 by 2^-4, or by half of its smallest step, 2^-10 (in units of the scale)."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402

DEV = "cuda:0"
EPS = 1e-6
SLACK = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def inputs(n, h, seed):
    g = torch.Generator().manual_seed(seed)
    gain = 1 + 20 * (torch.rand(h, generator=g) < 0.02)
    x = torch.randn(n, h, generator=g).to(torch.bfloat16)
    res = (torch.randn(n, h, generator=g) * gain).to(torch.bfloat16)
    w = (1 + 0.3 * torch.randn(h, generator=g)).to(torch.bfloat16)
    return x, res, w


def ref(x, res, w, eps=EPS):
    h = x.double() if res is None else x.double() + res.double()
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.double()


def check_bf16(got, want, what):
    err = (got.double().cpu() - want).abs() - (2 ** -8 + SLACK) * want.abs()
    assert torch.isfinite(got).all() and err.max() <= 1e-38, (what, float(err.max()))


def check_sum(got, want):
    """h is exact in fp32 but for one rounding, 2^-24; then bf16."""
    assert ((got.double().cpu() - want).abs() <= (2 ** -8 + 2 ** -23) * want.abs()).all()


def check_e4m3(codes, scales, want):
    s = want.abs().amax(1) / 448
    assert ((scales.double().cpu() - s).abs() <= SLACK * s).all()
    got = codes.view(torch.float8_e4m3fn).double().cpu() * scales.double().cpu()[:, None]
    err = (got - want).abs() - (2 ** -4 + SLACK) * want.abs() - 2 ** -10 * (1 + SLACK) * s[:, None]
    assert err.max() <= 1e-38, float(err.max())


HIDDEN = [1, 7, 8, 33, 64, 512, 520, 1000, 1024, 1032, 2048, 2056, 4095, 4096, 4104, 5120, 5128, 8192, 8200, 16384, 16392, 32767,
          32768]


@pytest.mark.parametrize("h", HIDDEN)
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_every_width(h, fmt):
    for n, with_res in ((1, True), (3, False), (37, True)):
        print_case(f"norm {n} x {h} {fmt} residual {with_res}")
        x, res, w = inputs(n, h, h + n)
        if not with_res:
            res = None
        hs, y = ref(x, res, w)
        xd, wd = x.to(DEV), w.to(DEV)
        rd = None if res is None else res.to(DEV)
        rout = None if res is None else torch.full_like(rd, float("nan"))
        if fmt == "bf16":
            out = torch.full_like(xd, float("nan"))
            ak.add_rms_norm(xd, wd, out, EPS, residual=rd, residual_out=rout)
            check_bf16(out, y, (n, h))
        else:
            out = torch.full((n, h), 0x7F, dtype=torch.uint8, device=DEV)
            scales = torch.full((n,), float("nan"), device=DEV)
            ak.add_rms_norm(xd, wd, out, EPS, residual=rd, residual_out=rout, scales=scales)
            check_e4m3(out, scales, y)
        if res is not None:
            check_sum(rout, hs)
            assert torch.equal(rd.cpu(), res)
        assert torch.equal(xd.cpu(), x)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("h,shift", [(4096, 1), (520, 3), (1000, 4), (333, 1)])
def test_any_address_and_stride(h, shift, fmt):
    """Rows that start at any bf16 address, rows of x that lie apart; what lies between them stays."""
    print_case(f"norm {h} shift {shift} {fmt}")
    n, stride = 19, h + 40 + shift
    x, res, w = inputs(n, h, 5)
    hs, y = ref(x, res, w)

    def shifted(t):
        buf = torch.full((t.numel() + 32,), float("nan"), dtype=t.dtype, device=DEV)
        v = buf[shift:shift + t.numel()].view(t.shape)
        v.copy_(t)
        return buf, v

    wide = torch.full((n * stride + 16,), float("nan"), dtype=torch.bfloat16, device=DEV)
    xd = wide[shift:shift + n * stride].view(n, stride)[:, :h]
    xd.copy_(x)
    before = wide.clone()
    (rbuf, rd), (_, wd) = shifted(res), shifted(w)
    if fmt == "bf16":
        obuf, out = shifted(torch.zeros(n, h, dtype=torch.bfloat16))
        scales = None
    else:
        obuf = torch.full((n * h + 32,), 0x55, dtype=torch.uint8, device=DEV)
        out, scales = obuf[shift:shift + n * h].view(n, h), torch.empty(n, device=DEV)
    ak.add_rms_norm(xd, wd, out, EPS, residual=rd, scales=scales)        # residual_out: in place
    check_sum(rd, hs)
    check_bf16(out, y, h) if fmt == "bf16" else check_e4m3(out.contiguous(), scales, y)
    assert torch.equal(wide.view(torch.int16), before.view(torch.int16))
    assert torch.isnan(rbuf[:shift]).all() and torch.isnan(rbuf[shift + n * h:]).all()
    edge = torch.cat([obuf[:shift], obuf[shift + n * h:]])
    assert (torch.isnan(edge) if fmt == "bf16" else edge == 0x55).all()


def test_in_place_forms():
    print_case("norm in place")
    x, res, w = inputs(50, 1024, 9)
    hs, y = ref(x, res, w)
    wd = w.to(DEV)
    for form in ("out is x", "out is residual", "sum is x"):
        xd, rd = x.to(DEV), res.to(DEV)
        if form == "out is x":
            ak.add_rms_norm(xd, wd, xd, EPS, residual=rd)
            out, total = xd, rd
        elif form == "out is residual":
            total = torch.empty_like(xd)
            ak.add_rms_norm(xd, wd, rd, EPS, residual=rd, residual_out=total)
            out = rd
        else:
            out = torch.empty_like(xd)
            ak.add_rms_norm(xd, wd, out, EPS, residual=rd, residual_out=xd)
            total = xd
        check_bf16(out, y, form)
        check_sum(total, hs)


def test_rows_of_zeros_infinities_and_nan():
    print_case("norm special rows")
    x, _, w = inputs(6, 256, 3)
    x[0] = 0
    x[1, 7] = float("inf")
    x[2, 9] = float("nan")
    x[3] = x[3] * 1e-30                              # eps rules
    out, codes = torch.empty(6, 256, dtype=torch.bfloat16, device=DEV), torch.empty(6, 256, dtype=torch.uint8, device=DEV)
    scales = torch.empty(6, device=DEV)
    ak.add_rms_norm(x.to(DEV), w.to(DEV), out, EPS)
    ak.add_rms_norm(x.to(DEV), w.to(DEV), codes, EPS, scales=scales)
    out, codes, scales = out.cpu(), codes.cpu(), scales.cpu()
    assert (out[0] == 0).all() and (codes[0] & 0x7F == 0).all() and scales[0] == 0
    assert torch.isnan(out[1, 7]) and (out[1, :7] == 0).all()       # inf / inf, and finite / inf
    assert torch.isnan(scales[1]) and (codes[1] & 0x7F == 0x7F).all()
    assert torch.isnan(out[2]).all() and torch.isnan(scales[2]) and (codes[2] & 0x7F == 0x7F).all()
    _, y = ref(x[3:], None, w)
    check_bf16(out[3:], y, "small rows")
    check_e4m3(codes[3:], scales[3:], y)


def test_scales_that_are_no_normal_numbers():
    """Rows so small that max|y| / 448 is below 2^-126 stand for zeros; the next larger ones are kept."""
    print_case("norm tiny scales")
    x = torch.ones(2, 64, dtype=torch.bfloat16)
    w = torch.full((64,), 2.0 ** -118, dtype=torch.bfloat16)      # y = 2^-118, and 2^-118 / 448 < 2^-126
    codes, scales = torch.full((2, 64), 0x55, dtype=torch.uint8, device=DEV), torch.ones(2, device=DEV)
    ak.add_rms_norm(x.to(DEV), w.to(DEV), codes, 0.0, scales=scales)
    assert (codes == 0).all() and (scales == 0).all()
    ak.add_rms_norm(x.to(DEV), (w * 4).to(DEV), codes, 0.0, scales=scales)
    assert (codes == 0x7E).all() and ((scales.double() * 448 - 2.0 ** -116).abs() <= SLACK * 2.0 ** -116).all()     # 448


def test_more_rows_than_a_launch_takes():
    """A launch has 2^21 rows at most."""
    print_case("norm 2^21 + 9 rows")
    n = (1 << 21) + 9
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(n, 16, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.ones(16, dtype=torch.bfloat16, device=DEV)
    out, codes, scales = torch.empty_like(x), torch.empty(n, 16, dtype=torch.uint8, device=DEV), torch.empty(n, device=DEV)
    ak.add_rms_norm(x, w, out, EPS)
    ak.add_rms_norm(x, w, codes, EPS, scales=scales)
    at = torch.cat([torch.arange(64), torch.arange(n - 64, n)])
    _, y = ref(x[at].cpu(), None, w.cpu())
    check_bf16(out[at], y, "many rows")
    check_e4m3(codes[at], scales[at], y)
    ss = out.float().square().mean(1)
    assert bool(((ss - 1).abs() < 0.05).all())       # every row was normed (16 roundings of 2^-8)


def test_many_rows_other_stream_and_graph():
    print_case("norm 70001 rows, stream, graph")
    x, res, w = inputs(70001, 64, 11)
    hs, y = ref(x, res, w)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        xd, rd, wd = x.to(DEV), res.to(DEV), w.to(DEV)
        out, total = torch.empty_like(xd), torch.empty_like(rd)
        ak.add_rms_norm(xd, wd, out, EPS, residual=rd, residual_out=total)
    s.synchronize()
    check_bf16(out, y, "stream")
    check_sum(total, hs)
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ak.add_rms_norm(xd, wd, out, EPS, residual=rd, residual_out=total)
    for _ in range(3):
        out.fill_(float("nan"))
        total.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        check_sum(total, hs)


def test_the_norm_feeds_the_producer():
    """x of the producer is the norm's output: the projection of the normed rows is what the formula gives."""
    print_case("norm into qkv_rope")
    n, h, hq, hkv, d = 33, 256, 4, 2, 64
    x, res, w = inputs(n, h, 21)
    g = torch.Generator().manual_seed(4)
    wq = (torch.randn((hq + 2 * hkv) * d, h, generator=g) / 16).to(torch.bfloat16)
    xd = torch.empty(n, h, dtype=torch.bfloat16, device=DEV)
    ak.add_rms_norm(x.to(DEV), w.to(DEV), xd, EPS, residual=res.to(DEV))
    q, k, v = (torch.empty(n, c, d, dtype=torch.bfloat16, device=DEV) for c in (hq, hkv, hkv))
    cu, sl = torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    ak.qkv_rope(xd, wq.to(DEV), cu, sl, hq, hkv, 1e4, q, k, v, torch.empty(4 * n * d, dtype=torch.uint8, device=DEV))
    want = xd.cpu().double() @ wq.double().T                # values pass through unrotated
    got = v.cpu().double().view(n, -1)
    want = want[:, (hq + hkv) * d:]
    # fp32 sums of 256 products, then bf16
    bound = 2 ** -8 * want.abs() + 256 * 2 ** -24 * (xd.cpu().double().abs() @ wq.double().T.abs())[:, (hq + hkv) * d:] * 1.01
    assert ((got - want).abs() <= bound).all()
    _, y = ref(x, res, w)
    check_bf16(xd, y, "x")
    assert np.isfinite(q.float().cpu().numpy()).all() and np.isfinite(k.float().cpu().numpy()).all()
