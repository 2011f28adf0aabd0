"""Outputs of the norm that would overwrite each other, or rows that other work-groups have not read yet, are refused (CPU)."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import _lib  # noqa: E402
from tests.test_step_refusals import A, Tensor, norm  # noqa: E402

X, RES, SUM, OUT, W = (A + k * 0x10000 for k in range(5))


@pytest.mark.parametrize("kw", [
    dict(res=RES, rout=RES, out=RES), dict(res=RES, rout=SUM, out=SUM), dict(res=RES, rout=X, out=X),      # the sum would be lost
    dict(out=X, x_stride=80), dict(res=RES, rout=X, x_stride=80), dict(res=RES, rout=SUM, out=X, x_stride=80),
    dict(out=X, fmt=1, scales=A), dict(res=RES, rout=SUM, out=RES, fmt=1, scales=A), dict(res=RES, rout=SUM, out=SUM, fmt=1, scales=A)])
def test_overlaps_are_refused(kw):
    assert norm(**{**dict(x=X, w=W, out=OUT), **kw}) == _lib.EINVAL
    assert "overlap" in _lib.load().arckv_last_error().decode()


def test_the_binding_says_so(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def at(address, *shape):
        t = Tensor(*shape, index=0)
        t.data_ptr = lambda: address
        return t

    with pytest.raises(ak.ArckvError, match="overlap"):
        ak.add_rms_norm(at(X, 5, 64), at(W, 64), at(RES, 5, 64), 1e-6, residual=at(RES, 5, 64), stream=0)
