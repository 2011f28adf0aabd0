"""What the calls of a device-side step refuse, before any device work (CPU)."""

from __future__ import annotations

from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import _lib  # noqa: E402
from tests.test_binding_device import Tensor as _Tensor  # noqa: E402

A, M = 0x20000, 0x20001          # an aligned and a misaligned address, never read


class Tensor(_Tensor):
    dtype = "torch.bfloat16"

    def stride(self, k):
        return getattr(self, "row", self.shape[1]) if k == 0 else getattr(self, "step", 1)


def norm(x=A, x_stride=64, res=None, rout=None, w=A, n=4, h=64, eps=1e-6, out=A, fmt=0, scales=None):
    return _lib.load().arckv_add_rms_norm(x, x_stride, res, rout, w, n, h, eps, out, fmt, scales, None)


def test_norm_refuses():
    E, U = _lib.EINVAL, _lib.EUNSUPPORTED
    assert norm(n=-1) == norm(n=1 << 31) == norm(h=0) == norm(x_stride=63) == norm(eps=-1.0) == norm(eps=float("nan")) == E
    assert norm(fmt=2) == norm(fmt=1) == E                       # no such format; no scales
    assert norm(h=32769, x_stride=70000) == U
    assert norm(res=A) == norm(rout=A) == E
    assert norm(x=None) == norm(w=None) == norm(out=None) == E
    assert norm(x=M) == norm(w=M) == norm(out=M) == norm(res=M, rout=A) == norm(res=A, rout=M) == E
    assert norm(fmt=1, scales=A + 2) == E
    assert norm(x=None, w=None, out=None, n=0) == _lib.OK        # nothing to do


def maps(new=A, held=A, n=3, bt=A, stride=4, free=A, cap=8, count=A, left=A, cu=A, sl=A, off=None, true=None, sm=A, slots=9, nb=100):
    return _lib.load().arckv_batch_maps(new, held, n, bt, stride, free, cap, count, left, cu, sl, off, true, sm, slots, nb, None)


def test_maps_refuse():
    bad = [dict(n=-1), dict(n=(1 << 24) + 1), dict(stride=-1), dict(cap=-1), dict(cap=1 << 31), dict(slots=-1), dict(slots=(1 << 30) + 1),
           dict(nb=0), dict(nb=(1 << 27) + 1), dict(true=A)]
    bad += [{k: None} for k in ("new", "held", "bt", "free", "count", "left", "cu", "sl", "sm")]
    for kw in bad:
        assert maps(**kw) == _lib.EINVAL, kw


def test_norm_binding_refuses():
    x, w, out = Tensor(5, 64), Tensor(64), Tensor(5, 64)
    call = lambda **kw: ak.add_rms_norm(**{**dict(x=x, weight=w, out=out, eps=1e-6), **kw})  # noqa: E731
    gap = Tensor(5, 64)
    gap.step = 2
    over = Tensor(5, 64)
    over.row = 60
    half = Tensor(5, 64)
    half.dtype = "torch.float16"
    wide = Tensor(5, 64, size=4)
    for kw in (dict(x=Tensor(5)), dict(x=gap), dict(x=over), dict(x=half), dict(x=wide), dict(out=Tensor(5, 63)), dict(weight=Tensor(63)),
               dict(residual=Tensor(4, 64)), dict(residual_out=out), dict(residual=out, residual_out=Tensor(5, 1)),
               dict(scales=Tensor(4, size=4, real=True)), dict(scales=Tensor(5, size=4, real=True)),       # (a 16-bit out)
               dict(scales=Tensor(5, size=4), out=Tensor(5, 64, size=1)), dict(out=Tensor(5, 64, size=1)),
               dict(weight=half), dict(x=SimpleNamespace(dim=lambda: 3))):
        with pytest.raises(ValueError):
            call(**kw)


def test_maps_binding_refuses():
    def i32(*s):
        return Tensor(*s, size=4)

    good = dict(new_tokens=i32(3), held=i32(3), block_tables=i32(3, 4), free_blocks=i32(8), free_count=i32(1), cu_q=i32(4),
                seq_lens=i32(3), slot_mapping=i32(9), free_left=i32(1), num_blocks=100)
    for kw in (dict(new_tokens=i32(2)), dict(block_tables=i32(12)), dict(block_tables=i32(2, 4)), dict(cu_q=i32(3)), dict(seq_lens=i32(4)),
               dict(free_count=i32(2)), dict(free_left=i32(2)), dict(true_lens=i32(3)), dict(true_offset=i32(3)),
               dict(true_lens=i32(3), true_offset=i32(2)), dict(held=Tensor(3, size=8)), dict(slot_mapping=Tensor(9, size=4, real=True))):
        with pytest.raises(ValueError):
            ak.batch_maps(**{**good, **kw})


@pytest.mark.parametrize("device", [0, 1])
def test_calls_run_on_their_tensors_device(device, monkeypatch):
    """On the tensors' device, whichever is the current one; tensors of several are refused."""
    from tests.test_binding_device import i32
    seen = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ak, "_current_stream", lambda index=None: 100 + index)

    class Guard:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            seen.append(("device", self.index))

        def __exit__(self, *exc):
            return False

    monkeypatch.setattr(torch.cuda, "device", Guard)
    fake = SimpleNamespace(arckv_add_rms_norm=lambda *a: seen.append(("norm", a[-1].value)) or 0,
                           arckv_batch_maps=lambda *a: seen.append(("maps", a[-1].value)) or 0)
    monkeypatch.setattr(ak, "lib", lambda: fake)

    def on(t, index=device):
        t.device = SimpleNamespace(index=index)
        t.dtype = "torch.int32"
        return t

    def t16(*s, index=device):
        return on(Tensor(*s), index)

    ak.add_rms_norm(t16(5, 64), t16(64), t16(5, 64), 1e-6)
    ints = dict(new_tokens=i32(3), held=i32(3), block_tables=i32(3, 4), free_blocks=i32(8), free_count=i32(1), cu_q=i32(4),
                seq_lens=i32(3), slot_mapping=i32(9), free_left=i32(1))
    ak.batch_maps(**{k: on(v) for k, v in ints.items()}, num_blocks=100)
    assert [s for s in seen if s[0] != "device"] == [("norm", 100 + device), ("maps", 100 + device)]
    assert [s for s in seen if s[0] == "device"] == ([] if device == 0 else [("device", 1)] * 2)
    with pytest.raises(ValueError, match="one device"):
        ak.add_rms_norm(t16(5, 64), t16(64, index=device + 1), t16(5, 64), 1e-6)
    with pytest.raises(ValueError, match="one device"):
        ak.batch_maps(**{k: on(v, device + (k == "free_left")) for k, v in ints.items()}, num_blocks=100)
