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
    """A contiguous device tensor, as far as the checks look; step, row: its strides, if it is not."""

    def __init__(self, *shape, dtype=torch.bfloat16, index=1, step=1, row=None):
        super().__init__(*shape, size=dtype.itemsize, index=index, real=dtype.is_floating_point)
        self.dtype, self.index, self.strides = dtype, index, (row or (shape[-1] if len(shape) > 1 else 1), step)

    def is_contiguous(self):
        return self.strides[1] == 1 and (len(self.shape) != 2 or self.strides[0] == self.shape[1])

    def stride(self, k):
        return self.strides[k]

    def get_device(self):
        return self.index


def i32(*shape, **kw):
    return Tensor(*shape, dtype=torch.int32, **kw)


def f32(*shape, **kw):
    return Tensor(*shape, dtype=torch.float32, **kw)


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
    half, wide, u8 = (Tensor(5, 64, dtype=t) for t in (torch.float16, torch.float32, torch.uint8))
    for kw in (dict(x=Tensor(5)), dict(x=Tensor(5, 64, step=2)), dict(x=Tensor(5, 64, row=60)), dict(x=half), dict(x=wide),
               dict(x=Tensor(5, 64, index=-1)), dict(out=Tensor(5, 63)), dict(out=Tensor(5, 64, row=70)), dict(out=half), dict(out=u8),
               dict(weight=Tensor(63)), dict(weight=Tensor(64, dtype=torch.float16)), dict(residual=Tensor(4, 64)), dict(residual=half),
               dict(residual_out=out), dict(residual=out, residual_out=Tensor(5, 1)), dict(scales=f32(4), out=u8),
               dict(scales=f32(5)), dict(scales=i32(5), out=u8), dict(weight=Tensor(64, index=-1))):
        with pytest.raises(ValueError):
            call(**kw)


def good_maps(index=1):
    kw = dict(new_tokens=(3,), held=(3,), block_tables=(3, 4), free_blocks=(8,), free_count=(1,), cu_q=(4,), seq_lens=(3,),
              slot_mapping=(9,), free_left=(1,))
    return {**{k: i32(*v, index=index) for k, v in kw.items()}, "num_blocks": 100}


def test_maps_binding_refuses():
    for kw in (dict(new_tokens=i32(2)), dict(held=i32(3, 1)), dict(block_tables=i32(12)), dict(block_tables=i32(2, 4)), dict(cu_q=i32(3)),
               dict(seq_lens=i32(4)), dict(free_count=i32(2)), dict(free_left=i32(2)), dict(true_lens=i32(3)), dict(true_offset=i32(3)),
               dict(true_lens=i32(3), true_offset=i32(2)), dict(held=Tensor(3, dtype=torch.int64)), dict(slot_mapping=f32(9)),
               dict(block_tables=i32(3, 4, row=8)), dict(held=i32(3, index=-1))):
        with pytest.raises(ValueError):
            ak.batch_maps(**{**good_maps(), **kw})


BOUNDS = ak.SharedBounds(3, 2, 6, 4, 2, 5, 8, 2, 64, 256)


def good_plan(index=1):
    ints, _ = ak.shared_prefix_sizes(BOUNDS)
    return dict(b=BOUNDS, **{k: i32(*v, index=index) for k, v in dict(group_start=(3,), prefix_lens=(2,), cu_q=(4,), seq_lens=(3,),
                                                                   plan=(ints,)).items()})


def good_attention(index=1):
    ints, ws = ak.shared_prefix_sizes(BOUNDS)
    t = lambda *s, **kw: Tensor(*s, index=index, **kw)  # noqa: E731
    return dict(b=BOUNDS, k_pool=t(9, 2, 16, 64), v_pool=t(9, 2, 64, 16), q=t(6, 8, 64), out=t(6, 8, 64), lse=f32(6, 8, index=index),
                block_tables=i32(3, 5, index=index), cu_q=i32(4, index=index), seq_lens=i32(3, index=index), plan=i32(ints, index=index),
                scale=0.1, workspace=t(ws, dtype=torch.uint8))


def test_shared_prefix_bindings_refuse(monkeypatch):
    ints, ws = ak.shared_prefix_sizes(BOUNDS)
    for kw in (dict(group_start=i32(2)), dict(prefix_lens=i32(3)), dict(cu_q=i32(3)), dict(seq_lens=i32(4)), dict(plan=f32(ints)),
               dict(plan=i32(ints, index=-1)), dict(cu_q=i32(4, index=0))):
        with pytest.raises(ValueError):
            ak.shared_prefix_plan(**{**good_plan(), **kw})
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ak.ArckvError, match="ENOSPC"):
        ak.shared_prefix_plan(**{**good_plan(0), "plan": i32(ints - 1, index=0), "stream": 0})
    for kw in (dict(k_pool=Tensor(9, 2, 16, 128)), dict(v_pool=Tensor(8, 2, 64, 16)), dict(q=Tensor(5, 8, 64)), dict(out=Tensor(6, 8, 32)),
               dict(q=f32(6, 8, 64)), dict(lse=f32(6, 4)), dict(lse=Tensor(6, 8)), dict(block_tables=i32(3, 4)), dict(cu_q=i32(3)),
               dict(seq_lens=i32(2)), dict(plan=i32(ints - 1)), dict(workspace=Tensor(ws - 1, dtype=torch.uint8)),
               dict(workspace=Tensor(ws, dtype=torch.uint8, index=0)), dict(q=Tensor(6, 8, 64, index=-1))):
        with pytest.raises(ValueError):
            ak.shared_prefix_attention(**{**good_attention(), **kw})


def sizes(n=3, g=2, q=6, gq=4, new=2, stride=5, hq=8, hkv=2, d=64, cus=256):
    import ctypes as C
    a, b = _lib.i64(), _lib.i64()
    return _lib.load().arckv_shared_prefix_sizes(n, g, q, gq, new, stride, hq, hkv, d, cus, C.byref(a), C.byref(b))


def test_shared_prefix_calls_refuse():
    E, U, L = _lib.EINVAL, _lib.EUNSUPPORTED, _lib.load()
    assert sizes() == _lib.OK
    for kw in (dict(n=-1), dict(n=(1 << 20) + 1), dict(g=4), dict(g=-1), dict(q=-1), dict(q=(1 << 23) + 1), dict(gq=7), dict(gq=-1), dict(new=7),
               dict(stride=-1), dict(stride=(1 << 26) + 1), dict(hq=9), dict(hq=0), dict(hkv=0), dict(cus=0)):
        assert sizes(**kw) == E, kw
    assert sizes(d=96) == sizes(hq=6) == U
    assert L.arckv_shared_prefix_sizes(3, 2, 6, 4, 2, 5, 8, 2, 64, 256, None, None) == E
    ints, ws = ak.shared_prefix_sizes(BOUNDS)

    def plan(gs=A, pl=A, cu=A, sl=A, p=A, n=ints):
        return L.arckv_shared_prefix_plan(gs, pl, 2, cu, sl, 3, 6, 4, 2, 5, 8, 2, 64, 256, p, n, None)

    for kw in (dict(gs=None), dict(pl=None), dict(cu=None), dict(sl=None), dict(p=None), dict(p=A + 4)):
        assert plan(**kw) == E, kw
    assert plan(n=ints - 1) == _lib.ENOSPC

    def attention(kp=A, vp=A, q=A, out=A, bt=A, cu=A, sl=A, nb=9, scale=0.1, p=A, w=A, n=ws):
        return L.arckv_shared_prefix_attention(kp, vp, q, out, None, bt, 5, cu, sl, 3, 2, 6, 4, 2, nb, 8, 2, 64, 256, scale, p, w, n, None)

    for kw in ({k: None} for k in ("kp", "vp", "q", "out", "bt", "cu", "sl", "p", "w")):
        assert attention(**kw) == E, kw
    for kw in (dict(nb=0), dict(nb=(1 << 27) + 1), dict(scale=0.0), dict(scale=float("nan")), dict(kp=A + 8), dict(vp=A + 8), dict(p=A + 8),
               dict(w=A + 8)):
        assert attention(**kw) == E, kw
    assert attention(n=ws - 1) == _lib.ENOSPC


@pytest.mark.parametrize("device", [0, 1])
def test_calls_run_on_their_tensors_device(device, monkeypatch):
    """On the tensors' device, whichever is the current one; tensors of several are refused."""
    seen = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ak, "_current_stream", lambda index=None: 100 + index)
    real = ak.lib()

    class Guard:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            seen.append(("device", self.index))

        def __exit__(self, *exc):
            return False

    monkeypatch.setattr(torch.cuda, "device", Guard)
    names = ("arckv_add_rms_norm", "arckv_batch_maps", "arckv_shared_prefix_plan", "arckv_shared_prefix_attention")
    fake = SimpleNamespace(arckv_shared_prefix_sizes=real.arckv_shared_prefix_sizes,
                           **{n: (lambda *a, n=n: seen.append((n, a[-1])) or 0) for n in names})
    monkeypatch.setattr(ak, "lib", lambda: fake)
    norm_args = lambda i: dict(x=Tensor(5, 64, index=i), weight=Tensor(64, index=i), out=Tensor(5, 64, index=i), eps=1e-6,  # noqa: E731
                               residual=Tensor(5, 64, index=i))
    calls = [(ak.add_rms_norm, norm_args), (ak.batch_maps, good_maps), (ak.shared_prefix_plan, good_plan),
             (ak.shared_prefix_attention, good_attention)]
    for f, args in calls:
        f(**args(device))
    assert [s for s in seen if s[0] != "device"] == [(n, 100 + device) for n in names]
    assert [s for s in seen if s[0] == "device"] == ([] if device == 0 else [("device", 1)] * 4)
    for f, args in calls:
        other = args(device + 1)
        for name, t in args(device).items():
            if isinstance(t, Tensor):
                with pytest.raises(ValueError):
                    f(**{**args(device), name: other[name]})
    f, args = calls[0]
    f(**args(device), stream=7)
    assert seen[-1] == (names[0], 7)
