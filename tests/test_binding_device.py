"""Every device call of the binding runs on its tensors' device, whichever is torch's current one, on that device's
current stream, and refuses tensors of several devices (CPU: devices, streams and the library are stand-ins)."""

from __future__ import annotations

from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2606_21238_amd as ak  # noqa: E402

T, HQ, HKV, D, NB = 5, 4, 2, 64, 3


class Tensor:
    is_cuda = True

    def __init__(self, *shape, size=2, index=1, real=False):
        self.shape, self.size, self.real = shape, size, real
        self.device = SimpleNamespace(index=index)

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.size

    def is_floating_point(self):
        return self.real

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def data_ptr(self):
        return 0x1000


def i32(*shape):
    return Tensor(*shape, size=4)


def f32(*shape):
    return Tensor(*shape, size=4, real=True)


def calls():
    """(name of the library's call, the binding's function, its tensors, its other arguments)."""
    kp, vp, mx = Tensor(NB, HKV, 16, D), Tensor(NB, HKV, D, 16), Tensor(NB, HKV, 17 * D, size=1)
    rows, q, slots, bt, cu, sl, work = Tensor(T, HKV, D), Tensor(T, HQ, D), i32(T), i32(1, NB), i32(2), i32(1), i32(8, 8)
    ws, x, w, lse, wts, kept = Tensor(1 << 14, size=1), Tensor(T, 32), Tensor((HQ + 2 * HKV) * D, 32), f32(T, HQ), f32(1, HKV, 9), i32(1, HKV, 4)
    batch = dict(q=q, out=Tensor(T, HQ, D), block_tables=bt, cu_q=cu, seq_lens=sl, work=work)
    plan = dict(n_work=8, n_combine=0, tile_cols=128, scale=0.1)
    pools = dict(k_pool=kp, v_pool=vp)
    rope = dict(x=x, w_qkv=w, cu_q=cu, seq_lens=sl, q_out=Tensor(T, HQ, D), workspace=ws)
    heads = dict(num_q_heads=HQ, num_kv_heads=HKV, rope_theta=1e4)
    move = dict(block_tables=bt, kept=kept, dst_tables=i32(1, 1))
    return [
        ("kv_scatter", ak.kv_scatter, dict(pools, k_new=rows, v_new=rows, slot_mapping=slots), {}),
        ("kv_scatter_mx4", ak.kv_scatter_mx4, dict(kv_pool=mx, k_new=rows, v_new=rows, slot_mapping=slots), {}),
        ("kv_gather_mx4", ak.kv_gather_mx4, dict(kv_pool=mx, k_out=rows, v_out=rows, slot_mapping=slots), {}),
        ("qkv_rope", ak.qkv_rope, dict(rope, k_out=rows, v_out=rows), heads),
        ("qkv_rope_to_pool", ak.qkv_rope_to_pool, dict(rope, **pools, slot_mapping=slots), heads),
        ("prefill_attention", ak.prefill_attention, dict(pools, **batch, workspace=ws), plan),
        ("prefill_attention_lse", ak.prefill_attention, dict(pools, **batch, workspace=ws, lse=lse), plan),
        ("prefill_attention_mx4", ak.prefill_attention_mx4, dict(kv_pool=mx, **batch, workspace=ws, lse=lse), plan),
        ("prefill_attention_noalloc", ak.prefill_attention_noalloc, dict(pools, **batch), dict(plan, ws_bytes=0)),
        ("attention_weights", ak.attention_weights,
         dict(k_pool=kp, q=q, lse=lse, weights=wts, block_tables=bt, cu_q=cu, seq_lens=sl), dict(scale=0.1)),
        ("evict_select", ak.evict_select, dict(weights=wts, seq_lens=sl, kept=kept, kept_weights=f32(1, HKV, 4)), {}),
        ("kv_compact", ak.kv_compact, dict(pools, **move), {}),
        ("kv_compact_mx4", ak.kv_compact_mx4, dict(kv_pool=mx, **move), {}),
    ]


@pytest.fixture
def on(monkeypatch):
    """The library's calls as (name, current device, stream); torch's current device is 0, device k's stream 100 k + 7."""
    got, now = [], [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            now.append(self.index)

        def __exit__(self, *exc):
            now.pop()

    class Lib:
        def __getattr__(self, name):
            return lambda *args: got.append((name, now[-1], args[-1].value)) or 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(ak, "_current_stream", lambda index=None: 100 * (now[-1] if index is None else index) + 7)
    monkeypatch.setattr(ak, "lib", lambda: Lib())
    return got


@pytest.mark.parametrize("name", [c[0] for c in calls()])
def test_device_and_stream(on, name):
    _, f, tensors, more = next(c for c in calls() if c[0] == name)
    f(**tensors, **more)
    f(**tensors, **more, stream=55)
    assert on == [(f"arckv_{name}", 1, 107), (f"arckv_{name}", 1, 55)]
    for key, t in tensors.items():
        t.device = SimpleNamespace(index=0)
        if any(x.device.index == 1 for x in tensors.values()):
            with pytest.raises(ValueError, match="one device"):
                f(**tensors, **more)
    on.clear()
    f(**tensors, **more)
    assert on == [(f"arckv_{name}", 0, 7)]
