"""What the engine's producer calls refuse of their tensors, before any device work (CPU: the addresses of host tensors
must not reach a kernel)."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests.test_engine_streams import D, HKV, HQ, Tensor, world  # noqa: E402,F401

T, H, N = 5, 32, (HQ + 2 * HKV) * D


def good(to_pool):
    r = dict(x=Tensor(T, H), w_qkv=Tensor(N, H), q=Tensor(T, HQ, D))
    return r if to_pool else dict(r, k_new=Tensor(T, HKV, D), v_new=Tensor(T, HKV, D))


@pytest.mark.parametrize("to_pool", [False, True])
def test_tensors(world, to_pool):
    call = world.eng.project_to_pool if to_pool else world.eng.project
    call(world.db, **good(to_pool), rope_theta=1e4)
    assert [e[:2] for e in world.log] == [("call", "arckv_qkv_rope_to_pool" if to_pool else "arckv_qkv_rope")]
    for name, t in good(to_pool).items():
        host, wide, other = Tensor(*t.shape), Tensor(*t.shape, size=4), Tensor(t.shape[0] + 1, *t.shape[1:])
        host.is_cuda = False
        slices = Tensor(*t.shape)
        slices.is_contiguous = lambda: False
        for bad in (host, wide, other, slices):
            with pytest.raises(ValueError, match="16-bit"):
                call(world.db, **dict(good(to_pool), **{name: bad}), rope_theta=1e4)
    assert len(world.log) == 1
