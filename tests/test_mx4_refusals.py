"""What the 4-bit cache's and eviction's calls refuse, before any device work (CPU: the addresses given are
never read)."""

from __future__ import annotations

import pytest

import paper_2606_21238_amd as ak
from paper_2606_21238_amd import _lib

A, M = 0x10000, 0x10008        # an aligned and a misaligned address


def code(status, word=""):
    assert status != _lib.OK and word.encode() in ak.lib().arckv_last_error(), ak.lib().arckv_last_error()
    return _lib.STATUS_NAMES[status]


def test_pool_bytes():
    assert ak.mx4_pool_bytes(10, 8, 128) == 10 * 8 * 17 * 128
    assert ak.mx4_pool_bytes(3, 1, 64) == 3 * 17 * 64
    assert [ak.mx4_pool_bytes(*a) for a in ((-1, 8, 128), (1, 0, 128), (1, 8, 96))] == [-1] * 3


@pytest.mark.parametrize("name", ["arckv_kv_scatter_mx4", "arckv_kv_gather_mx4"])
def test_rows(name):
    f = getattr(ak.lib(), name)

    def call(pool=A, k=A, v=A, slots=A, n=4, nb=4, hkv=2, d=64):
        return f(pool, k, v, slots, n, nb, hkv, d, None)

    assert code(call(d=96), "head_dim") == "EUNSUPPORTED"
    for kw in (dict(n=-1), dict(nb=-1), dict(nb=(1 << 27) + 1), dict(hkv=0), dict(hkv=70000), dict(n=1 << 31)):
        assert code(call(**kw), "sizes") == "EINVAL"
    for kw in (dict(pool=None), dict(k=None), dict(v=None), dict(slots=None)):
        assert code(call(**kw), "NULL") == "EINVAL"
    for kw in (dict(pool=M), dict(k=M), dict(v=M)):
        assert code(call(**kw), "aligned") == "EINVAL"
    assert call(n=0, pool=None) == _lib.OK


def test_attention():
    def call(pool=A, q=A, out=A, lse=None, bt=A, cu=A, seq=A, n=1, n_q=1, nb=4, work=A, n_work=8, n_combine=0,
             cols=128, hq=8, hkv=4, d=128, scale=0.1, ws=None, ws_bytes=0, stride=1):
        return ak.lib().arckv_prefill_attention_mx4(pool, q, out, lse, bt, stride, cu, seq, n, n_q, nb, work, n_work,
                                                    n_combine, cols, hq, hkv, d, scale, ws, ws_bytes, None)

    assert code(call(d=96), "head_dim") == "EUNSUPPORTED"
    assert code(call(hq=12), "group") == "EUNSUPPORTED"
    for kw in (dict(n=-1), dict(hq=7), dict(scale=0.0), dict(scale=float("nan")), dict(n_work=-8), dict(ws_bytes=-1)):
        assert code(call(**kw), "sizes") == "EINVAL"
    assert code(call(cols=200), "tile_cols") == "EINVAL"
    assert code(call(n_work=7), "lists") == "EINVAL"
    assert code(call(nb=(1 << 27) + 1), "num_blocks") == "EINVAL"
    for kw in (dict(pool=None), dict(q=None), dict(out=None), dict(bt=None), dict(cu=None), dict(seq=None), dict(work=None)):
        assert code(call(**kw), "NULL") == "EINVAL"
    assert code(call(pool=M), "aligned") == "EINVAL"
    assert code(call(ws=M, ws_bytes=1 << 20), "aligned") == "EINVAL"
    assert code(call(n_combine=1), "workspace") == "EINVAL"
    assert call(n_work=0, pool=None) == _lib.OK and call(n_q=0, pool=None) == _lib.OK


def test_lse_of_the_bf16_attention():
    a = (A, A, A, A, None, A, 1, A, A, 1, 1, 4, A, 8, 0, 128, 8, 4, 128, 0.1, None, 0, None)
    assert code(ak.lib().arckv_prefill_attention_lse(*a), "NULL lse") == "EINVAL"


def test_weights():
    def call(pool=A, layout=2, q=A, lse=A, bt=A, stride=4, cu=A, seq=A, n=1, n_q=1, nb=4, hq=8, hkv=4, d=128,
             scale=0.1, w=A, ws=64):
        return ak.lib().arckv_attention_weights(pool, layout, q, lse, bt, stride, cu, seq, n, n_q, nb, hq, hkv, d, scale,
                                                w, ws, 1, None)

    assert code(call(layout=3), "layout") == "EINVAL"
    assert code(call(d=32), "head_dim") == "EUNSUPPORTED"
    assert code(call(hq=12), "group") == "EUNSUPPORTED"
    for kw in (dict(n=-1), dict(scale=float("inf")), dict(ws=-1), dict(n=70000), dict(nb=(1 << 27) + 1)):
        assert code(call(**kw), "sizes") == "EINVAL"
    assert code(call(nb=0), "num_blocks") == "EINVAL"
    for kw in (dict(pool=None), dict(q=None), dict(lse=None), dict(bt=None), dict(cu=None), dict(seq=None), dict(w=None)):
        assert code(call(**kw), "NULL") == "EINVAL"
    assert code(call(pool=M, layout=1), "aligned") == "EINVAL"
    assert call(n=0, pool=None) == _lib.OK and call(ws=0, w=None) == _lib.OK


def test_select():
    def call(w=A, stride=64, seq=A, n=1, hkv=2, keep=16, first=0, recent=0, kept=A, kw=None, kws=0):
        return ak.lib().arckv_evict_select(w, stride, seq, n, hkv, keep, first, recent, kept, kw, kws, None)

    for kw in (dict(n=-1), dict(n=70000), dict(hkv=0), dict(keep=-1), dict(first=-1), dict(recent=-1),
               dict(first=10, recent=7), dict(first=(1 << 31) - 1, recent=(1 << 31) - 1), dict(stride=-1)):
        assert code(call(**kw), "sizes") == "EINVAL"
    assert code(call(kw=A, kws=15), "kw_stride") == "EINVAL"
    for kw in (dict(w=None), dict(seq=None), dict(kept=None)):
        assert code(call(**kw), "NULL") == "EINVAL"
    assert call(n=0, w=None) == _lib.OK and call(keep=0, w=None) == _lib.OK


@pytest.mark.parametrize("mx4", [False, True])
def test_compact(mx4):
    def call(pool=A, v=A, bt=A, stride=4, kept=A, keep=16, dst=A, ds=1, n=1, nb=4, hkv=2, d=128):
        tail = (bt, stride, kept, keep, dst, ds, n, nb, hkv, d, None)
        return ak.lib().arckv_kv_compact_mx4(pool, *tail) if mx4 else ak.lib().arckv_kv_compact(pool, v, *tail)

    assert code(call(d=256), "head_dim") == "EUNSUPPORTED"
    for kw in (dict(n=-1), dict(n=70000), dict(keep=-1), dict(keep=17), dict(ds=0), dict(hkv=0), dict(nb=(1 << 27) + 1),
               dict(stride=-1)):
        assert code(call(**kw), "sizes") == "EINVAL"
    for kw in (dict(pool=None), dict(bt=None), dict(kept=None), dict(dst=None)):
        assert code(call(**kw), "NULL") == "EINVAL"
    assert code(call(pool=M), "aligned") == "EINVAL"
    assert call(n=0, pool=None) == _lib.OK and call(keep=0, pool=None) == _lib.OK
