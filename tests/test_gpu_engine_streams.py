"""One engine whose batches run on several streams: the split plans' workspace, the metadata ring and the pools
are shared, so results must be those of the same calls on one stream."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import BatchPlan  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402

DEV = "cuda"
HQ, HKV, D = 32, 8, 128


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def busy(n=6):
    x = torch.randn(4096, 4096, device=DEV)
    for _ in range(n):
        x = x @ x * 1e-4


def engine(fmt, lens):
    """An engine whose pools hold random tokens for requests of these lengths, and the requests' block tables."""
    nb = [-(-L // 16) for L in lens]
    eng = PrefillEngine(HQ, HKV, D, 8, 16, 4, kv_format=fmt, private_blocks=sum(nb), pool_fill=0)
    at = np.cumsum([0] + nb) + eng.num_phys
    tables = np.full((len(lens), max(nb)), -1, dtype=np.int32)
    for r, n in enumerate(nb):
        tables[r, :n] = np.random.default_rng(1).permutation(np.arange(at[r], at[r + 1]))
    slots = np.concatenate([tables[r, np.arange(L) // 16] * 16 + np.arange(L) % 16 for r, L in enumerate(lens)])
    db = eng.upload(batch(lens, lens, tables, slots))
    eng.scatter(db, randn_bf16((sum(lens), HKV, D), 1), randn_bf16((sum(lens), HKV, D), 2))
    return eng, tables


def batch(lens, new, tables, slots=None):
    """A plan by hand: the last `new` tokens of requests that are in the pool."""
    lens, new = np.array(lens, np.int32), np.array(new, np.int32)
    if slots is None:
        slots = np.concatenate([tables[r, np.arange(L - s, L) // 16] * 16 + np.arange(L - s, L) % 16
                                for r, (L, s) in enumerate(zip(lens, new))])
    return BatchPlan(tables, np.concatenate([[0], np.cumsum(new)]).astype(np.int32), lens, lens - new,
                     ((lens - new) // 16).astype(np.int32), slots.astype(np.int32), int(new.max()), int(lens.max()))


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_two_split_batches_on_two_streams(fmt):
    print_case(f"two decode batches of one engine on two streams, {fmt}")
    lens = [6000, 33, 4097, 2000, 9000, 777]
    eng, tables = engine(fmt, lens)
    rows = [[0, 1, 2], [3, 4, 5]]
    qs = [randn_bf16((3, HQ, D), 5 + k) for k in range(2)]

    def run(streams, rounds, raw=False):
        """Both batches `rounds` times in turn, the second one's longer for more rounds than the ring is deep."""
        res = []
        for k in range(rounds):
            for x, st in enumerate(streams):
                given = st.cuda_stream if raw else st
                db = eng.upload(batch([lens[r] - k for r in rows[x]], [1] * 3, tables[rows[x]]), stream=given)
                assert db.n_combine > 0 and db.ws_bytes > 0
                out, lse = torch.full_like(qs[x], float("nan")), torch.full((3, HQ), float("nan"), device=DEV)
                if st is not None:
                    st.wait_stream(torch.cuda.current_stream())        # `out` and `lse` are filled
                    with torch.cuda.stream(st):
                        busy(1 + k % 2)
                eng.attention(db, qs[x], out, stream=given, lse=lse)
                res += [out, lse]
        torch.cuda.synchronize()
        return res

    want = run([None, None], 7)
    two = [torch.cuda.Stream(), torch.cuda.Stream()]
    for streams, raw in ((two, False), ([None, torch.cuda.Stream()], False), (two, True)):
        got = run(streams, 7, raw)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_an_engine_is_used_on_another_stream_than_it_was_made_on(fmt):
    """The pools are filled on the stream that is current when the engine is made, behind long work here."""
    print_case(f"an engine made on a busy stream, {fmt}")
    side = torch.cuda.Stream()
    k, v, q = randn_bf16((40, HKV, D), 1), randn_bf16((40, HKV, D), 2), randn_bf16((40, HQ, D), 3)
    toks = [np.arange(40, dtype=np.int32)]
    res = []
    for st in (None, side):
        torch.cuda.synchronize()
        busy()
        eng = PrefillEngine(HQ, HKV, D, 8, 16, 4, kv_format=fmt)
        db = eng.prepare(toks, stream=st)
        eng.scatter(db, k, v, stream=st)
        with torch.cuda.stream(st or torch.cuda.current_stream()):
            out = torch.empty_like(q)
        eng.attention(db, q, out, stream=st)
        torch.cuda.synchronize()
        eng.release()
        res.append([out] + [p.clone() for p in (eng.k_pool, eng.v_pool, eng.kv_pool) if p is not None])
    assert all(torch.equal(a, b) for a, b in zip(*res))
