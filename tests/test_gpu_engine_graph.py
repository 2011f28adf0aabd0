"""The engine's steps captured into graphs that are replayed while the engine goes on: with other batches, a larger
workspace, and another graph at the same time."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.test_gpu_engine_streams import D, DEV, HKV, HQ, batch, busy, engine  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


class Step:
    """A decode step of some requests: store, attend with lse, weigh."""

    def __init__(self, eng, lens, tables, rows, seed):
        self.eng, n = eng, len(rows)
        self.db = eng.upload(batch([lens[r] for r in rows], [1] * n, tables[rows]))
        assert self.db.n_combine > 0
        self.q, self.k, self.v = randn_bf16((n, HQ, D), seed), randn_bf16((n, HKV, D), seed + 1), randn_bf16((n, HKV, D), seed + 2)
        self.out = torch.empty_like(self.q)
        self.lse = torch.empty(n, HQ, device=DEV)
        self.w = torch.zeros(n, HKV, max(lens[r] for r in rows), device=DEV)

    def call(self):
        self.eng.scatter(self.db, self.k, self.v)
        self.eng.attention(self.db, self.q, self.out, lse=self.lse)
        self.eng.attention_weights(self.db, self.q, self.lse, self.w, accumulate=False)

    def results(self):
        return [t.clone() for t in (self.out, self.lse, self.w)]

    def spoil(self):
        self.out.fill_(float("nan"))
        self.lse.fill_(float("nan"))
        self.w.zero_()

    def capture(self):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.call()
        return g


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_graphs_of_steps_replay_beside_the_engines_other_work(fmt):
    print_case(f"graphs of engine steps, {fmt}")
    lens = [3000, 33, 4097, 2000, 9000, 777, 30000, 20000]
    eng, tables = engine(fmt, lens)
    steps = [Step(eng, lens, tables, [0, 1, 2], 10), Step(eng, lens, tables, [3, 4, 5], 20)]
    want = []
    for s in steps:
        s.call()
        torch.cuda.synchronize()
        want.append(s.results())
    small = eng._ws.numel()
    graphs = [s.capture() for s in steps]
    for k in range(3):
        # eager work: more batches than the ring is deep, the later ones with a larger workspace
        for j in range(5):
            Step(eng, lens, tables, [6, 7] if k > 0 else [0, 4], 30 + j).call()
        assert k == 0 or eng._ws.numel() > small
        junk = torch.full((1 << 22,), float("nan"), device=DEV)
        torch.cuda.synchronize()
        for s in steps:
            s.spoil()
        torch.cuda.synchronize()
        sides = [torch.cuda.Stream() for _ in graphs]                  # both at the same time
        for g, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                busy(2)
                g.replay()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert all(torch.equal(a, b) for a, b in zip(s.results(), w)), f"replay {k}"
        del junk
