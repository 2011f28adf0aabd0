"""A decode loop that stays on the device, as a serving program runs it: maps and plan, norm, producer into the pools and attention over
shared prefixes, in whole steps captured into a graph and replayed while the requests grow.  Beside it the same steps
planned on the host: the pools' bytes are the same, the attention is right against 64 bits."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import BatchPlan  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import DEV, check_out, i32, reference  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402

HIDDEN, THETA, EPS = 256, 1e4, 1e-6


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


class Loop:
    """Requests in groups [(shared tokens, [own tokens])], on an engine of its own."""

    def __init__(self, groups, hq=8, hkv=2, d=64, max_tokens=16, spare=40, true_shift=None, seed=3, max_new=None):
        self.hq, self.hkv, self.d, self.T = hq, hkv, d, max_tokens
        rng = np.random.default_rng(seed)
        self.held = np.array([p + o for p, os in groups for o in os])
        n = len(self.held)
        private = sum(p // 16 for p, _ in groups) + sum(-(-o // 16) for _, os in groups for o in os) + spare
        self.eng = PrefillEngine(hq, hkv, d, 8, 16, 4, private_blocks=private, pool_fill=-1)
        ids = self.eng.num_phys + rng.permutation(private)
        self.tables = np.full((n, int(max(self.held)) // 16 + 12), -1, np.int32)
        r, at = 0, 0
        for p, os in groups:
            pre, at = ids[at:at + p // 16], at + p // 16
            for o in os:
                k = -(-o // 16)
                self.tables[r, :p // 16], self.tables[r, p // 16:p // 16 + k] = pre, ids[at:at + k]
                r, at = r + 1, at + k
        self.free = ids[at:].astype(np.int32)
        slots = [self.tables[r, np.arange(L) // 16] * 16 + np.arange(L) % 16 for r, L in enumerate(self.held)]
        slots = np.unique(np.concatenate(slots))
        ak.kv_scatter(self.eng.k_pool, self.eng.v_pool, randn_bf16((len(slots), hkv, d), seed), randn_bf16((len(slots), hkv, d), seed + 1),
                      i32(slots))
        self.true = None if true_shift is None else self.held + np.array(true_shift)
        self.sb = self.eng.step_batch(self.tables, self.held, [len(os) for _, os in groups], [p for p, _ in groups], max_tokens,
                                      max_new=max_new, free_blocks=self.free, true_lens=self.true)
        self.w_norm = (1 + 0.1 * randn_bf16((HIDDEN,), seed + 2)).to(torch.bfloat16)
        self.w_qkv = (randn_bf16(((hq + 2 * hkv) * d, HIDDEN), seed + 4) / 16).to(torch.bfloat16)
        e = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        self.new = torch.zeros(n, dtype=torch.int32, device=DEV)
        self.delta, self.res, self.x = e(max_tokens, HIDDEN), e(max_tokens, HIDDEN), e(max_tokens, HIDDEN)
        self.q, self.out = e(max_tokens, hq, d), e(max_tokens, hq, d)
        self.lse = torch.zeros(max_tokens, hq, device=DEV)

    def step(self, stream=None):
        self.eng.advance(self.sb, self.new, stream=stream)
        raw = None if stream is None else stream if isinstance(stream, int) else stream.cuda_stream
        ak.add_rms_norm(self.delta, self.w_norm, self.x, EPS, residual=self.res, stream=raw)
        self.eng.project_to_pool(self.sb, self.x, self.w_qkv, self.q, THETA, stream=stream)
        self.eng.shared_attention(self.sb, self.q, self.out, lse=self.lse, stream=stream)

    def give(self, new, seed):
        self.new.copy_(i32(new))
        self.delta.copy_(randn_bf16((self.T, HIDDEN), seed))
        self.res.copy_(randn_bf16((self.T, HIDDEN), seed + 1))
        self.out.fill_(float("nan"))
        self.lse.fill_(float("nan"))

    def check(self, new, twin, what):
        """The step just made, which gave `new` (after refusals): the maps, the pools' bytes (against the same step planned on the
        host, in the pools of `twin`), and the attention in 64 bits."""
        torch.cuda.synchronize()
        held = self.held
        self.held = held + new
        cu = np.concatenate([[0], np.cumsum(new)])
        sb, n = self.sb, len(held)
        assert np.array_equal(sb.seq_lens.cpu().numpy(), self.held) and np.array_equal(sb.cu_q.cpu().numpy(), cu), what
        self.tables = sb.block_tables.cpu().numpy()
        slots = np.concatenate([self.tables[r, np.arange(h, h + s) // 16] * 16 + np.arange(h, h + s) % 16
                                for r, (h, s) in enumerate(zip(held, new))] + [np.full(self.T - cu[-1], -1)])
        assert np.array_equal(sb.slot_mapping.cpu().numpy(), slots), what
        if self.true is not None:
            self.true = self.true + new
            assert np.array_equal(sb.true_lens.cpu().numpy(), self.true)
        lens = self.held if self.true is None else self.true
        ws = torch.empty(4 * self.T * self.d, dtype=torch.uint8, device=DEV)
        q = torch.empty_like(self.q)
        ak.qkv_rope_to_pool(self.x, self.w_qkv, i32(cu), i32(lens), self.hq, self.hkv, THETA, q, *twin, i32(slots), ws)
        assert torch.equal(twin[0], self.eng.k_pool) and torch.equal(twin[1], self.eng.v_pool), what
        t = int(cu[-1])
        assert torch.equal(q[:t], self.q[:t]), what
        rows = [self.tables[r, np.arange(L) // 16].astype(np.int64) * 16 + np.arange(L) % 16 for r, L in enumerate(self.held)]
        kr = self.eng.k_pool.view(torch.bfloat16).permute(0, 2, 1, 3).reshape(-1, self.hkv, self.d)
        vr = self.eng.v_pool.view(torch.bfloat16).permute(0, 3, 1, 2).reshape(-1, self.hkv, self.d)
        b = dict(hq=self.hq, hkv=self.hkv, d=self.d, scale=self.d ** -0.5, q=self.q[:t], cu=cu, reqs=[(int(L), int(L - s)) for L, s in zip(self.held, new)],
                 k=[kr[torch.from_numpy(x).to(DEV)].double() for x in rows], v=[vr[torch.from_numpy(x).to(DEV)].double() for x in rows])
        check_out(b, self.out[:t], self.lse[:t], reference(b), what)
        assert torch.isnan(self.out[t:]).all() and torch.isnan(self.lse[t:]).all(), what

    def twin(self):
        return self.eng.k_pool.clone(), self.eng.v_pool.clone()


GROUPS = [(256, [40, 0, 17]), (64, [5]), (1024, [300, 1, 33, 48])]


@pytest.mark.parametrize("true", [None, [0, 500, 3, 0, 9, 0, 0, 7]])
def test_eager_and_replayed_steps(true):
    print_case(f"decode loop, true lengths {true}")
    loop = Loop(GROUPS, true_shift=true)
    n = len(loop.held)
    rng = np.random.default_rng(1)
    twin = loop.twin()
    loop.give(np.ones(n), 50)
    loop.step()
    loop.check(np.ones(n, int), twin, "first step")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.step()
    for k in range(8):
        new = rng.integers(0, 4, n)
        new[rng.random(n) < 0.2] = -1                    # an ended request
        if k == 4:
            new[:] = 0                                   # a step of nobody
        loop.give(new, 60 + 2 * k)
        if k % 3 == 2:
            loop.step()                                  # the engine's own call between replays
        else:
            graph.replay()
        new = new.clip(0)
        fits = np.cumsum(new) <= loop.T                  # the rows last that far
        loop.check(new * fits, twin, f"step {k}")


def test_steps_until_the_blocks_are_gone():
    """The first requests take the last blocks; then those go on that have room in their own."""
    print_case("decode loop, blocks run out")
    loop = Loop([(128, [15, 16, 31])], spare=2, max_tokens=4)
    twin = loop.twin()
    left = 2
    for k in range(20):
        loop.give([1, 1, 1], 200 + 2 * k)
        loop.step()
        need = [int(h % 16 == 0) for h in loop.held]
        give = [int(not b or sum(need[:r + 1]) <= left) for r, b in enumerate(need)]
        left -= sum(b * g for b, g in zip(need, give))
        loop.check(np.array(give), twin, f"step {k}")
        assert int(loop.sb.free_count.cpu()) == left
    assert left == 0 and 0 in give


@pytest.mark.parametrize("raw", [False, True])
def test_steps_on_several_streams(raw):
    """Calls on different streams run in the order of the calls."""
    print_case(f"decode loop on streams, raw {raw}")
    loop = Loop([(512, [100, 20]), (48, [7])])
    twin = loop.twin()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(6):
        loop.give([1, 2, 1], 300 + 2 * k)
        torch.cuda.synchronize()
        s = streams[k % 2]
        loop.eng.advance(loop.sb, loop.new, stream=s.cuda_stream if raw else s)
        other = streams[1 - k % 2]
        other.wait_stream(s) if raw else None
        with torch.cuda.stream(other):
            ak.add_rms_norm(loop.delta, loop.w_norm, loop.x, EPS, residual=loop.res)
        loop.eng.project_to_pool(loop.sb, loop.x, loop.w_qkv, loop.q, THETA, stream=other.cuda_stream if raw else other)
        loop.eng.shared_attention(loop.sb, loop.q, loop.out, lse=loop.lse, stream=s.cuda_stream if raw else s)
        loop.check(np.array([1, 2, 1]), twin, f"step {k}")


def test_a_batch_that_is_let_go_while_its_work_runs():
    """Its memory goes back only when the stream of its last call is done with it."""
    print_case("step batch let go")
    loop = Loop([(2048, [100] * 12)], hq=32, hkv=8, d=128, spare=30)
    side = torch.cuda.Stream()
    loop.give(np.ones(12), 400)
    torch.cuda.synchronize()
    loop.step(side)
    torch.cuda.synchronize()
    want = loop.out.clone()
    x = torch.randn(4096, 4096, device=DEV)
    loop.out.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            x = x @ x * 1e-4
    loop.eng.shared_attention(loop.sb, loop.q, loop.out, stream=side)
    size = loop.sb.workspace.numel()
    loop.sb = None
    junk = [torch.full((size,), 0x7F, dtype=torch.uint8, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(loop.out[:12], want[:12]) and torch.isnan(loop.out[12:]).all() and len(junk) == 4     # (NaN is not equal)


def test_weights_and_rows_of_a_step():
    """attention_weights and scatter take a StepBatch like a planned batch."""
    print_case("step batch: weights, project and scatter")
    loop = Loop([(256, [40, 3]), (64, [5])], max_tokens=6)
    loop.give([1, 1, 2], 500)
    loop.eng.advance(loop.sb, loop.new)
    ak.add_rms_norm(loop.delta, loop.w_norm, loop.x, EPS, residual=loop.res)
    k, v = (torch.empty(6, loop.hkv, loop.d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    twin = loop.twin()
    loop.eng.project(loop.sb, loop.x, loop.w_qkv, loop.q, k, v, THETA)
    loop.eng.scatter(loop.sb, k, v)
    loop.eng.shared_attention(loop.sb, loop.q, loop.out, lse=loop.lse)
    stride = int(loop.held.max()) + 4
    w = torch.zeros(3, loop.hkv, stride, device=DEV)
    loop.eng.attention_weights(loop.sb, loop.q, loop.lse, w, accumulate=False)
    loop.check(np.array([1, 1, 2]), twin, "project and scatter")
    held, cu = loop.held, loop.sb.cu_q.cpu().numpy()
    plan = BatchPlan(loop.tables, cu, held.astype(np.int32), (held - np.diff(cu)).astype(np.int32), np.zeros(3, np.int32),
                     loop.sb.slot_mapping.cpu().numpy()[:4], 2, int(held.max()))
    db = loop.eng.upload(plan)
    w2 = torch.zeros_like(w)
    loop.eng.attention_weights(db, loop.q[:4], loop.lse[:4], w2, accumulate=False)
    assert torch.equal(w, w2)


def test_a_prefilled_batch_goes_on_in_steps():
    """Prompts that share a document are prefilled through the block cache, and their batch, not released, goes on
    with blocks of its own; the shared blocks are those that the cache gave to all."""
    print_case("prefill, then steps")
    hq, hkv, d = 8, 2, 64
    rng = np.random.default_rng(7)
    doc = rng.integers(0, 1000, 320)
    toks = [np.concatenate([doc, rng.integers(0, 1000, m)]).astype(np.int32) for m in (9, 30, 1)]
    eng = PrefillEngine(hq, hkv, d, 64, 80, 8, private_blocks=6)
    db = eng.prepare(toks)
    t = db.n_tokens
    eng.scatter(db, randn_bf16((t, hkv, d), 1), randn_bf16((t, hkv, d), 2))
    held = db.plan.seq_lens
    tables = np.full((3, 40), -1, np.int32)
    tables[:, :db.plan.block_tables.shape[1]] = db.plan.block_tables
    assert (tables[:, :20] == tables[0, :20]).all()
    sb = eng.step_batch(tables, held, [3], [320], max_tokens=3, free_blocks=np.arange(eng.num_phys, eng.num_phys + 6))
    k, v, q = randn_bf16((3, hkv, d), 3), randn_bf16((3, hkv, d), 4), randn_bf16((3, hq, d), 5)
    out = torch.empty_like(q)
    one = torch.ones(3, dtype=torch.int32, device=DEV)
    for step in range(8):                                 # each takes a block on the way
        eng.advance(sb, one)
        eng.scatter(sb, k, v)
        eng.shared_attention(sb, q, out)
        bt = sb.block_tables.cpu().numpy()
        lens = held + step + 1
        assert np.array_equal(sb.seq_lens.cpu().numpy(), lens)
        kr = eng.k_pool.view(torch.bfloat16).permute(0, 2, 1, 3).reshape(-1, hkv, d)
        vr = eng.v_pool.view(torch.bfloat16).permute(0, 3, 1, 2).reshape(-1, hkv, d)
        rows = [torch.from_numpy(bt[r, np.arange(L) // 16].astype(np.int64) * 16 + np.arange(L) % 16).to(DEV) for r, L in enumerate(lens)]
        b = dict(hq=hq, hkv=hkv, d=d, scale=d ** -0.5, q=q, cu=np.arange(4), reqs=[(int(L), int(L) - 1) for L in lens],
                 k=[kr[x].double() for x in rows], v=[vr[x].double() for x in rows])
        check_out(b, out, None, reference(b), f"step {step}")
    assert (bt >= eng.num_phys).any()
    eng.release()
