"""The 4-bit cache's and eviction's calls as programs make them: captured into a graph and replayed, on another
stream than torch's current one, on views, and in the device-checked build."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd import _lib  # noqa: E402
from paper_2606_21238_amd.build import CHECKED_LIB  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import DEV, attend, check_out, i32, make_batch, reference  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


class Steps:
    """Store, read back, attend with lse, weigh, choose and move, on buffers made once."""

    def __init__(self, reqs, hq, hkv, d, fmt, num_cus, keep=24):
        nb = -(-keep // 16)
        b = self.b = make_batch(reqs, hq, hkv, d, seed=11, fmt=fmt, extra_blocks=len(reqs) * nb)
        self.ap = ak.attention_plan(b["cu"], b["seq"], hq, hkv, d, num_cus)
        L = int(b["seq"].max())
        self.dev = [i32(b[x]) for x in ("bt", "cu", "seq", "slots")]
        self.work = i32(self.ap.work)
        self.ws = torch.empty(max(self.ap.ws_bytes, 16), dtype=torch.uint8, device=DEV)
        n = sum(x for x, _ in reqs)
        self.k, self.v = randn_bf16((n, hkv, d), 21), randn_bf16((n, hkv, d), 22)
        self.back = [torch.zeros_like(self.k) for _ in range(2 if fmt == "mx4" else 0)]
        self.out = torch.zeros_like(b["q"])
        self.lse = torch.zeros(b["q"].shape[:2], device=DEV)
        self.w = torch.full((len(reqs), hkv, L), 3.0, device=DEV)    # behind a request it stays
        self.kept = torch.zeros(len(reqs), hkv, keep, dtype=torch.int32, device=DEV)
        self.kw = torch.zeros(len(reqs), hkv, keep, device=DEV)
        self.dst = i32(b["free"][: len(reqs) * nb].reshape(len(reqs), nb))

    def call(self, stream=None):
        b, ap = self.b, self.ap
        bt, cu, seq, slots = self.dev
        mx4 = b["fmt"] == "mx4"
        if mx4:
            ak.kv_scatter_mx4(*b["pool"], self.k, self.v, slots, stream=stream)
            ak.kv_gather_mx4(*b["pool"], slots, *self.back, stream=stream)
        else:
            ak.kv_scatter(*b["pool"], self.k, self.v, slots, stream=stream)
        (ak.prefill_attention_mx4 if mx4 else ak.prefill_attention)(
            *b["pool"], b["q"], self.out, bt, cu, seq, self.work, ap.n_work, ap.n_combine, ap.tile_cols, b["scale"], self.ws,
            ap.ws_bytes, stream=stream, lse=self.lse)
        ak.attention_weights(b["pool"][0], b["q"], self.lse, self.w, bt, cu, seq, b["scale"], accumulate=False, stream=stream)
        ak.evict_select(self.w, seq, self.kept, 2, 5, kept_weights=self.kw, stream=stream)
        if mx4:
            ak.kv_compact_mx4(*b["pool"], bt, self.kept, self.dst, stream=stream)
        else:
            ak.kv_compact(*b["pool"], bt, self.kept, self.dst, stream=stream)

    def results(self):
        return [x.clone() for x in (*self.b["pool"], *self.back, self.out, self.lse, self.w, self.kept, self.kw)]

    def spoil(self):
        for x in (*self.b["pool"], *self.back, self.out, self.lse, self.w, self.kept, self.kw, self.ws):
            x.view(torch.uint8).fill_(0xFF)
        self.w.fill_(3.0)


CASES = [([(300, 299), (77, 76), (1000, 999)], 32, 8, 128, 256),
         ([(900, 880), (60, 40)], 16, 4, 64, 100000),
         ([(700, 400), (130, 0)], 8, 1, 128, 100000),
         ([(400, 200)] * 3, 8, 8, 64, 16)]


@pytest.mark.parametrize("fmt", ["mx4", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_captured_steps_replay_as_the_eager_ones(case, fmt):
    print_case(f"graph of all steps {CASES[case]} {fmt}")
    s = Steps(*CASES[case][:4], fmt, CASES[case][4])
    s.call()
    torch.cuda.synchronize()
    want = s.results()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.call()
    for k in range(3):
        s.spoil()                                  # eager work between the replays
        junk = torch.randn(1 << 18, device=DEV).sum()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(s.results(), want)), f"replay {k}"
        assert torch.isfinite(junk)
    s.spoil()
    s.call()                                       # and eager again
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.results(), want))


@pytest.mark.parametrize("raw", [False, True])
def test_steps_on_another_stream(raw):
    """Behind long work on torch's stream, the calls run on a stream of their own, given as its handle or
    as the current one."""
    print_case("steps on a side stream")
    s = Steps(*CASES[1][:4], "mx4", 256)
    s.call()
    torch.cuda.synchronize()
    want = s.results()
    s.spoil()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    x = torch.randn(4096, 4096, device=DEV)
    for _ in range(20):
        x = x @ x * 1e-4
    if raw:
        s.call(side.cuda_stream)
    else:
        with torch.cuda.stream(side):
            s.call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.results(), want))
    torch.cuda.synchronize()


def test_engine_steps_on_another_stream():
    print_case("engine, evict on a side stream")
    rng = np.random.default_rng(2)
    toks = [rng.integers(0, 1000, n, dtype=np.int32) for n in (130, 70)]
    res = []
    for side in (None, torch.cuda.Stream()):
        eng = PrefillEngine(8, 2, 64, 20, 24, 2, kv_format="mx4", private_blocks=4, pool_fill=0)
        db = eng.prepare(toks, stream=side)
        T = db.n_tokens
        q, k, v = randn_bf16((T, 8, 64), 1), randn_bf16((T, 2, 64), 2), randn_bf16((T, 2, 64), 3)
        out, lse = torch.empty_like(q), torch.empty(T, 8, device=DEV)
        w = torch.zeros(2, 2, 130, device=DEV)
        torch.cuda.synchronize()
        x = torch.randn(4096, 4096, device=DEV)
        for _ in range(10):
            x = x @ x * 1e-4
        eng.scatter(db, k, v, stream=side)
        eng.attention(db, q, out, stream=side, lse=lse)
        eng.attention_weights(db, q, lse, w, stream=side)
        kept, kw = eng.evict(db, w, 20, np.arange(4, dtype=np.int32).reshape(2, 2) + 24, 1, 4, stream=side)
        (side or torch.cuda.current_stream()).synchronize()
        res.append([t.clone() for t in (out, lse, w, kept, kw, eng.kv_pool)])
        torch.cuda.synchronize()
        eng.release()
    assert all(torch.equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("fmt", ["mx4", "bf16"])
@pytest.mark.parametrize("reqs,hq,hkv,d", [([(600, 400), (33, 0)], 8, 2, 128), ([(200, 199), (70, 68)], 5, 1, 64)])
def test_weights_of_views(reqs, hq, hkv, d, fmt):
    """q and lse that start anywhere in their storage: the same bits as aligned ones."""
    print_case(f"weights of views {reqs} {fmt}")
    b = make_batch(reqs, hq, hkv, d, seed=31, fmt=fmt)
    _, lse, _ = attend(b)

    def weigh(q, l):
        w = torch.zeros(len(reqs), hkv, 600, device=DEV)
        ak.attention_weights(b["pool"][0], q, l, w, i32(b["bt"]), i32(b["cu"]), i32(b["seq"]), b["scale"])
        torch.cuda.synchronize()
        return w

    want = weigh(b["q"], lse)
    n, m = b["q"].numel(), lse.numel()
    q = torch.empty(n + 8, dtype=torch.bfloat16, device=DEV)[3:3 + n].view_as(b["q"]).copy_(b["q"])
    l = torch.empty(m + 8, device=DEV)[1:1 + m].view_as(lse).copy_(lse)
    assert torch.equal(weigh(q, l), want)


@pytest.mark.parametrize("fmt", ["mx4", "bf16"])
def test_weights_of_a_request_without_new_tokens(fmt):
    """Nothing is added, and without accumulation zeros are written, whatever its keys are."""
    print_case(f"weights without rows {fmt}")

    def edit(k):
        k[:] = float("nan")

    for many in (False, True):                       # both kernels: by the batch's mean number of columns
        reqs = [(90, 90), (70, 0) if many else (70, 69)]
        b = make_batch(reqs, 8, 2, 64, seed=41, fmt=fmt, k_edit=edit)
        lse = torch.zeros(b["q"].shape[:2], device=DEV)
        for accumulate in (True, False):
            w = torch.full((2, 2, 95), 5.0, device=DEV)
            ak.attention_weights(b["pool"][0], b["q"], lse, w, i32(b["bt"]), i32(b["cu"]), i32(b["seq"]), b["scale"],
                                 accumulate=accumulate)
            torch.cuda.synchronize()
            assert (w[0, :, :90] == (5.0 if accumulate else 0.0)).all() and (w[0, :, 90:] == 5).all()
            assert torch.isnan(w[1, :, :70]).all() and (w[1, :, 70:] == 5).all()


def test_short_tables():
    """A block table that ends before its request: weights stop there."""
    b = make_batch([(100, 99)], 8, 2, 64, seed=51)
    _, lse, _ = attend(b)
    w = torch.full((1, 2, 100), 5.0, device=DEV)
    ak.attention_weights(b["pool"][0], b["q"], lse, w, i32(b["bt"][:, :3]), i32(b["cu"]), i32(b["seq"]), b["scale"],
                         accumulate=False)
    torch.cuda.synchronize()
    assert (w[:, :, 48:] == 5).all() and (w[:, :, :48] < 1.001).all()


def test_the_same_token_and_slot_twice():
    """A kept position named twice is moved twice; a slot named twice with equal rows holds that row."""
    b = make_batch([(40, 40)], 2, 2, 64, seed=61, extra_blocks=2)
    rows, at = randn_bf16((1, 2, 64), 1).repeat(2, 1, 1), i32([int(b["slots"][7])] * 2)
    ak.kv_scatter_mx4(*b["pool"], rows, rows, at)
    kept = i32(np.array([[[7, 7, 9], [7, 8, 7]]]))
    ak.kv_compact_mx4(*b["pool"], i32(b["bt"]), kept, i32(b["free"][:1].reshape(1, 1)))
    back = [torch.empty(5, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ak.kv_gather_mx4(*b["pool"], i32(list(b["free"][0] * 16 + np.arange(3)) + [int(b["slots"][7])] * 2), *back)
    torch.cuda.synchronize()
    for x in back:
        assert torch.equal(x[0, 0], x[3, 0]) and torch.equal(x[1, 0], x[3, 0]) and torch.equal(x[0, 1], x[3, 1])
        assert torch.equal(x[2, 1], x[3, 1]) and torch.equal(x[3], x[4])


def test_refusals_of_the_binding():
    b = make_batch([(40, 30)], 8, 2, 64, seed=71)
    pool, q = b["pool"][0], b["q"]
    ints = [i32(b[x]) for x in ("bt", "cu", "seq")]
    lse, w = torch.zeros(10, 8, device=DEV), torch.zeros(1, 2, 40, device=DEV)
    k = randn_bf16((3, 2, 64), 1)
    slots = i32([0, 1, 2])
    bad = [
        lambda: ak.kv_scatter_mx4(pool, k, k[:2], slots),
        lambda: ak.kv_scatter_mx4(pool[:, :, :-1].contiguous(), k, k, slots),
        lambda: ak.kv_scatter_mx4(pool, k, k, slots[:2]),
        lambda: ak.kv_scatter_mx4(pool, k.cpu(), k, slots),
        lambda: ak.kv_gather_mx4(pool, slots, k.float(), k),
        lambda: ak.attention_weights(pool, q, lse[:5], w, *ints, 0.1),
        lambda: ak.attention_weights(pool, q, lse, w[:, :1].contiguous(), *ints, 0.1),
        lambda: ak.attention_weights(pool, q, lse, w.to(torch.int32), *ints, 0.1),
        lambda: ak.attention_weights(pool[:, :, :100].contiguous(), q, lse, w, *ints, 0.1),
        lambda: ak.attention_weights(pool, q, None, w, *ints, 0.1),
        lambda: ak.evict_select(w, ints[2], torch.zeros(1, 3, 4, dtype=torch.int32, device=DEV)),
        lambda: ak.evict_select(w, ints[2].cpu(), torch.zeros(1, 2, 4, dtype=torch.int32, device=DEV)),
        lambda: ak.kv_compact_mx4(pool, ints[0], torch.zeros(2, 2, 4, dtype=torch.int32, device=DEV), ints[0]),
        lambda: PrefillEngine(8, 2, 64, 4, 6, 2, kv_format="fp8"),
        lambda: PrefillEngine(8, 2, 64, 4, 6, 2, private_blocks=-1),
    ]
    for k2, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print(k2)
    with pytest.raises(ak.ArckvError):
        ak.evict_select(w, ints[2], torch.zeros(1, 2, 4, dtype=torch.int32, device=DEV), n_first=3, n_recent=2)
    eng = PrefillEngine(8, 2, 64, 4, 6, 2, kv_format="mx4", pool_fill=0)
    db = eng.prepare([np.arange(20, dtype=np.int32)])
    q, k = randn_bf16((20, 8, 64), 1), randn_bf16((20, 2, 64), 2)
    eng.scatter(db, k, k)
    w = torch.zeros(1, 2, 20, device=DEV)
    lse, out = torch.zeros(20, 8, device=DEV), torch.empty_like(q)
    dst = np.array([[5]], dtype=np.int32)
    for f in (lambda: eng.project_to_pool(db, q, q, q, 1e4), lambda: eng.attention(db, q, out, lse=lse[:3]),
              lambda: eng.attention(db, q, out.cpu()), lambda: eng.attention_weights(db, q, lse, w.cpu()),
              lambda: eng.attention_weights(db, q, lse.half(), w), lambda: eng.gather(i32([0]).cpu(), k[:1], k[:1]),
              lambda: eng.evict(db, w[:, :, :10].contiguous(), 8, dst), lambda: eng.evict(db, w, 17, dst),
              lambda: eng.evict(db, w, 8, np.array([[6]], dtype=np.int32)),
              lambda: eng.evict(db, w, 8, db.plan.block_tables[:, :1])):
        with pytest.raises(ValueError):
            f()
    kept, kw = eng.evict(db, w, 0, np.zeros((1, 0), dtype=np.int32))
    assert kept.shape == (1, 2, 0) and kw.shape == (1, 2, 0)
    eng.release()
    with pytest.raises(ValueError):
        PrefillEngine(8, 2, 64, 4, 6, 2).gather(i32([0]), k[:1], k[:1])


def test_evict_is_not_captured(monkeypatch):
    """Its host table would be gone when the graph is replayed."""
    eng = PrefillEngine(8, 2, 64, 4, 6, 2, kv_format="mx4", pool_fill=0, private_blocks=1)
    db = eng.prepare([np.arange(20, dtype=np.int32)])
    w = torch.zeros(1, 2, 20, device=DEV)
    dst = np.array([[6]], dtype=np.int32)
    for stream in (None, torch.cuda.Stream()):
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
            with pytest.raises(ValueError, match="captured"):
                eng.evict(db, w, 8, dst, stream=stream)
    kept, _ = eng.evict(db, w, 8, dst)
    assert kept[0, 0].tolist() == list(range(8))
    eng.release()


def test_checked_build_records_what_it_turns_away(monkeypatch):
    print_case("checked build, 4-bit calls")
    chk = _lib.load(CHECKED_LIB)
    monkeypatch.setattr(_lib, "_lib", chk)
    ak.device_checks(reset=True)
    for reqs in ([(300, 299), (40, 39)], [(700, 400), (130, 0)]):
        s = Steps(reqs, 8, 2, 128, "mx4", 100000)
        s.call()
        torch.cuda.synchronize()
        check_out(s.b, s.out, s.lse, reference(dict(s.b, k=_stored(s.k, reqs), v=_stored(s.v, reqs))), "checked build")
        assert ak.device_checks() == (0, 0)
        bt = s.b["bt"].copy()
        bt[0, 1] = len(s.b["pool"][0])
        good, s.dev[0] = s.dev[0], i32(bt)
        s.call()
        kind, count = ak.device_checks()
        assert kind == ak._lib.CHECK_BLOCK and count > 0
        s.dev[0] = good
        slots = s.dev[3].clone()
        slots[5] = 16 * len(s.b["pool"][0])
        ak.kv_scatter_mx4(*s.b["pool"], s.k, s.v, slots)
        assert ak.device_checks()[0] == ak._lib.CHECK_SLOT
        work = s.ap.work.copy()
        work[0, 0] = 99
        s.work = i32(work)
        s.call()
        assert ak.device_checks()[0] == ak._lib.CHECK_WORK


def _stored(x, reqs):
    from oracle import mx4 as omx
    from tests.gpu_helpers import bits
    rows, at, res = torch.from_numpy(omx.stored(bits(x))).to(DEV), 0, []
    for L, _ in reqs:
        res.append(rows[at:at + L])
        at += L
    return res
