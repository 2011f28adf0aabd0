"""Eviction by accumulated attention weight on the GPU: the weights against 64 bits, the choice against its
definition, the moved tokens bit for bit, and the steps together as a session runs them."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from oracle import mx4 as omx  # noqa: E402
from paper_2606_21238_amd import BatchPlan  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.gpu_helpers import bits, print_case  # noqa: E402
from tests.mx4_helpers import DEV, attend, check_out, i32, make_batch, reference  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


# ---- the weights ------------------------------------------------------------------------------------

def exact_lse(b, ref):
    return torch.cat([r[2] for r in ref]).float() if len(b["q"]) else torch.empty(0, b["hq"], device=DEV)


def weights_tolerance(b, ref, given):
    """A weight's exponent s - lse is off by the score's error (D 2^-24 of its products' magnitudes) and
    2^-24 of lse's and the exponent's size for the base change and the fused step, its exponential by
    2^-22; lse itself is given.  A sum adds at most as many roundings as it has terms of 32 columns, and the
    terms inside a tile 5 levels."""
    res = []
    for r, (L, P) in enumerate(b["reqs"]):
        g, S = b["hq"] // b["hkv"], L - P
        t = torch.zeros(b["hkv"], L, dtype=torch.float64, device=DEV)
        q = b["q"][b["cu"][r]:b["cu"][r + 1]].double()
        for h in range(b["hq"]):
            kt = b["k"][r][:, h // g].t().contiguous().nan_to_num(nan=0.0)
            s = q[:, h].contiguous() @ kt * b["scale"]
            mag = q[:, h].abs().contiguous() @ kt.abs() * b["scale"]
            l = given[b["cu"][r]:b["cu"][r + 1], h].double()
            s = s.masked_fill(torch.arange(L, device=DEV)[None, :] > torch.arange(P, L, device=DEV)[:, None], -torch.inf)
            p = torch.exp(s - l[:, None])
            rel = 2.0 ** -24 * (b["d"] * mag + 4 * l.abs()[:, None] + 4 * mag) + 2.0 ** -22
            t[h // g] += (p * rel).sum(0) + p.sum(0) * 2.0 ** -24 * (S * g / 32 + 16)
        res.append(t + 2.0 ** -125 * (S * g + 1))
    return res


def run_weights(b, lse, stride, accumulate=True, before=1.0, q=None):
    w = torch.full((len(b["reqs"]), b["hkv"], stride), before, device=DEV)
    ak.attention_weights(b["pool"][0], b["q"] if q is None else q, lse, w, i32(b["bt"]), i32(b["cu"]), i32(b["seq"]),
                         b["scale"], accumulate=accumulate)
    torch.cuda.synchronize()
    return w


WEIGHTS = [
    ([(1, 0)], 4, 2, 64),
    ([(64, 0), (65, 1), (17, 17)], 4, 4, 64),
    ([(L, L - 1) for L in (1, 2, 31, 33, 64, 511, 513, 2049)], 32, 8, 128),
    ([(L, L - 1) for L in (700, 5, 1300)], 5, 1, 64),
    ([(900, 857), (40, 8), (515, 2)], 16, 2, 128),
    ([(1030, 0)], 8, 1, 128),
    ([(700, 600), (260, 0)], 10, 2, 64),
    ([(3000, 2000)], 4, 4, 128),
    ([(6000, 5990), (100, 90)], 64, 8, 128),
]


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("case", range(len(WEIGHTS)))
def test_attention_weights(case, fmt):
    reqs, hq, hkv, d = WEIGHTS[case]
    print_case(f"weights {reqs} hq={hq} hkv={hkv} d={d} {fmt}")
    b = make_batch(reqs, hq, hkv, d, seed=2000 + case, fmt=fmt)
    ref = reference(b)
    lse = exact_lse(b, ref)
    # the reference's own weights go by an lse in 64 bits: half a step of fp32 of each more
    tol = weights_tolerance(b, ref, lse)
    longest = max(L for L, _ in reqs)
    for accumulate in (True, False):
        w = run_weights(b, lse, longest + 3, accumulate)
        for r, (L, _) in enumerate(reqs):
            want = ref[r][4] + (1.0 if accumulate else 0.0)
            err = (w[r, :, :L].double() - want).abs() - tol[r] - 2.0 ** -24 * want.abs() \
                - ref[r][4] * 2.0 ** -24 * float(lse.abs().max() if lse.numel() else 0)
            assert float(err.max()) <= 0, f"request {r}: {float(err.max()):.3g} over its tolerance"
            assert (w[r, :, L:] == 1).all()              # behind the request: as it was
    # an attention call's own lse; a short stride leaves the later tokens out; the same bits again
    _, own, _ = attend(b)
    if lse.numel():
        w = run_weights(b, own, longest, False)
        short = run_weights(b, own, max(1, longest // 2), False)
        assert torch.equal(short, torch.where(torch.arange(short.shape[2], device=DEV) < i32(b["seq"])[:, None, None],
                                              w[:, :, : short.shape[2]], torch.ones_like(short)))
        assert torch.equal(run_weights(b, own, longest, False), w)


MIXED = [
    ([(400, 300)] + [(60 + 31 * i, 59 + 31 * i) for i in range(40)], 16, 4, 64),
    ([(260, 228), (260, 227), (700, 699)] + [(33, 33)] * 3 + [(50 + i, 49 + i) for i in range(9)], 8, 4, 128),
    ([(130, 66), (130, 65)] + [(40 + i, 39 + i) for i in range(20)], 3, 3, 128),
    ([(1500, 0)] + [(20, 20 - i % 2) for i in range(60)], 2, 2, 64),
]


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("case", range(len(MIXED)))
def test_weights_of_decode_and_prefill_in_one_batch(case, fmt):
    """Requests with few columns, with many, with none and at the limits between: each gets its weights once."""
    reqs, hq, hkv, d = MIXED[case]
    print_case(f"weights of a mixed batch {reqs[:3]} hq={hq} hkv={hkv} d={d} {fmt}")
    b = make_batch(reqs, hq, hkv, d, seed=2100 + case, fmt=fmt)
    ref = reference(b)
    lse = exact_lse(b, ref)
    tol = weights_tolerance(b, ref, lse)
    longest = max(L for L, _ in reqs)
    for accumulate in (True, False):
        w = run_weights(b, lse, longest + 3, accumulate)
        for r, (L, _) in enumerate(reqs):
            want = ref[r][4] + (1.0 if accumulate else 0.0)
            err = (w[r, :, :L].double() - want).abs() - tol[r] - 2.0 ** -24 * want.abs() \
                - ref[r][4] * 2.0 ** -24 * float(lse.abs().max())
            assert float(err.max()) <= 0, f"request {r}: {float(err.max()):.3g} over its tolerance"
            assert (w[r, :, L:] == 1).all()


@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
def test_weights_of_non_finite_keys_and_queries(fmt):
    """A NaN key is NaN where some column sees it and touches no other key; so does the NaN column of a query
    reach the keys that it sees and no later ones."""
    print_case(f"weights non-finite {fmt}")
    reqs, hq, hkv, d = [(300, 200), (90, 0), (700, 699)], 8, 2, 128

    def edit(k):
        k[250, 0, 3] = float("nan")
        k[300 + 89, 1, 100] = float("inf")

    b = make_batch(reqs, hq, hkv, d, seed=5, fmt=fmt, k_edit=edit)
    clean = make_batch(reqs, hq, hkv, d, seed=5, fmt=fmt)
    lse = exact_lse(clean, reference(clean))
    want = run_weights(clean, lse, 700, False)
    got = run_weights(b, lse, 700, False)
    bad = torch.zeros_like(want, dtype=torch.bool)
    bad[0, 0, 250] = bad[1, 1, 89] = True
    # (an infinite bf16 key has scores of either infinity or NaN, weights of 0, infinity or NaN)
    assert not torch.isfinite(got[0, 0, 250])
    assert torch.equal(torch.where(bad, 0, got), torch.where(bad, 0, want))
    q = clean["q"].clone()
    q[40, 1] = float("nan")                    # token 240 of request 0, KV head 0
    got = run_weights(clean, lse, 700, False, q=q)
    assert torch.isnan(got[0, 0, :241]).all() and torch.equal(got[0, 0, 241:], want[0, 0, 241:])
    assert torch.equal(got[0, 1], want[0, 1]) and torch.equal(got[1:], want[1:])


# ---- the choice -------------------------------------------------------------------------------------

def choose(w, L, keep, first, recent):
    """The definition, for one request and head."""
    if L <= keep:
        kept = list(range(L))
    else:
        held = set(range(first)) | set(range(L - recent, L))
        v = np.where(np.isnan(w), -np.inf, w.astype(np.float64))
        rest = sorted((i for i in range(L) if i not in held), key=lambda i: (not np.isnan(w[i]), v[i], -i), reverse=True)
        kept = sorted(held | set(rest[: keep - len(held)]))
    return kept


@pytest.mark.parametrize("lens,hkv,keep,first,recent", [
    ([1, 2, 16, 17], 2, 1, 0, 0), ([1, 2, 16, 17], 2, 1, 1, 0), ([40, 300, 0, 5], 3, 33, 4, 7), ([40, 300], 1, 33, 16, 17),
    ([1023, 1024, 1025, 5000], 2, 1024, 1, 100), ([5000, 4097], 4, 4096, 0, 0), ([70000], 1, 3000, 5, 300),
    ([2000], 8, 1, 0, 1), ([900, 33], 2, 900, 3, 3)])
def test_select(lens, hkv, keep, first, recent):
    print_case(f"select {lens} hkv={hkv} keep={keep} first={first} recent={recent}")
    rng = np.random.default_rng(sum(lens) + keep)
    stride = max(lens) + 5
    n = len(lens)
    kinds = {
        "heavy": np.exp(2 * rng.standard_normal((n, hkv, stride))),
        "ties": rng.integers(0, 4, (n, hkv, stride)).astype(np.float64),
        "same": np.full((n, hkv, stride), 0.25),
        "odd": np.where(rng.random((n, hkv, stride)) < 0.3,
                        rng.choice([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.0, 1e-42, -1e-42], (n, hkv, stride)),
                        rng.standard_normal((n, hkv, stride))),
        "near": 1.0 + rng.integers(0, 40, (n, hkv, stride)) * 2.0 ** -23,
    }
    for name, w in kinds.items():
        w = w.astype(np.float32)
        if name == "heavy":
            w[:, :, 1::3] = 0.0
        wt = torch.from_numpy(w).to(DEV)
        kept = torch.full((n, hkv, keep), -9, dtype=torch.int32, device=DEV)
        kw = torch.full((n, hkv, keep + 2), 7.0, device=DEV)
        ak.evict_select(wt, i32(lens), kept, first, recent, kept_weights=kw)
        only = torch.empty_like(kept)
        ak.evict_select(wt, i32(lens), only, first, recent)
        torch.cuda.synchronize()
        got, gw = kept.cpu().numpy(), kw.cpu().numpy()
        for r, L in enumerate(lens):
            for h in range(hkv):
                want = choose(w[r, h], L, keep, first, recent)
                assert got[r, h].tolist() == want + [-1] * (keep - len(want)), f"{name} request {r} head {h}"
                assert np.array_equal(gw[r, h, :keep], np.r_[w[r, h][want], np.zeros(keep - len(want), np.float32)],
                                      equal_nan=True)
        assert (gw[:, :, keep:] == 7).all() and torch.equal(only, kept)


@pytest.mark.parametrize("lens,hkv", [([20000, 16385], 5), ([17000], 257), ([33000, 40], 129), ([16384], 3)])
def test_select_of_long_rows(lens, hkv):
    """Rows longer than what a work-group holds, few and many of them: the choice by a stable sort."""
    print_case(f"select of long rows {lens} hkv={hkv}")
    rng = np.random.default_rng(hkv)
    keep, first, recent = 3001, 4, 100
    w = (rng.integers(0, 9000, (len(lens), hkv, max(lens))) / 8).astype(np.float32)
    kept = torch.empty(len(lens), hkv, keep, dtype=torch.int32, device=DEV)
    kw = torch.empty(len(lens), hkv, keep, device=DEV)
    ak.evict_select(torch.from_numpy(w).to(DEV), i32(lens), kept, first, recent, kept_weights=kw)
    torch.cuda.synchronize()
    got, gw = kept.cpu().numpy(), kw.cpu().numpy()
    for r, L in enumerate(lens):
        if L <= keep:
            assert (got[r] == np.r_[np.arange(L), np.full(keep - L, -1)]).all()
            continue
        rest = np.argsort(-w[r, :, first:L - recent], axis=1, kind="stable")[:, : keep - first - recent] + first
        held = np.tile(np.r_[np.arange(first), np.arange(L - recent, L)], (hkv, 1))
        want = np.sort(np.concatenate([rest, held], axis=1), axis=1)
        assert np.array_equal(got[r], want) and np.array_equal(gw[r], np.take_along_axis(w[r], want, axis=1))


def test_select_takes_a_longer_request_as_its_first_tokens():
    w = torch.rand(1, 1, 50, device=DEV)
    kept = torch.empty(1, 1, 60, dtype=torch.int32, device=DEV)
    ak.evict_select(w, i32([1000]), kept)
    torch.cuda.synchronize()
    assert kept[0, 0].tolist() == list(range(50)) + [-1] * 10


# ---- the move ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["bf16", "mx4"])
@pytest.mark.parametrize("hkv,d,keep", [(2, 64, 1), (3, 128, 16), (2, 128, 45), (5, 64, 100)])
def test_compact(fmt, hkv, d, keep):
    print_case(f"compact {fmt} hkv={hkv} d={d} keep={keep}")
    lens = [200, 90, 17]
    nd = (keep + 15) // 16
    b = make_batch([(L, L) for L in lens], hkv, hkv, d, seed=keep, fmt=fmt, extra_blocks=3 * nd + 2)
    rng = np.random.default_rng(keep)
    kept = np.full((3, hkv, keep), -1, dtype=np.int32)
    for r, L in enumerate(lens):
        for h in range(hkv):
            m = min(L, keep)
            kept[r, h, :m] = np.sort(rng.choice(L, m, replace=False))
    kept[0, 0, keep // 2] = 1 << 20                  # past the table: nothing moves
    dst = np.full((3, nd + 1), -5, dtype=np.int32)
    dst[:, :nd] = b["free"][: 3 * nd].reshape(3, nd)
    before = [p.cpu().numpy().copy() for p in b["pool"]]
    if fmt == "mx4":
        ak.kv_compact_mx4(*b["pool"], i32(b["bt"]), i32(kept), i32(dst))
    else:
        ak.kv_compact(*b["pool"], i32(b["bt"]), i32(kept), i32(dst))
    torch.cuda.synchronize()
    want = [p.copy() for p in before]
    for r in range(3):
        for h in range(hkv):
            for i, p in enumerate(kept[r, h]):
                if not 0 <= p < lens[r]:
                    continue
                sb, so, db, do = b["bt"][r, p // 16], p % 16, dst[r, i // 16], i % 16
                if fmt == "bf16":
                    want[0][db, h, do] = before[0][sb, h, so]
                    want[1][db, h, :, do] = before[1][sb, h, :, so]
                else:
                    src = omx._fields(before[0][sb:sb + 1])
                    kc, vc, ks, vs = (x.copy() for x in omx._fields(want[0][db:db + 1]))
                    kc[0, h, do], ks[0, h, do] = src[0][0, h, so], src[2][0, h, so]
                    vc[0, h, do // 8, :, do % 8], vs[0, h, :, do] = src[1][0, h, so // 8, :, so % 8], src[3][0, h, :, so]
                    want[0][db] = np.concatenate([x[0].reshape(hkv, -1) for x in (kc, vc, ks, vs)], axis=1)
    for got, w in zip(b["pool"], want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_compact_skips_blocks_outside_the_pool():
    b = make_batch([(64, 64)], 2, 2, 64, seed=1, fmt="mx4", extra_blocks=4)
    before = b["pool"][0].clone()
    kept = i32(np.arange(32).reshape(1, 1, 32).repeat(2, 1))
    bt = b["bt"].copy()
    ak.kv_compact_mx4(*b["pool"], i32(bt), kept, i32([[len(before), -1]]))
    bt[0, :2] = [len(before) + 9, -4]
    ak.kv_compact_mx4(*b["pool"], i32(bt), kept, i32([[b["free"][0], b["free"][1]]]))
    torch.cuda.synchronize()
    assert torch.equal(b["pool"][0], before)


# ---- together, as a session runs them -----------------------------------------------------------------

@pytest.mark.parametrize("fmt,hq,hkv,d", [("mx4", 8, 2, 128), ("bf16", 8, 2, 128), ("mx4", 4, 4, 64), ("bf16", 10, 2, 64)])
def test_sessions_are_cut_and_go_on(fmt, hq, hkv, d):
    """Three prompts are prefilled; their weights are taken over the prefill and two decode steps; they are
    cut to `keep` tokens for each head; two more decode steps run on the private blocks.  Every output is
    compared with 64 bits on the tokens that the definition keeps."""
    print_case(f"session {fmt} {hq}/{hkv} heads of {d}")
    rng = np.random.default_rng(3)
    lens, keep, first, recent, steps = [150, 61, 20], 48, 3, 16, 2
    n, nb = len(lens), (48 + 2 + 15) // 16
    toks = [rng.integers(0, 1000, L, dtype=np.int32) for L in lens]
    eng = PrefillEngine(hq, hkv, d, 40, 44, 4, policy="arc", kv_format=fmt, private_blocks=n * nb + 1)
    cap = max(lens) + steps
    weights = torch.zeros(n, hkv, cap, device=DEV)
    rows = [[], []]                                        # per step: K and V rows [tokens, Hkv, D] of each request

    def value(x):
        return torch.from_numpy(omx.stored(bits(x))).to(DEV) if fmt == "mx4" else x.double()

    def as_batch(q, cu, k, v, P):
        L = [len(x) for x in k]
        return dict(hq=hq, hkv=hkv, d=d, q=q, cu=cu, k=k, v=v, reqs=list(zip(L, P)), scale=d ** -0.5)

    K, V = [[] for _ in lens], [[] for _ in lens]           # what each request's cache holds, 64 bits
    total = [torch.zeros(hkv, cap, dtype=torch.float64, device=DEV) for _ in lens]
    for step in range(1 + steps):
        db = eng.prepare(toks)
        plan = db.plan
        T = db.n_tokens
        q, k, v = randn_bf16((T, hq, d), 10 + step), randn_bf16((T, hkv, d), 20 + step), randn_bf16((T, hkv, d), 30 + step)
        eng.scatter(db, k, v)
        out, lse = torch.empty_like(q), torch.empty(T, hq, device=DEV)
        eng.attention(db, q, out, lse=lse)
        eng.attention_weights(db, q, lse, weights, accumulate=True)
        for r in range(n):
            P = int(plan.prefix_lens[r])
            part = slice(int(plan.cu_q[r]), int(plan.cu_q[r + 1]))
            K[r] = torch.cat([K[r][:P], value(k[part])]) if step else value(k[part])
            V[r] = torch.cat([V[r][:P], value(v[part])]) if step else value(v[part])
        b = as_batch(q, plan.cu_q, K, V, plan.prefix_lens.tolist())
        ref = reference(b)
        check_out(b, out, lse, ref, f"step {step}")
        for r in range(n):
            total[r][:, : len(K[r])] += ref[r][4]
        if step < steps:
            eng.release()
            toks = [np.append(t, np.int32(rng.integers(0, 1000))) for t in toks]
    for r in range(n):
        got, L = weights[r].double(), len(K[r])
        assert float(((got - total[r]).abs() / total[r].clamp(min=1e-6))[:, :L].max()) < 1e-4

    dst = np.arange(n * nb, dtype=np.int32).reshape(n, nb) + eng.num_phys
    with pytest.raises(ValueError, match="batch"):
        eng.evict(db, weights, keep, np.vstack([db.plan.block_tables[0, :nb], dst[1:]]), first, recent)
    with pytest.raises(ValueError, match="twice"):
        eng.evict(db, weights, keep, dst[[0, 0, 1]], first, recent)
    with pytest.raises(ValueError, match="outside"):
        eng.evict(db, weights, keep, dst + n * nb, first, recent)
    with pytest.raises(ValueError, match="dst_tables"):
        eng.evict(db, weights, keep, dst[:, : nb - 2], first, recent)
    with pytest.raises(ak.ArckvError):
        eng.evict(db, weights, keep, dst, keep, 1)
    kept, kw = eng.evict(db, weights, keep, dst, n_first=first, n_recent=recent)
    eng.release()
    torch.cuda.synchronize()
    w = weights.cpu().numpy()
    length = [min(len(K[r]), keep) for r in range(n)]
    for r in range(n):
        nk, nv = [], []
        for h in range(hkv):
            want = choose(w[r, h], len(K[r]), keep, first, recent)
            assert kept[r, h].tolist() == want + [-1] * (keep - len(want))
            assert torch.equal(kw[r, h, : len(want)], weights[r, h][want])
            nk.append(K[r][want, h])
            nv.append(V[r][want, h])
        K[r], V[r] = torch.stack(nk, 1), torch.stack(nv, 1)

    weights = torch.zeros(n, hkv, keep + steps, device=DEV)
    weights[:, :, :keep] = kw
    for step in range(steps):
        seq = np.array([x + 1 for x in length], dtype=np.int32)
        plan = BatchPlan(dst, np.arange(n + 1, dtype=np.int32), seq, seq - 1, (seq - 1) // 16,
                         np.array([dst[r, (s - 1) // 16] * 16 + (s - 1) % 16 for r, s in enumerate(seq)], dtype=np.int32),
                         1, int(seq.max()))
        db = eng.upload(plan)
        q, k, v = randn_bf16((n, hq, d), 60 + step), randn_bf16((n, hkv, d), 70 + step), randn_bf16((n, hkv, d), 80 + step)
        eng.scatter(db, k, v)
        out, lse = torch.empty_like(q), torch.empty(n, hq, device=DEV)
        eng.attention(db, q, out, lse=lse)
        eng.attention_weights(db, q, lse, weights)
        K = [torch.cat([K[r], value(k[r:r + 1])]) for r in range(n)]
        V = [torch.cat([V[r], value(v[r:r + 1])]) for r in range(n)]
        b = as_batch(q, plan.cu_q, K, V, (seq - 1).tolist())
        check_out(b, out, lse, reference(b), f"after the cut, step {step}")
        length = seq.tolist()
    if fmt == "mx4":
        slots = i32((dst[:, :, None] * 16 + np.arange(16)).reshape(n, -1)[0][: length[0]])
        ko, vo = (torch.empty(length[0], hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        eng.gather(slots, ko, vo)
        torch.cuda.synchronize()
        assert torch.equal(ko.double(), K[0]) and torch.equal(vo.double(), V[0])
