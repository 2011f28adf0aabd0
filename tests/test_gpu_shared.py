"""Attention over shared prefixes against 64 bits, request by request, with the tolerances of mx4_helpers.reference (the
join of the pieces adds fp32 roundings that its fp32 terms, taken twice, cover)."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import DEV, check_out, i32, reference  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def shared_batch(groups, hq, hkv, d, seed, alone=(), k_edit=None, v_edit=None, room=2):
    """groups: [(P, [(own tokens, new ones among them)])]; alone: requests behind the groups, in none.  Blocks at random
    places of pools whose every byte was 0xFF; the shared blocks of a group are named by all its tables."""
    rng = np.random.default_rng(seed)
    shared = [-(-p // 16) for p, _ in groups]                # (a last block that is not full is shared too: own tokens
    assert all(p % 16 == 0 for p, _ in groups)               # begin in a block of their own)
    reqs = [(p, own, s) for p, rs in groups for own, s in rs] + [(0, own, s) for own, s in alone]
    nb = sum(shared) + sum(-(-own // 16) for _, own, _ in reqs) + 3
    perm, at = rng.permutation(nb).astype(np.int32), 0
    stride = max([(p + own + 15) // 16 for p, own, _ in reqs] + [1]) + room
    bt = np.full((len(reqs), stride), -1, np.int32)
    k_parts, v_parts, slots, r = [], [], [], 0
    pres = []
    for p, rs in groups:
        blocks, at = perm[at:at + p // 16], at + p // 16
        pres.append((blocks, randn_bf16((p, hkv, d), seed + 10 + r), randn_bf16((p, hkv, d), seed + 11 + r)))
        for _ in rs:
            bt[r, :len(blocks)] = blocks
            r += 1
    of = [g for g, (_, rs) in enumerate(groups) for _ in rs] + [-1] * len(alone)
    kp = torch.full((nb, hkv, 16, d), -1, dtype=torch.int16, device=DEV)
    vp = torch.full((nb, hkv, d, 16), -1, dtype=torch.int16, device=DEV)
    for blocks, k, v in pres:
        k_edit and k_edit(k)
        v_edit and v_edit(v)
        ak.kv_scatter(kp, vp, k, v, i32((blocks[:, None] * 16 + np.arange(16)).ravel()))
    b = dict(hq=hq, hkv=hkv, d=d, fmt="bf16", k=[], v=[], reqs=[], scale=d ** -0.5)
    for r, (p, own, s) in enumerate(reqs):
        n = -(-own // 16)
        bt[r, p // 16:p // 16 + n], at = perm[at:at + n], at + n
        k, v = randn_bf16((own, hkv, d), seed + 1000 + r), randn_bf16((own, hkv, d), seed + 3000 + r)
        if own:
            ak.kv_scatter(kp, vp, k, v, i32(bt[r, (p + np.arange(own)) // 16] * 16 + np.arange(own) % 16))
        pk, pv = (pres[of[r]][1], pres[of[r]][2]) if of[r] >= 0 else (k[:0], v[:0])
        b["k"].append(torch.cat([pk, k]).double())
        b["v"].append(torch.cat([pv, v]).double())
        b["reqs"].append((p + own, p + own - s))
    S = [s for _, _, s in reqs]
    b.update(pool=(kp, vp), bt=bt, cu=np.concatenate([[0], np.cumsum(S)]).astype(np.int32), new=S,
             seq=np.array([L for L, _ in b["reqs"]], np.int32), starts=np.cumsum([0] + [len(rs) for _, rs in groups]),
             prefix=np.array([p for p, _ in groups], np.int32), q=randn_bf16((sum(S), hq, d), seed + 3), sizes=[len(rs) for _, rs in groups])
    return b


def bounds_of(b, max_q=None, **more):
    rows = [int(b["cu"][y] - b["cu"][x]) for x, y in zip(b["starts"], b["starts"][1:])]
    kw = dict(max_q=int(b["cu"][-1]) if max_q is None else max_q, max_group_q=max(rows + [0]), max_new=max(b["new"] + [0]))
    kw.update(more)
    return ak.SharedBounds(len(b["reqs"]), len(b["prefix"]), kw["max_q"], kw["max_group_q"], kw["max_new"], b["bt"].shape[1],
                           b["hq"], b["hkv"], b["d"], kw.get("num_cus", 256))


def attend(b, bounds=None, q=None, out=None, stream=None, lse=True, bt=None, seq=None, prefix=None):
    """(out, lse) of the library; workspace and plan begin as garbage."""
    bounds = bounds or bounds_of(b)
    ints, ws_bytes = ak.shared_prefix_sizes(bounds)
    plan = torch.full((ints,), 0x7F7F7F7F, dtype=torch.int32, device=DEV)
    ws = torch.full((max(ws_bytes, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    q = b["q"] if q is None else q
    out = torch.full_like(q, float("nan")) if out is None else out
    lse = torch.full(q.shape[:2], float("nan"), device=DEV) if lse else None
    cu, sl, tables = i32(b["cu"]), i32(b["seq"] if seq is None else seq), i32(b["bt"] if bt is None else bt)
    ak.shared_prefix_plan(bounds, i32(b["starts"]), i32(b["prefix"] if prefix is None else prefix), cu, sl, plan, stream=stream)
    ak.shared_prefix_attention(bounds, *b["pool"], q, out, tables, cu, sl, plan, b["scale"], ws, lse=lse, stream=stream)
    torch.cuda.synchronize()
    return out, lse


def run(b, what, **kw):
    print_case(what)
    out, lse = attend(b, **kw)
    check_out(b, out, lse, reference(b), what)
    return out, lse


SHAPES = [(4, 4, 64), (4, 2, 64), (8, 2, 64), (10, 2, 64), (16, 2, 64), (4, 4, 128), (4, 2, 128), (8, 2, 128), (10, 2, 128), (16, 2, 128)]


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_decode(hq, hkv, d):
    """One row each: a group of a few, one whose columns pass one tile, lengths at and around a tile, requests alone."""
    run(shared_batch([(256, [(24, 1)] * 4), (1008, [(1, 1), (16, 1), (17, 1), (63, 1), (64, 1), (65, 1), (300, 1)])], hq, hkv, d, 1,
                     alone=[(1, 1), (33, 1), (500, 1)]), f"decode {hq}/{hkv} d {d}")
    run(shared_batch([(2048, [(7 * r + 1, 1) for r in range(70)])], hq, hkv, d, 2), f"decode, 70 requests, {hq}/{hkv} d {d}")


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_several_rows(hq, hkv, d):
    """2 rows (the tail kernel's columns), 20 and 128 (narrow tiles), 300 (wide ones), and all of them beside each other."""
    run(shared_batch([(320, [(2, 2), (40, 2), (1, 1)])], hq, hkv, d, 3), f"2 rows {hq}/{hkv} d {d}")
    run(shared_batch([(704, [(20, 20), (45, 9)]), (64, [(20, 3)])], hq, hkv, d, 4, alone=[(33, 16)]), f"20 rows {hq}/{hkv} d {d}")
    run(shared_batch([(512, [(128, 128), (130, 1), (200, 77)])], hq, hkv, d, 5), f"128 rows {hq}/{hkv} d {d}")
    run(shared_batch([(1024, [(300, 300), (10, 1), (500, 129)]), (128, [(400, 260)])], hq, hkv, d, 6, alone=[(600, 300)]),
        f"300 rows {hq}/{hkv} d {d}")


@pytest.mark.parametrize("p", [0, 16, 48, 64, 80, 112, 128, 4080])
def test_prefixes_that_are_no_whole_tiles(p):
    run(shared_batch([(p, [(5, 1), (18, 1), (1, 1)])], 8, 2, 128, 20 + p), f"prefix {p}")


def test_idle_requests_and_empty_groups():
    """Requests without a row, at the ends and between; a group none of whose requests has one."""
    g = [(256, [(10, 0), (9, 1), (0, 0)]), (128, [(4, 0), (0, 0)]), (512, [(0, 0), (1, 1), (40, 0)])]
    run(shared_batch(g, 8, 2, 64, 30, alone=[(5, 0), (6, 2), (0, 0)]), "idle requests")
    b = shared_batch([(64, [(3, 0)] * 3)], 8, 2, 64, 31)
    bounds = bounds_of(b, max_q=4)
    q = randn_bf16((4, 8, 64), 1)
    out, lse = attend(b, bounds=bounds, q=q)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    empty = ak.SharedBounds(0, 0, 0, 0, 0, 0, 8, 2, 64)
    assert ak.shared_prefix_sizes(empty)[0] >= 0


def test_groups_that_begin_behind_the_first_request_and_have_gaps():
    """Requests 0, 3 and 6 are in no group; their tables may name the same blocks all the same."""
    print_case("gaps")
    b = shared_batch([(192, [(5, 1)] * 7)], 8, 2, 128, 33)
    want = reference(b)
    # groups as pairs of starts: [1, 3), [3, 3) empty, [3, 4) with nothing shared, [4, 6)
    b["starts"], b["prefix"] = np.array([1, 3, 3, 4, 6]), np.array([192, 64, 0, 192], np.int32)
    out, lse = attend(b)
    check_out(b, out, lse, want, "gaps")


def test_a_prefix_that_not_every_row_sees():
    """prefix_lens says more than a request has seen: its rows lie inside the shared blocks."""
    print_case("rows inside the prefix")
    b = shared_batch([(512, [(1, 1), (9, 1), (40, 2)])], 8, 2, 64, 35)
    # request 1 now ends inside the shared tokens: 5 rows at 295 .. 299
    b["seq"][1], b["reqs"][1], b["new"][1] = 300, (300, 295), 5
    b["k"][1], b["v"][1] = b["k"][1][:300], b["v"][1][:300]
    b["cu"] = np.concatenate([[0], np.cumsum(b["new"])]).astype(np.int32)
    b["q"] = randn_bf16((int(b["cu"][-1]), 8, 64), 5)
    for prefix in (512, 320, 256, 10_000):
        out, lse = attend(b, prefix=np.array([prefix], np.int32))
        check_out(b, out, lse, reference(b), f"prefix {prefix}")


def test_bounds_only_choose_the_kernels():
    """The same batch with bounds that are too large or too small: other tiles and cuts, the same results."""
    b = shared_batch([(1024, [(9, 3), (100, 1), (33, 20)]), (320, [(40, 4), (3, 1)])], 8, 2, 128, 37)
    for kw in (dict(), dict(max_group_q=1), dict(max_new=1), dict(max_group_q=0, max_new=0), dict(num_cus=1), dict(num_cus=7),
               dict(num_cus=2000), dict(max_group_q=29, max_new=29)):
        run(b, f"bounds {kw}", bounds=bounds_of(b, **kw))


def test_rows_behind_the_last_are_left_alone():
    print_case("rows behind")
    b = shared_batch([(512, [(9, 1), (70, 2)])], 8, 2, 128, 39)
    want = reference(b)
    n = int(b["cu"][-1])
    q = torch.cat([b["q"], torch.full((40, 8, 128), float("nan"), dtype=torch.bfloat16, device=DEV)])
    out = torch.full_like(q, 3.0)
    for kw in (dict(), dict(max_new=43, max_group_q=43)):
        _, lse = attend(b, bounds=bounds_of(b, max_q=n + 40, **kw), q=q, out=out)
        check_out(b, out[:n], lse[:n], want, "rows behind")
        assert (out[n:] == 3.0).all() and torch.isnan(lse[n:]).all()


@pytest.mark.parametrize("shift", [1, 4])
def test_queries_and_outputs_at_any_address(shift):
    for groups, what in (([(512, [(9, 1), (70, 2)])], "tail"), ([(1024, [(128, 100), (70, 40)])], "wide"), ([(256, [(30, 10)])], "narrow")):
        print_case(f"shift {shift} {what}")
        b = shared_batch(groups, 8, 2, 128, 41)
        n = b["q"].numel()
        buf, obuf = (torch.full((n + 16,), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        q, out = (x[shift:shift + n].view(b["q"].shape) for x in (buf, obuf))
        q.copy_(b["q"])
        _, lse = attend(b, q=q, out=out)
        check_out(b, out, lse, reference(b), what)
        assert torch.isnan(obuf[:shift]).all() and torch.isnan(obuf[shift + n:]).all()


@pytest.mark.parametrize("num_cus", [256, 16])
def test_one_long_request_among_many(num_cus):
    """More units than the chip takes at a time, and one with most of the keys: it is cut to a unit's share."""
    for rows, what in ((1, "tail"), (30, "narrow"), (70, "wide")):
        n = 20 if num_cus == 16 else 180
        groups = [(128, [(rows + r % 9, rows) for r in range(n)] + [(9000, rows)]), (4096, [(rows, rows), (5000, rows)])]
        b = shared_batch(groups, 8, 2, 64, 57)
        run(b, f"one long among {n}, {what}, {num_cus} units", bounds=bounds_of(b, num_cus=num_cus))


def test_very_long_prefix():
    """More keys than one item may hold (65536), of few and of many rows."""
    for rs in ([(3, 1)] * 3, [(90, 70)] * 2):
        run(shared_batch([(70_016, rs)], 4, 2, 64, 43), f"prefix 70016, {len(rs)} x {rs[0][1]}")


@pytest.mark.parametrize("n,per", [(600, 1), (600, 3), (1500, 1500), (2100, 7)])
def test_many_requests(n, per):
    rng = np.random.default_rng(n)
    groups = [(int(rng.integers(0, 9)) * 16, [(int(rng.integers(1, 40)), 1) for _ in range(per)]) for _ in range(n // per)]
    run(shared_batch(groups, 4, 2, 64, 45), f"{n} requests in groups of {per}")


def test_scores_that_move_infinities_and_nan():
    """Keys whose scores grow along the prefix, an infinite value and a NaN key in one group only."""
    def grow(k):
        k.mul_(torch.linspace(0.1, 6, max(len(k), 1), device=k.device)[:len(k), None, None].to(k.dtype))

    run(shared_batch([(2048, [(30, 1)] * 6)], 8, 2, 128, 47, k_edit=grow), "growing scores")
    for what in ("inf value", "nan key"):
        b = shared_batch([(256, [(9, 1), (20, 2)]), (512, [(5, 1), (80, 3)])], 8, 2, 128, 49)
        blk = int(b["bt"][0, 4])
        if what == "inf value":
            b["pool"][1][blk, 1, 5, 3] = 0x7F80                      # token 67 of group 0, head 1, dim 5
            for r in (0, 1):
                b["v"][r][67, 1, 5] = float("inf")
        else:
            b["pool"][0][blk, 1, 3, 5] = 0x7FC0
            for r in (0, 1):
                b["k"][r][67, 1, 5] = float("nan")
        print_case(what)
        out, lse = attend(b)
        ref = reference(b)
        if what == "inf value":        # inf times a positive weight: inf, where the reference says NaN
            for r in (0, 1):
                rows = slice(int(b["cu"][r]), int(b["cu"][r + 1]))
                assert not torch.isfinite(out[rows, 4:, 5]).any()
                out[rows, 4:, 5] = float("nan")
        else:
            assert torch.isnan(out[:3, 4:]).all() and torch.isnan(lse[:3, 4:]).all()
        check_out(b, out, lse, ref, what)


def test_table_entries_outside_the_pool():
    """They read block 0 in the place; other requests and heads do not notice."""
    print_case("bad entries")
    b = shared_batch([(256, [(30, 1)] * 3), (128, [(70, 1)] * 2)], 8, 2, 128, 51, alone=[(90, 1)])
    want = reference(b)
    bt = b["bt"].copy()
    bt[0, 3], bt[1, 3], bt[2, 3] = -5, -5, -5             # in the shared keys of group 0
    bt[5, 2] = 2 ** 30                                    # own key of the last
    out, lse = attend(b, bt=bt)
    for r in (3, 4):
        rows = slice(int(b["cu"][r]), int(b["cu"][r + 1]))
        sub = dict(b, reqs=[b["reqs"][r]], cu=np.array([0, b["new"][r]]))
        check_out(sub, out[rows], lse[rows], [want[r]], f"request {r}")


def test_other_stream_two_at_once_and_same_bits():
    print_case("streams")
    bs = [shared_batch([(3000 // 16 * 16, [(50, 1)] * 20)], 32, 8, 128, 53), shared_batch([(1024, [(200, 60)] * 3)], 32, 8, 128, 54)]
    want = [attend(b) for b in bs]
    for b, (o, l) in zip(bs, want):
        check_out(b, o, l, reference(b), "alone")
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for b, s in zip(bs, side):
            with torch.cuda.stream(s):
                bounds = bounds_of(b)
                ints, ws_bytes = ak.shared_prefix_sizes(bounds)
                plan, ws = torch.empty(ints, dtype=torch.int32, device=DEV), torch.empty(ws_bytes, dtype=torch.uint8, device=DEV)
                t = [i32(x) for x in (b["starts"], b["prefix"], b["cu"], b["seq"], b["bt"])]
                out, lse = torch.empty_like(b["q"]), torch.empty(b["q"].shape[:2], device=DEV)
                ak.shared_prefix_plan(bounds, *t[:4], plan)
                ak.shared_prefix_attention(bounds, *b["pool"], b["q"], out, t[4], t[2], t[3], plan, b["scale"], ws, lse=lse)
                got.append((out, lse))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


def test_without_lse_the_same_bits():
    print_case("no lse")
    b = shared_batch([(512, [(9, 1), (70, 2)])], 8, 2, 128, 55)
    assert torch.equal(attend(b)[0], attend(b, lse=False)[0])
