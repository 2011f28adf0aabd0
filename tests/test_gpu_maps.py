"""The maps of a step made on the device, against a plain loop over the requests and their tokens: whole numbers, so equal."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def plain(new, held, tables, free, count, slot_cap, num_blocks):
    """(seq_lens, cu_q, tables, slots, free left) by the definition, one request after the other."""
    n, stride = tables.shape
    tables, seq = tables.copy(), np.array(held, np.int64)
    left = count = min(max(count, 0), len(free))
    cu, slots = [0], []
    blocks = tokens = 0
    for r in range(n):
        h, w, got = int(held[r]), int(new[r]), 0
        if w >= 0 and h >= 0 and h + w <= 16 * stride and h + w < 2 ** 31:
            b = -(-(h + w) // 16) - -(-h // 16)
            blocks, tokens = blocks + b, tokens + w
            if tokens <= slot_cap and (b == 0 or blocks <= count):
                got = w
                for c in range(-(-h // 16), -(-h // 16) + b):
                    left -= 1
                    tables[r, c] = free[left]
                for p in range(h, h + w):
                    blk = int(tables[r, p // 16])
                    slots.append(blk * 16 + p % 16 if 0 <= blk < num_blocks else -1)
        seq[r] = h + got
        cu.append(cu[-1] + got)
    return seq, np.array(cu), tables, np.array(slots + [-1] * (slot_cap - len(slots))), left


class Case:
    def __init__(self, seed, n, stride, mean_new, free_share, slot_share=1.0, idle=0.2, odd=True):
        rng = np.random.default_rng(seed)
        self.new = rng.integers(0, 2 * mean_new + 1, n)
        self.new[rng.random(n) < idle] = 0
        self.held = rng.integers(0, max(16 * stride - mean_new, 1), n)
        if odd and n > 4:
            self.held[0], self.new[1], self.held[2] = 0, -3, -5           # empty, ended, no request
            self.new[3] = 2 ** 31 - 1
            self.held[4] = 16 * stride                                    # full
        used = -(-np.maximum(self.held, 0) // 16)
        need = np.maximum(-(-(self.held + np.minimum(self.new, 16 * stride)) // 16) - used, 0)
        self.count = int(need.sum() * free_share)
        total = int(used.sum())
        self.num_blocks = total + self.count + 3
        ids = rng.permutation(self.num_blocks).astype(np.int32)
        self.tables = np.full((n, stride), -1, np.int32)
        self.tables[np.arange(stride) < used[:, None]] = ids[:total]
        self.free = ids[total:total + self.count].copy()
        self.slot_cap = int(max(self.new[self.new < 2 ** 30].clip(0).sum() * slot_share, 0)) + (5 if slot_share >= 1 else 0)

    def tensors(self):
        i = lambda a: torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(np.int32))).to(DEV)  # noqa: E731
        n = len(self.new)
        return dict(new_tokens=i(self.new), held=i(self.held), block_tables=i(self.tables), free_blocks=i(self.free),
                    free_count=i([self.count]), cu_q=torch.full((n + 1,), -7, dtype=torch.int32, device=DEV),
                    seq_lens=torch.full((n,), -7, dtype=torch.int32, device=DEV),
                    slot_mapping=torch.full((self.slot_cap,), -7, dtype=torch.int32, device=DEV),
                    free_left=torch.full((1,), -7, dtype=torch.int32, device=DEV), num_blocks=self.num_blocks)

    def want(self):
        return plain(self.new, self.held, self.tables, self.free, self.count, self.slot_cap, self.num_blocks)


def same(t, want):
    seq, cu, tables, slots, left = want
    for name, x in (("seq_lens", seq), ("cu_q", cu), ("block_tables", tables), ("slot_mapping", slots), ("free_left", [left])):
        assert np.array_equal(t[name].cpu().numpy(), np.asarray(x)), name


@pytest.mark.parametrize("n", [0, 1, 5, 64, 1023, 1024, 1025, 3000])
@pytest.mark.parametrize("mean_new,free_share,slot_share", [(1, 1.0, 1.0), (1, 0.4, 1.0), (40, 1.2, 1.0), (40, 0.7, 1.0), (7, 1.0, 0.5),
                                                           (16, 0.0, 1.0)])
def test_against_the_loop(n, mean_new, free_share, slot_share):
    print_case(f"maps n {n} new {mean_new} free {free_share} slots {slot_share}")
    c = Case(n + mean_new, n, 9, mean_new, free_share, slot_share)
    t = c.tensors()
    ak.batch_maps(**t)
    same(t, c.want())
    assert np.array_equal(t["held"].cpu().numpy(), c.held.astype(np.int32))


def test_one_long_request_and_a_long_chunk():
    print_case("maps 1 x 200000")
    for held, new, free_share in ((0, 200_000, 1.0), (12_345, 100_001, 1.0), (15, 8193, 0.999)):
        c = Case(1, 1, 20_000, 1, 1.0, odd=False)
        c.held, c.new = np.array([held]), np.array([new])
        used, need = -(-held // 16), -(-(held + new) // 16) - -(-held // 16)
        c.num_blocks, c.count, c.slot_cap = used + need, int(need * free_share), new + 3
        ids = np.random.default_rng(2).permutation(c.num_blocks).astype(np.int32)
        c.tables[:] = -1
        c.tables[0, :used] = ids[:used]
        c.free = ids[used:used + c.count]
        t = c.tensors()
        ak.batch_maps(**t)
        same(t, c.want())


def test_bad_counts_and_blocks():
    print_case("maps bad counts and blocks")
    for count in (-4, 10 ** 9):
        c = Case(3, 40, 9, 5, 0.6)
        c.count = count
        t = c.tensors()
        ak.batch_maps(**t)
        same(t, c.want())
    c = Case(4, 60, 9, 20, 1.0)
    c.free[::3] = -9
    c.free[1::3] = c.num_blocks                        # just outside
    c.tables[5:, 0] = 2 ** 30
    t = c.tensors()
    ak.batch_maps(**t)
    same(t, c.want())


def test_in_place_steps_and_a_replayed_graph():
    """seq_lens in held's place and free_left in free_count's: each call, or replay, goes on from the last."""
    for mean_new, cap in ((1, 100), (200, 40_000)):
        print_case(f"maps in place, new {mean_new}")
        rng = np.random.default_rng(mean_new)
        n, stride = 80, 200
        c = Case(5, n, stride, 1, 1.0, odd=False)
        c.held = rng.integers(0, 200, n)
        used = -(-c.held // 16)
        c.num_blocks = 9000
        ids = rng.permutation(9000).astype(np.int32)
        c.tables[:] = -1
        c.tables[np.arange(stride) < used[:, None]] = ids[:used.sum()]
        c.free, c.count, c.slot_cap = ids[used.sum():used.sum() + 2500], 2500, cap
        c.new = rng.integers(0, 2 * mean_new + 1, n)
        t = c.tensors()
        t["seq_lens"], t["free_left"] = t["held"], t["free_count"]
        t["true_offset"] = torch.arange(n, dtype=torch.int32, device=DEV)
        t["true_lens"] = torch.empty(n, dtype=torch.int32, device=DEV)
        start = {k: t[k].clone() for k in ("held", "free_count", "block_tables")}
        ak.batch_maps(**t)
        torch.cuda.synchronize()
        for k, v in start.items():
            t[k].copy_(v)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ak.batch_maps(**t)
        for step in range(6):
            c.new = rng.integers(0, 2 * mean_new + 1, n)
            t["new_tokens"].copy_(torch.from_numpy(c.new.astype(np.int32)))
            t["slot_mapping"].fill_(-7)
            if step % 2:
                ak.batch_maps(**t)                     # eager and replayed steps in turn
            else:
                g.replay()
            torch.cuda.synchronize()
            want = c.want()
            same(t, want)
            assert np.array_equal(t["true_lens"].cpu().numpy(), want[0] + np.arange(n))
            c.held, c.tables, c.count = want[0], want[2], want[4]


def test_other_stream():
    print_case("maps on another stream")
    c = Case(8, 500, 30, 100, 1.0)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        t = c.tensors()
        ak.batch_maps(**t)
    s.synchronize()
    same(t, c.want())
