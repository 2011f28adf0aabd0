"""The 4-bit KV cache on the GPU: rows into the pool and back against the oracle, bit for bit."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from oracle import mx4 as omx  # noqa: E402
from oracle.attention import bf16_to_f64  # noqa: E402
from tests.gpu_helpers import bits, print_case  # noqa: E402

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def dev_bits(b):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).to(DEV).view(torch.bfloat16)


def random_rows(n, hkv, d, rng, kind):
    """bf16 bits of K or V rows: normal ones, or any bit patterns (few groups without NaN or infinity)."""
    if kind == "normal":
        x = (rng.standard_normal((n, hkv, d)) * 2.0 ** rng.integers(-20, 20, (n, hkv, 1))).astype(np.float32)
        return (x.view(np.uint32) >> 16).astype(np.uint16)
    b = rng.integers(0, 65536, (n, hkv, d)).astype(np.uint16)
    e = rng.integers(0, 255, (n, hkv, d // 32, 1))                # half of the groups: magnitudes around one exponent
    near = (np.clip(e - rng.integers(0, 4, (n, hkv, d // 32, 32)), 0, 254) << 7).astype(np.uint16)
    near |= b.reshape(near.shape) & 0x807F
    pick = rng.integers(0, 2, (n, hkv, d // 32, 1)) == 1
    return np.where(pick, near, b.reshape(near.shape)).reshape(n, hkv, d).astype(np.uint16)


def store(k, v, slots, nblk):
    hkv, d = k.shape[1:]
    pool = torch.full((nblk, hkv, 17 * d), 0xFF, dtype=torch.uint8, device=DEV)
    ak.kv_scatter_mx4(pool, dev_bits(k), dev_bits(v), torch.from_numpy(np.asarray(slots, dtype=np.int32)).to(DEV))
    torch.cuda.synchronize()
    return pool


def finite_bytes_equal(pool, want, k, v, slots):
    """Pool bytes equal, but for the codes of groups that stand for NaN."""
    got = pool.cpu().numpy()
    kg, vg = omx.gather(got, slots)
    assert np.array_equal(kg, omx.stored(k), equal_nan=True) and np.array_equal(vg, omx.stored(v), equal_nan=True)
    if np.isfinite(kg).all() and np.isfinite(vg).all():
        assert np.array_equal(got, want)


@pytest.mark.parametrize("d,hkv,n,kind", [(64, 2, 1, "normal"), (128, 1, 1, "any"), (64, 3, 37, "normal"),
                                          (128, 8, 65, "normal"), (128, 2, 700, "any"), (64, 5, 700, "any")])
def test_scatter_and_gather(d, hkv, n, kind):
    print_case(f"mx4 store d={d} hkv={hkv} n={n} {kind}")
    rng = np.random.default_rng(n * 7 + d)
    nblk = (n + 15) // 16 + 3
    slots = rng.permutation(nblk * 16)[:n].astype(np.int32)
    k, v = random_rows(n, hkv, d, rng, kind), random_rows(n, hkv, d, rng, kind)
    given = slots.copy()
    given[n // 2 + 1::50] = [-1, nblk * 16, 1 << 30, -(1 << 31)][n % 4]       # slots outside the pool are skipped
    pool = store(k, v, given, nblk)
    keep = (given >= 0) & (given < nblk * 16)
    want = omx.new_pool(nblk, hkv, d)
    omx.scatter(want, k[keep], v[keep], given[keep])
    finite_bytes_equal(pool, want, k[keep], v[keep], given[keep])
    ko, vo = (torch.full((n, hkv, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ak.kv_gather_mx4(pool, torch.from_numpy(given).to(DEV), ko, vo)
    torch.cuda.synchronize()
    for got, rows in ((ko, k), (vo, v)):
        w = np.where(keep[:, None, None], omx.stored(rows), 0.0)
        assert np.array_equal(bf16_to_f64(bits(got)), w, equal_nan=True)


@pytest.mark.parametrize("d,hkv,n,start", [(128, 8, 1000, 5), (64, 2, 300, 0), (128, 2, 2049, 8), (64, 3, 1500, 3),
                                           (128, 1, 1025, 15), (64, 2, 3001, 0)])
def test_scatter_of_whole_requests(d, hkv, n, start):
    """Prefill-shaped slots: consecutive slots of scattered blocks."""
    print_case(f"mx4 store in runs d={d} hkv={hkv} n={n} start={start}")
    rng = np.random.default_rng(n + d)
    nblk = (n + start + 15) // 16 + 4
    table = rng.permutation(nblk)
    j = np.arange(n) + start
    slots = (table[j // 16] * 16 + j % 16).astype(np.int32)
    slots[rng.integers(0, n, n // 200)] = -1
    k, v = random_rows(n, hkv, d, rng, "normal"), random_rows(n, hkv, d, rng, "normal")
    pool = store(k, v, slots, nblk)
    keep = slots >= 0
    want = omx.new_pool(nblk, hkv, d)
    omx.scatter(want, k[keep], v[keep], slots[keep])
    assert np.array_equal(pool.cpu().numpy(), want)
    ko, vo = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ak.kv_gather_mx4(pool, torch.from_numpy(slots).to(DEV), ko, vo)
    torch.cuda.synchronize()
    for got, rows in ((ko, k), (vo, v)):
        assert np.array_equal(bf16_to_f64(bits(got)), np.where(keep[:, None, None], omx.stored(rows), 0.0))


@pytest.mark.parametrize("d", [64, 128])
def test_unrelated_slots_in_bulk(d):
    """More tokens than a small batch has, none beside another, and some in pairs."""
    print_case(f"mx4 store of unrelated slots d={d}")
    rng = np.random.default_rng(d)
    n, hkv = 1300, 2
    slots = rng.permutation(90 * 16)[:n].astype(np.int32)
    slots[100:108] = np.arange(8) + 90 * 16                 # one whole half block among them
    slots[201:217] = np.arange(16) + 91 * 16                # a block
    k, v = random_rows(n, hkv, d, rng, "any"), random_rows(n, hkv, d, rng, "normal")
    pool = store(k, v, slots, 92)
    want = omx.new_pool(92, hkv, d)
    omx.scatter(want, k, v, slots)
    finite_bytes_equal(pool, want, k, v, slots)
    ko, vo = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ak.kv_gather_mx4(pool, torch.from_numpy(slots).to(DEV), ko, vo)
    torch.cuda.synchronize()
    for got, rows in ((ko, k), (vo, v)):
        assert np.array_equal(bf16_to_f64(bits(got)), omx.stored(rows), equal_nan=True)


@pytest.mark.parametrize("d,hkv,n", [(128, 8, 4097), (128, 8, 4203), (64, 16, 4109), (64, 33, 2011), (128, 3, 10931)])
def test_many_rows(d, hkv, n):
    """Enough to be stored and read 8 tokens at a time: whole requests from any first slot, then unrelated slots with a
    whole half block among them, some of each outside the pool."""
    print_case(f"mx4 many rows d={d} hkv={hkv} n={n}")
    rng = np.random.default_rng(n)
    nblk = n // 16 + 30
    table = rng.permutation(nblk)
    m = n * 3 // 4
    at, slots = 0, []
    while sum(map(len, slots)) < m:                            # requests that start in a new block each
        j = np.arange(int(rng.integers(1, 900)))
        slots.append(table[at + j // 16] * 16 + j % 16)
        at += len(j) // 16 + 1
        if at > nblk - 60 - (n - m) // 16:
            break
    slots = np.concatenate(slots)[:m]
    rest = rng.permutation(np.concatenate([table[at + 2:] * 16 + i for i in range(16)]))
    slots = np.concatenate([slots, table[at + 1] * 16 + 8 + np.arange(8), rest])[:n].astype(np.int32)
    n = len(slots)
    assert n * hkv * d > 1 << 22 and len(set(slots.tolist())) == n
    k, v = random_rows(n, hkv, d, rng, "normal"), random_rows(n, hkv, d, rng, "normal")
    given = slots.copy()
    given[rng.integers(0, n, n // 300)] = -1
    given[rng.integers(0, n, n // 700)] = nblk * 16
    pool = store(k, v, given, nblk)
    keep = (given >= 0) & (given < nblk * 16)
    want = omx.new_pool(nblk, hkv, d)
    omx.scatter(want, k[keep], v[keep], given[keep])
    assert np.array_equal(pool.cpu().numpy(), want)
    ko, vo = (torch.full((n, hkv, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ak.kv_gather_mx4(pool, torch.from_numpy(given).to(DEV), ko, vo)
    torch.cuda.synchronize()
    for got, rows in ((ko, k), (vo, v)):
        assert np.array_equal(bf16_to_f64(bits(got)), np.where(keep[:, None, None], omx.stored(rows), 0.0))


def test_every_code_rounds_as_defined():
    """Every bf16 magnitude under each of several scales, beside a value that sets the scale."""
    print_case("mx4 rounding, all magnitudes")
    m = np.arange(0x7F80, dtype=np.uint16).reshape(-1, 16)
    rows = []
    for top in (0x0000, 0x0100, 0x3F80, 0x40E0, 0x40E1, 0x7E60, 0x7F7F):
        g = np.where(m <= top, m, 0)
        g = np.concatenate([g, np.full((len(g), 1), top, np.uint16), g[:, :15] | 0x8000], axis=1)
        rows.append(g)
    x = np.concatenate(rows).astype(np.uint16)
    x = x[: len(x) // 2 * 2].reshape(-1, 1, 64)
    n = len(x)
    slots = np.arange(n, dtype=np.int32)
    pool = store(x, x[::-1].copy(), slots, (n + 15) // 16)
    k, v = omx.gather(pool.cpu().numpy(), slots)
    assert np.array_equal(k, omx.stored(x)) and np.array_equal(v, omx.stored(x[::-1]))
