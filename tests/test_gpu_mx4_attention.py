"""Attention over the 4-bit cache on the GPU, and the log-sum-exp that both attention calls give,
against 64 bits on the values that the cache stands for."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import bits, print_case  # noqa: E402
from tests.mx4_helpers import DEV, attend, check_out, i32, make_batch, reference  # noqa: E402
from tests.test_gpu_parity import SWEEP  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


MORE = [
    ([(1, 0), (5, 5), (40, 39)], 64, 8, 128),             # a request without a new token
    ([(31, 30), (32, 31), (33, 32), (1, 0)], 5, 1, 64),   # the end of a chunk of 32 keys
    ([(3000, 2996), (190, 187), (700, 660)], 16, 4, 64),  # column counts on both sides of 16 and 32
    ([(2300, 2290), (600, 597), (1200, 1199)], 32, 4, 128),
    ([(2100, 1000), (900, 100)], 64, 8, 128),
    ([(1500, 0)], 2, 2, 128),
]


@pytest.mark.parametrize("num_cus", [256, 100000, 24])
@pytest.mark.parametrize("case", range(len(SWEEP) + len(MORE)))
def test_attention_sweep(case, num_cus):
    reqs, hq, hkv, d = (SWEEP + MORE)[case]
    print_case(f"mx4 attention {reqs} hq={hq} hkv={hkv} d={d} num_cus={num_cus}")
    b = make_batch(reqs, hq, hkv, d, seed=1300 + case)
    out, lse, _ = attend(b, num_cus)
    check_out(b, out, lse, reference(b), f"case {case}")


@pytest.mark.parametrize("case", [2, 5, 8, 9, 16, 18, 20])
@pytest.mark.parametrize("num_cus", [256, 100000])
def test_lse_of_the_bf16_attention(case, num_cus):
    """prefill_attention with and without lse: the same bits out, and the sums within tolerance."""
    reqs, hq, hkv, d = SWEEP[case]
    print_case(f"bf16 lse {reqs} hq={hq} hkv={hkv} d={d} num_cus={num_cus}")
    b = make_batch(reqs, hq, hkv, d, seed=1400 + case, fmt="bf16")
    out, lse, _ = attend(b, num_cus)
    plain, _, _ = attend(b, num_cus, lse=False)
    assert torch.equal(out, plain)
    check_out(b, out, lse, reference(b), f"case {case}")


KINDS = {
    "narrow": ([(300, 292), (700, 697), (45, 29)], 8, 2, 128),
    "decode": ([(130, 129), (2051, 2050), (17, 16)], 16, 4, 64),
    "wide": ([(700, 400), (130, 0)], 8, 1, 128),
    "wide64": ([(400, 100), (70, 0)], 16, 4, 64),
}


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("num_cus", [256, 100000])
def test_scores_that_grow_fall_and_jump(kind, num_cus):
    """Keys scaled by their position: the running maximum moves late, early, and by thousands."""
    reqs, hq, hkv, d = KINDS[kind]
    pos = torch.from_numpy(np.concatenate([np.arange(L) for L, _ in reqs])).to(DEV)
    gains = {"grow": 0.1 + pos / 100.0, "fall": 12.0 / (1 + pos / 20.0), "jump": torch.where(pos % 97 == 40, 60.0, 0.2)}
    for name, gain in gains.items():
        print_case(f"mx4 {kind} num_cus={num_cus} scores {name}")
        b = make_batch(reqs, hq, hkv, d, seed=50, k_edit=lambda k: k.mul_(gain[:, None, None]))
        out, lse, _ = attend(b, num_cus)
        check_out(b, out, lse, reference(b), name)


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("num_cus", [256, 100000])
def test_nan_and_infinity_reach_only_who_sees_them(kind, num_cus):
    """A NaN or infinite group of a key's V makes those dimensions NaN for the columns that see the key; one of
    its K makes their rows NaN.  Earlier columns are as without it."""
    reqs, hq, hkv, d = KINDS[kind]
    at = np.concatenate([[0], np.cumsum([L for L, _ in reqs])])
    for name in ("v new", "v old", "k new"):
        print_case(f"mx4 {kind} num_cus={num_cus} non-finite {name}")

        def edit(x):
            for r, (L, P) in enumerate(reqs):
                j = L - 1 if L - P < 3 else (P + L) // 2
                if name == "v old":
                    j = P // 2
                x[at[r] + j, 0, 3] = float("nan") if r % 2 else float("inf")
                if name == "v new" and L - P > 2:
                    x[at[r] + L - 1, hkv - 1, d - 1] = float("nan")

        b = make_batch(reqs, hq, hkv, d, seed=60, **{("k_edit" if name[0] == "k" else "v_edit"): edit})
        out, lse, _ = attend(b, num_cus)
        ref = reference(b)
        if name[0] == "k":        # NaN scores: the whole row, in the reference too
            for r, (L, P) in enumerate(reqs):
                j = L - 1 if L - P < 3 else (P + L) // 2
                ref[r][0][max(j - P, 0):, : hq // hkv] = float("nan")
                ref[r][2][max(j - P, 0):, : hq // hkv] = float("nan")
        check_out(b, out, lse, ref, name)


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_views_at_any_bf16_address(kind):
    reqs, hq, hkv, d = KINDS[kind]
    print_case(f"mx4 views {kind}")
    b = make_batch(reqs, hq, hkv, d, seed=70)
    n = b["q"].numel()
    for num_cus in (256, 100000):
        want, _, _ = attend(b, num_cus)
        for shift in (1, 4):
            q = torch.empty(n + 8, dtype=torch.bfloat16, device=DEV)[shift:shift + n].view_as(b["q"]).copy_(b["q"])
            store = torch.full((n + 16,), 7.0, dtype=torch.bfloat16, device=DEV)
            out, _, _ = attend(b, num_cus, q=q, out=store[shift:shift + n].view_as(q))
            assert torch.equal(out, want)
            assert (store[:shift] == 7).all() and (store[shift + n:] == 7).all()


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_bad_block_table_entries_stay_in_the_pool(kind):
    """Entries outside the pool read block 0: only the request that has them is off."""
    reqs, hq, hkv, d = KINDS[kind]
    print_case(f"mx4 bad table entries {kind}")
    b = make_batch(reqs, hq, hkv, d, seed=80)
    want, _, _ = attend(b)
    bt = b["bt"].copy()
    bt[0, 1] = len(b["pool"][0])
    bt[0, 2] = -7
    out, _, _ = attend(b, bt=bt)
    n = int(b["cu"][1])
    assert torch.equal(out[n:], want[n:])


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_repeated_calls_give_the_same_bits(kind):
    reqs, hq, hkv, d = KINDS[kind]
    print_case(f"mx4 repeated {kind}")
    b = make_batch(reqs, hq, hkv, d, seed=90)
    for num_cus in (256, 100000):
        first = attend(b, num_cus)
        again = attend(b, num_cus)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_offsets_past_32_bits():
    """A pool of 4.6 GB: blocks on both sides of 2^32 bytes."""
    print_case("mx4 large pool")
    reqs, hq, hkv, d = [(300, 299), (400, 100)], 8, 8, 128
    small = make_batch(reqs, hq, hkv, d, seed=95)
    want, _, _ = attend(small)
    nb = 265000
    big = torch.empty((nb, hkv, 17 * d), dtype=torch.uint8, device=DEV)
    move = np.random.default_rng(1).permutation(len(small["pool"][0]))
    to = np.where(move % 2 == 0, move, nb - 1 - move)
    big[i32(to).long()] = small["pool"][0]
    b = dict(small, pool=(big,), bt=np.where(small["bt"] >= 0, to[small["bt"]], -1).astype(np.int32))
    out, _, _ = attend(b)
    assert torch.equal(out, want)
    rows = torch.from_numpy(small["slots"]).to(DEV)
    kv = [torch.empty(len(rows), hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    ak.kv_gather_mx4(small["pool"][0], rows, kv[0], kv[1])
    far = i32(to[small["slots"] // 16] * 16 + small["slots"] % 16)
    ak.kv_gather_mx4(big, far, kv[2], kv[3])
    torch.cuda.synchronize()
    assert torch.equal(kv[0], kv[2]) and torch.equal(kv[1], kv[3])


def test_nothing_to_do():
    b = make_batch([(20, 20), (7, 7)], 8, 2, 64, seed=3)
    out, _, ap = attend(b)
    assert ap.n_work == 0 and out.numel() == 0


def test_outputs_of_idle_rows_stay():
    """Rows of q behind the batch's last request are not written."""
    b = make_batch([(100, 98), (50, 49)], 8, 2, 128, seed=4)
    q = torch.cat([b["q"], b["q"]])
    out, lse, _ = attend(b, q=q)
    n = len(b["q"])
    assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all() and torch.isfinite(out[:n]).all()


@pytest.mark.parametrize("num_cus", [64, 256, 100000])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("reqs", [[(567, 88)], [(753, 69), (747, 283)], [(1918, 195)]])
def test_block_0_of_nobody_reaches_nobody(reqs, d, num_cus):
    """Tiles cut inside the keys that only some of their columns see, and a block 0 of NaN that no table names:
    what is read of it past a cut must not count."""
    for heads in (2, 8):
        print_case(f"mx4 block 0 of NaN {reqs} heads={heads} d={d} num_cus={num_cus}")
        b = make_batch(reqs, heads, heads, d, seed=110)
        b["pool"] = (torch.cat([torch.full_like(b["pool"][0][:1], 0xFF), b["pool"][0]]),)
        b["bt"] = np.where(b["bt"] >= 0, b["bt"] + 1, -1).astype(np.int32)
        out, lse, _ = attend(b, num_cus)
        check_out(b, out, lse, reference(b), f"heads {heads}")
