"""Attention weights where scores are infinite: a key that every column scores with minus infinity receives
exp(-inf) = 0, whichever kernel takes the request and however many of a tile's columns there are."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import DEV, i32, make_batch, reference  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


# (requests, hq, hkv, d): 1, 2, 4, 5, 8 columns of a tile of 32; 12, 20, 32 and 40 of them; many columns
CASES = [
    ([(90, 89), (40, 39)], 2, 2, 64),
    ([(90, 89)], 2, 1, 128),
    ([(300, 299), (40, 39), (77, 76)], 8, 2, 128),
    ([(90, 89), (200, 199)], 5, 1, 64),
    ([(90, 89)], 16, 2, 128),
    ([(90, 87)], 4, 1, 64),
    ([(90, 86)], 5, 1, 128),
    ([(90, 82)], 4, 1, 128),
    ([(90, 82), (40, 39), (41, 40)], 5, 1, 64),
    ([(400, 200), (90, 40)], 8, 2, 128),
    ([(400, 263)], 5, 1, 64),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_keys_at_minus_and_plus_infinity(case):
    reqs, hq, hkv, d = CASES[case]
    print_case(f"weights of infinite keys {reqs} hq={hq} hkv={hkv} d={d}")
    b = make_batch(reqs, hq, hkv, d, seed=300 + case, fmt="bf16")
    b["q"][..., 5] = b["q"][..., 5].abs() + 0.5           # every column scores dimension 5 with a positive number
    low, high = [(0, 7), (len(reqs) - 1, 20)], (0, 33)    # (request, key)
    ref = reference(b)
    lse = torch.cat([r[2] for r in ref]).float()
    longest = max(L for L, _ in reqs)

    def weigh(accumulate):
        w = torch.full((len(reqs), hkv, longest), 2.0, device=DEV)
        ak.attention_weights(b["pool"][0], b["q"], lse, w, i32(b["bt"]), i32(b["cu"]), i32(b["seq"]), b["scale"],
                             accumulate=accumulate)
        torch.cuda.synchronize()
        return w

    clean = {a: weigh(a) for a in (True, False)}
    pool = b["pool"][0].view(torch.bfloat16)
    for r, key in low + [high]:
        pool[int(b["bt"][r, key // 16]), :, key % 16, 5] = float("inf") if (r, key) == high else -float("inf")
    for accumulate in (True, False):
        want = clean[accumulate].clone()
        for r, key in low:
            want[r, :, key] = 2.0 if accumulate else 0.0
        want[high[0], :, high[1]] = float("inf")          # lse is given and finite
        got = weigh(accumulate)
        assert torch.equal(got, want), f"other weights at {(got != want).nonzero()[:8].tolist()}"
