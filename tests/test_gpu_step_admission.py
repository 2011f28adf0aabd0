"""Steps beside the block cache: a batch of the cache that steps go on with keeps the cache from planning another, so a server that
admits requests while steps run holds the shared prefix in private blocks."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.gpu_helpers import print_case  # noqa: E402
from tests.mx4_helpers import DEV, check_out, reference  # noqa: E402
from tests.test_gpu_parity import randn_bf16  # noqa: E402

HQ, HKV, D, DOC = 8, 2, 64, 320


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def rows_of(eng, tables, lens):
    kr = eng.k_pool.view(torch.bfloat16).permute(0, 2, 1, 3).reshape(-1, HKV, D)
    vr = eng.v_pool.view(torch.bfloat16).permute(0, 3, 1, 2).reshape(-1, HKV, D)
    at = [torch.from_numpy(np.asarray(t)[np.arange(L) // 16].astype(np.int64) * 16 + np.arange(L) % 16).to(DEV) for t, L in zip(tables, lens)]
    return dict(hq=HQ, hkv=HKV, d=D, scale=D ** -0.5, k=[kr[x].double() for x in at], v=[vr[x].double() for x in at])


def step(eng, sb, held, seed, what):
    """One token more for every request; the attention against 64 bits."""
    n = len(held)
    k, v, q = randn_bf16((n, HKV, D), seed), randn_bf16((n, HKV, D), seed + 1), randn_bf16((n, HQ, D), seed + 2)
    out = torch.empty_like(q)
    eng.advance(sb, torch.ones(n, dtype=torch.int32, device=DEV))
    eng.scatter(sb, k, v)
    eng.shared_attention(sb, q, out)
    held = held + 1
    assert np.array_equal(sb.seq_lens.cpu().numpy(), held)
    b = dict(rows_of(eng, sb.block_tables.cpu().numpy(), held), q=q, cu=np.arange(n + 1), reqs=[(int(L), int(L) - 1) for L in held])
    check_out(b, out, None, reference(b), what)
    return held


def test_requests_are_admitted_while_steps_run():
    print_case("admission beside steps")
    rng = np.random.default_rng(3)
    private = np.arange(24, 24 + 60)
    eng = PrefillEngine(HQ, HKV, D, 20, 24, 4, private_blocks=len(private))
    # the document, through the cache once; then all of its tokens into private blocks, and the batch released
    db = eng.prepare([rng.integers(0, 1000, DOC).astype(np.int32)])
    k, v = randn_bf16((DOC, HKV, D), 1), randn_bf16((DOC, HKV, D), 2)
    eng.scatter(db, k, v)
    doc = private[:DOC // 16]
    kept, _ = eng.evict(db, torch.zeros(1, HKV, DOC, device=DEV), DOC, doc[None])
    eng.release()
    assert (kept[0].cpu().numpy() == np.arange(DOC)).all()
    b = rows_of(eng, [doc], [DOC])
    assert torch.equal(b["k"][0], k.double()) and torch.equal(b["v"][0], v.double())

    def admit(own, blocks, seed):
        """A prompt behind the document: its own tokens are prefilled by resume()."""
        table = np.concatenate([doc, blocks])
        db = eng.resume(table[None], [DOC], [own], [DOC + own])
        q, out = randn_bf16((own, HQ, D), seed), torch.empty(own, HQ, D, dtype=torch.bfloat16, device=DEV)
        eng.scatter(db, randn_bf16((own, HKV, D), seed + 1), randn_bf16((own, HKV, D), seed + 2))
        eng.attention(db, q, out)
        b = dict(rows_of(eng, [table], [DOC + own]), q=q, cu=np.array([0, own]), reqs=[(DOC + own, DOC)])
        check_out(b, out, None, reference(b), "admitted")
        return table

    tables = [admit(9, private[20:23], 10), admit(30, private[23:26], 20)]
    held, free = np.array([DOC + 9, DOC + 30]), private[32:]
    sb = eng.step_batch(np.stack(tables), held, [2], [DOC], max_tokens=2, free_blocks=free)
    for i in range(12):
        held = step(eng, sb, held, 100 + 3 * i, f"two requests, step {i}")
        # a batch of other prompts through the cache, more of them than it holds: no block of the steps is touched
        db = eng.prepare([rng.integers(0, 1000, 130).astype(np.int32) for _ in range(2)])
        eng.scatter(db, randn_bf16((db.n_tokens, HKV, D), 7), randn_bf16((db.n_tokens, HKV, D), 8))
        eng.release()
    new = admit(5, private[26:29], 30)
    left = int(sb.free_count.cpu())
    now, width = sb.block_tables.cpu().numpy(), len(new)
    sb = eng.step_batch(np.concatenate([now[:, :width], new[None]]), np.append(held, DOC + 5), [3], [DOC], max_tokens=3, free_blocks=free[:left])
    held = np.append(held, DOC + 5)
    for i in range(4):
        held = step(eng, sb, held, 200 + 3 * i, f"three requests, step {i}")


def test_a_cache_batch_under_steps_is_the_only_one():
    """The cache refuses the next batch, and the steps go on; after their end it plans again."""
    print_case("cache batch under steps")
    rng = np.random.default_rng(4)
    doc = rng.integers(0, 1000, DOC)
    eng = PrefillEngine(HQ, HKV, D, 48, 56, 4, private_blocks=4)
    db = eng.prepare([np.concatenate([doc, rng.integers(0, 1000, m)]).astype(np.int32) for m in (9, 30)])
    eng.scatter(db, randn_bf16((db.n_tokens, HKV, D), 1), randn_bf16((db.n_tokens, HKV, D), 2))
    tables = np.concatenate([db.plan.block_tables, np.full((2, 3), -1, np.int32)], 1)
    held = db.plan.seq_lens.astype(int)
    sb = eng.step_batch(tables, held, [2], [DOC], max_tokens=2, free_blocks=np.arange(56, 60))
    for i in range(3):
        with pytest.raises(ak.ArckvError, match="not released"):
            eng.prepare([rng.integers(0, 1000, 40).astype(np.int32)])
        held = step(eng, sb, held, 10 + 3 * i, f"step {i}")
    eng.release()
    assert eng.prepare([rng.integers(0, 1000, 40).astype(np.int32)]).n_tokens == 40
    eng.release()
