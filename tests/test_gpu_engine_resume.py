"""Sessions that were cut go on through the engine's own producer: their new tokens are rotated for the positions that
they have in the whole prompt, and stored and attended behind the tokens that were kept."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2606_21238_amd as ak  # noqa: E402
from oracle import mx4 as omx  # noqa: E402
from oracle import qkv as oqkv  # noqa: E402
from oracle.attention import bf16_to_f64  # noqa: E402
from paper_2606_21238_amd.engine import PrefillEngine  # noqa: E402
from tests.gpu_helpers import bits, print_case  # noqa: E402
from tests.mx4_helpers import DEV, check_out, i32, reference  # noqa: E402
from tests.test_gpu_qkv import THETA, check, randn_bf16  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ak.lib()


def produced(eng, db, x, w, true_lens):
    """project(), checked against the oracle's producer at the true positions."""
    T = db.n_tokens
    q = torch.empty(T, eng.hq, eng.d, dtype=torch.bfloat16, device=DEV)
    k, v = (torch.empty(T, eng.hkv, eng.d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    eng.project(db, x, w, q, k, v, THETA)
    torch.cuda.synchronize()
    cu = db.plan.cu_q
    pos = oqkv.token_positions(cu, np.array(true_lens, np.int32))
    refbits, ref = oqkv.qkv_rope(bits(x), bits(w), pos, eng.hq, eng.hkv, eng.d, THETA)
    check(dict(q=q, k=k, v=v, ref=ref, refbits=refbits, y=bf16_to_f64(oqkv.f64_to_bf16_bits(oqkv.project(bits(x), bits(w)))),
               acc=x.shape[1] * 2.0 ** -24 * (np.abs(bf16_to_f64(bits(x))) @ np.abs(bf16_to_f64(bits(w))).T)),
          eng.hq, eng.hkv, eng.d)
    return q, k, v


@pytest.mark.parametrize("fmt,hq,hkv,d,hidden", [("mx4", 8, 2, 128, 256), ("bf16", 8, 2, 128, 256), ("bf16", 4, 4, 64, 128)])
def test_cut_sessions_go_on_at_their_true_positions(fmt, hq, hkv, d, hidden):
    print_case(f"cut sessions through the producer, {fmt} {hq}/{hkv} heads of {d}")
    lens, keep, new = [300, 70, 20], 32, [[1, 1, 1], [3, 1, 18]]
    n, nb = len(lens), 4
    rng = np.random.default_rng(5)
    eng = PrefillEngine(hq, hkv, d, 40, 48, 4, kv_format=fmt, private_blocks=n * nb)
    w = randn_bf16(((hq + 2 * hkv) * d, hidden), 1, hidden ** -0.5)
    db = eng.prepare([rng.integers(0, 1000, L, dtype=np.int32) for L in lens])
    q, k, v = produced(eng, db, randn_bf16((sum(lens), hidden), 2), w, lens)
    eng.scatter(db, k, v)
    out, lse = torch.empty_like(q), torch.empty(sum(lens), hq, device=DEV)
    weights = torch.zeros(n, hkv, max(lens), device=DEV)
    eng.attention(db, q, out, lse=lse)
    eng.attention_weights(db, q, lse, weights)
    tables = eng.num_phys + rng.permutation(n * nb).reshape(n, nb).astype(np.int32)
    kept, _ = eng.evict(db, weights, keep, tables, n_first=2, n_recent=8)
    eng.release()

    def value(x):
        return torch.from_numpy(omx.stored(bits(x))).to(DEV) if fmt == "mx4" else x.double()

    held = [min(L, keep) for L in lens]
    K, V = [], []                                      # what each session's blocks hold, 64 bits
    for r in range(n):
        at = torch.tensor(lens[:r], dtype=torch.int64).sum().to(DEV) + kept[r, :, : held[r]].long()     # [Hkv, held]
        head = torch.arange(hkv, device=DEV)[:, None]
        K.append(value(k)[at, head].transpose(0, 1).contiguous())
        V.append(value(v)[at, head].transpose(0, 1).contiguous())
    true = list(lens)
    for step, s in enumerate(new):
        true = [t + x for t, x in zip(true, s)]
        db = eng.resume(tables, held, s, true)
        x = randn_bf16((sum(s), hidden), 10 + step)
        q, k, v = produced(eng, db, x, w, true)
        # the positions matter: at the shortened lengths, other keys
        short = [torch.empty_like(t) for t in (q, k, v)]
        ak.qkv_rope(x, w, db.cu_q, db.seq_lens, hq, hkv, THETA, *short, torch.empty(4 * sum(s) * d, dtype=torch.uint8, device=DEV))
        rows = slice(int(db.plan.cu_q[0]), int(db.plan.cu_q[1]))                # of a request that was shortened
        assert not torch.equal(short[1][rows], k[rows]) and torch.equal(short[2], v)
        if fmt == "bf16" and step == 1:                # the producer that stores K and V itself
            again = torch.empty_like(q)
            eng.project_to_pool(db, x, w, again, THETA)
            torch.cuda.synchronize()
            assert torch.equal(again, q)
        else:
            eng.scatter(db, k, v)
        out, lse = torch.empty_like(q), torch.empty(sum(s), hq, device=DEV)
        eng.attention(db, q, out, lse=lse)
        torch.cuda.synchronize()
        cu = db.plan.cu_q
        K = [torch.cat([K[r], value(k[cu[r]:cu[r + 1]])]) for r in range(n)]
        V = [torch.cat([V[r], value(v[cu[r]:cu[r + 1]])]) for r in range(n)]
        b = dict(hq=hq, hkv=hkv, d=d, q=q, cu=cu, k=K, v=V, scale=d ** -0.5, reqs=[(len(x), h) for x, h in zip(K, held)])
        check_out(b, out, lse, reference(b), f"step {step}")
        held = [h + x for h, x in zip(held, s)]
