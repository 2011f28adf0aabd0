"""Batches over either pool, and their attention in 64 bits, for the GPU tests of the 4-bit cache and of
eviction (imported by tests only)."""

from __future__ import annotations

import numpy as np
import torch

import paper_2606_21238_amd as ak
from oracle import mx4 as omx
from tests.gpu_helpers import bits
from tests.test_gpu_parity import randn_bf16

DEV = "cuda"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def make_batch(reqs, hq, hkv, d, seed, fmt="mx4", k_edit=None, v_edit=None, extra_blocks=3):
    """reqs: [(L, P)].  Blocks at random places of one pool (every byte of it 0xFF before), K and V of all
    tokens written by the library.  k_edit / v_edit change the bf16 rows [sum L, Hkv, D] first."""
    rng = np.random.default_rng(seed)
    nb = [(L + 15) // 16 for L, _ in reqs]
    nphys = sum(nb) + extra_blocks
    perm, o = rng.permutation(nphys).astype(np.int32), 0
    bt = np.full((len(reqs), max(nb + [1])), -1, dtype=np.int32)
    for r, n in enumerate(nb):
        bt[r, :n] = perm[o:o + n]
        o += n
    Ls, Ss = [L for L, _ in reqs], [L - P for L, P in reqs]
    cu = np.concatenate([[0], np.cumsum(Ss)]).astype(np.int32)
    k, v = randn_bf16((sum(Ls), hkv, d), seed + 1), randn_bf16((sum(Ls), hkv, d), seed + 2)
    for x, edit in ((k, k_edit), (v, v_edit)):
        if edit is not None:
            edit(x)
    slots = np.concatenate([bt[r, np.arange(L) // 16] * 16 + np.arange(L) % 16 for r, L in enumerate(Ls)] + [[]])
    b = dict(fmt=fmt, reqs=reqs, hq=hq, hkv=hkv, d=d, bt=bt, cu=cu, seq=np.array(Ls, dtype=np.int32), free=perm[o:],
             q=randn_bf16((sum(Ss), hq, d), seed + 3), slots=slots.astype(np.int32), scale=d ** -0.5)
    if fmt == "mx4":
        b["pool"] = (torch.full((nphys, hkv, 17 * d), 0xFF, dtype=torch.uint8, device=DEV),)
        ak.kv_scatter_mx4(*b["pool"], k, v, i32(slots))
        kv = [torch.from_numpy(omx.stored(bits(x))).to(DEV) for x in (k, v)]
    else:
        b["pool"] = (torch.full((nphys, hkv, 16, d), -1, dtype=torch.int16, device=DEV),
                     torch.full((nphys, hkv, d, 16), -1, dtype=torch.int16, device=DEV))
        ak.kv_scatter(*b["pool"], k, v, i32(slots))
        kv = [k.double(), v.double()]
    at = np.concatenate([[0], np.cumsum(Ls)])
    b["k"], b["v"] = ([x[at[r]:at[r + 1]] for r in range(len(reqs))] for x in kv)
    return b


def attend(b, num_cus=256, lse=True, q=None, out=None, plan=None, bt=None, stream=None):
    """(out, lse, plan) of the library on a batch."""
    ap = plan or ak.attention_plan(b["cu"], b["seq"], b["hq"], b["hkv"], b["d"], num_cus)
    q = b["q"] if q is None else q
    out = torch.full_like(q, float("nan")) if out is None else out
    lse = torch.full(q.shape[:2], float("nan"), device=DEV) if lse else None
    ws = torch.full((max(ap.ws_bytes, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    f = ak.prefill_attention_mx4 if b["fmt"] == "mx4" else ak.prefill_attention
    f(*b["pool"], q, out, i32(b["bt"] if bt is None else bt), i32(b["cu"]), i32(b["seq"]), i32(ap.work), ap.n_work,
      ap.n_combine, ap.tile_cols, b["scale"], ws, ap.ws_bytes, stream=stream, lse=lse)
    torch.cuda.synchronize()
    return out, lse, ap


def reference(b, weights=False):
    """Per request, in 64 bits: out, its tolerance, lse, its tolerance [S, Hq(, D)], and the sum over a KV
    head's columns of the attention weights [Hkv, L].

    A probability is rounded to bf16 once and an output once: |out - ref| <= 2^-8 sum_j w_j |v_j| +
    2^-8 |ref|, of which the second is taken of the first's end.  fp32 adds the rest: a score's products
    are exact and their sum is off by at most D 2^-24 of the products' magnitudes (T, scaled), a sum of n
    weights by n 2^-24 of it, and an exponential or logarithm by 2^-22.  Exponentials below 2^-126, the
    smallest normal number, count as zero: up to 2^-125 max|v| for each of L keys."""
    g, res = b["hq"] // b["hkv"], []
    for r, (L, P) in enumerate(b["reqs"]):
        S, q = L - P, b["q"][b["cu"][r]:b["cu"][r + 1]].double()
        out = torch.zeros(S, b["hq"], b["d"], dtype=torch.float64, device=DEV)
        otol, lse, ltol = torch.zeros_like(out), out[..., 0].clone(), out[..., 0].clone()
        w = torch.zeros(b["hkv"], L, dtype=torch.float64, device=DEV)
        hidden = torch.arange(L, device=DEV)[None, :] > torch.arange(P, L, device=DEV)[:, None]
        for h in range(b["hq"]):
            if S == 0:
                break
            k, v = b["k"][r][:, h // g].contiguous(), b["v"][r][:, h // g].contiguous()
            kt = k.t().contiguous()
            s = (q[:, h].contiguous() @ kt * b["scale"]).masked_fill(hidden, -torch.inf)
            t = (q[:, h].abs().contiguous() @ kt.abs() * b["scale"]).masked_fill(hidden, 0).nan_to_num(nan=0.0).amax(1)
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - l[:, None])
            # a hidden key's value counts for nothing, whatever it is
            bad = torch.isnan(v) | torch.isinf(v)
            vz = torch.where(bad, 0.0, v)
            out[:, h] = p @ vz
            mag = p @ vz.abs()
            if bool(bad.any()):
                out[:, h] = torch.where((~hidden).double() @ bad.double() > 0, torch.nan, out[:, h])
            fp32 = 2.0 ** -24 * (b["d"] * t + L) + 2.0 ** -22
            otol[:, h] = 2.0 ** -8 * (mag + (out[:, h].abs() + 2.0 ** -8 * mag)) + 2 * fp32[:, None] * mag + L * 2.0 ** -125 * vz.abs().max()
            lse[:, h], ltol[:, h] = l, fp32 + 2.0 ** -22 * l.abs()
            w[h // g] += p.sum(0)
        res.append((out, otol, lse, ltol, w))
    return res


def check_out(b, out, lse, ref, what=""):
    for r in range(len(b["reqs"])):
        rows = slice(int(b["cu"][r]), int(b["cu"][r + 1]))
        o, otol, l, ltol, _ = ref[r]
        for name, got, want, tol in (("out", out, o, otol), ("lse", lse, l, ltol)):
            if got is None or want.numel() == 0:
                continue
            x = got[rows].double()
            assert torch.equal(torch.isnan(x), torch.isnan(want)), f"{what} request {r}: NaN in other places of {name}"
            err = torch.where(torch.isnan(want), 0.0, (x - want).abs() - tol)
            assert float(err.max()) <= 0, f"{what} request {r}: {name} {float(err.max()):.3g} over its tolerance"
