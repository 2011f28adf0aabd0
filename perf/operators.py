"""Cases of the 4-bit KV cache and of eviction by attention weight.

A serving program holds a ``PrefillEngine``; with ``kv_format="mx4"`` its pool keeps K and V in
4 bits.  Timed is what such a program does layer by layer: storing a batch's K/V rows in the 4-bit
pool and reading them back (``store``), attention over that pool (``attn``), the attention weight
that every cached token has received, from either pool (``weights``), and cutting sessions down to
their heaviest tokens (``evict``).  Layer shapes and length laws are those of ``workloads/configs.py``.

The plain forms hold the same cache as tensors of slots and find a request's tokens by index.
"""

from __future__ import annotations

import math
import random

import torch

own = False

VOCAB = 128256
MAX_HISTORY = 32768        # tokens of the longest cached history

# (query heads, KV heads, head_dim)
SHAPES = [(4, 2, 64), (16, 16, 64), (32, 8, 128), (40, 8, 128), (64, 8, 128)]
# magnitudes of the 4-bit codes 0..7; bit 3 is the sign
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, shape, n, cached, suffix, ragged=True, fmt="mx4", lens=1, name=None, **more):
    """n requests: `cached` tokens of history (median; whole blocks) and `suffix` new tokens (mean);
    ragged: lognormal histories and uniform suffixes instead of equal ones; lens: their seed."""
    c = dict(kind=kind, hq=shape[0], hkv=shape[1], d=shape[2], n=n, cached=cached, suffix=suffix, ragged=ragged,
             fmt=fmt, lens=lens, **more)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one new token of each of 64 running sessions goes into the cache
        _case("store", (32, 8, 128), 64, 0, 1, name="store_decode"),
        # a prefill batch goes into the cache: prompts of mixed length
        _case("store", (32, 8, 128), 8, 0, 3000, lens=9, name="store_prefill"),
        # the smallest call: one request of a small layer, latency only
        _case("attn", (4, 2, 64), 1, 256, 64, ragged=False, lse=False, name="attn_tiny"),
        # decode: one new token for each of 64 running sessions with lognormal histories
        _case("attn", (32, 8, 128), 64, 1808, 1, lens=1008, lse=False, name="attn_decode"),
        # questions about cached documents; the weights are wanted next, so the sums are too
        _case("attn", (40, 8, 128), 8, 8192, 128, ragged=False, lse=True, name="attn_question"),
        # uncached prompts on a multi-head layer of head_dim 64
        _case("attn", (16, 16, 64), 12, 0, 1100, lens=3, lse=False, name="attn_prefill64"),
        # a long document cached, a long new suffix
        _case("attn", (64, 8, 128), 1, 32768, 2048, ragged=False, lse=True, name="attn_longctx"),
        # a decode step adds its attention weights to those of the steps before
        _case("weights", (32, 8, 128), 64, 1808, 1, lens=1008, add=True, name="weights_decode"),
        # the weights of a batch of questions, from a bf16 pool
        _case("weights", (40, 8, 128), 8, 8192, 128, ragged=False, fmt="bf16", add=False, name="weights_question"),
        # the weights of a long suffix over a long document
        _case("weights", (64, 8, 128), 1, 32768, 2048, ragged=False, add=False, name="weights_longctx"),
        # running sessions are cut to 512 tokens for each head, bf16 pool
        _case("evict", (32, 8, 128), 64, 1808, 0, fmt="bf16", lens=1008, keep=512, first=4, recent=64, name="evict_decode"),
        # long documents are cut to an eighth, 4-bit pool
        _case("evict", (64, 8, 128), 4, 32768, 0, ragged=False, keep=4096, first=4, recent=256, name="evict_long"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["store", "store", "attn", "attn", "attn", "attn", "weights", "weights", "evict", "evict"])
    while True:
        shape = rng.choice(SHAPES)
        n = _log_int(rng, 1, 64)
        cached = 0 if kind == "store" or (kind != "evict" and rng.random() < 0.15) else _log_int(rng, 64, MAX_HISTORY)
        suffix = 1 if rng.random() < 0.3 else _log_int(rng, 1, 4096)
        more = {}
        if kind == "attn":
            more["lse"] = rng.random() < 0.5
        elif kind == "weights":
            more["add"] = rng.random() < 0.5
        elif kind == "evict":
            keep = _log_int(rng, 1, 8192)
            first = rng.randint(0, min(8, keep))
            more = dict(keep=keep, first=first, recent=rng.randint(0, keep - first))
            suffix = 0
        fmt = rng.choice(["bf16", "mx4"]) if kind in ("weights", "evict") else "mx4"
        c = _case(kind, shape, n, cached, suffix, ragged=rng.random() < 0.8, fmt=fmt, lens=rng.randrange(1 << 30), **more)
        P, S = lengths(c)
        L = max(p + s for p, s in zip(P, S))
        w = work(c)
        if sum(P) + sum(S) > 160_000 or w["flops"] > 2.2e12 or w["bytes"] > 5e8 or n * L * shape[1] * shape[2] > 1.1e9:
            continue
        if kind in ("attn", "weights") and n * shape[0] * max(S) * L > 4e9:
            continue
        if kind == "evict" and n * more["keep"] * shape[1] * shape[2] > 6e7:
            continue
        return c


def lengths(case):
    """(cached tokens, new tokens) of every request."""
    rng = random.Random(case["lens"])
    P, S = [], []
    for _ in range(case["n"]):
        p, s = case["cached"], case["suffix"]
        if case["ragged"]:
            if p:
                p = max(16, min(int(rng.lognormvariate(math.log(p), 0.8)), 9 * p, MAX_HISTORY))
            if s > 1:
                s = rng.randint(max(1, s // 4), s * 7 // 4)
        P.append(p // 16 * 16)
        S.append(s)
    return P, S


def work(case):
    P, S = lengths(case)
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    t, tokens = sum(S), sum(P) + sum(S)
    kv = (4.0 if case["fmt"] == "bf16" else 17 / 16) * hkv * d              # bytes of a cached token
    pairs = sum(s * p + s * (s + 1) / 2 for p, s in zip(P, S))
    if kind == "store":       # rows in, 4-bit tokens, rows out
        return {"bytes": 8.0 * t * hkv * d + t * kv + 4.0 * t, "flops": 0}
    if kind == "attn":
        return {"bytes": 4.0 * t * hq * d + tokens * kv + 4.0 * t * hq * case["lse"], "flops": 4.0 * d * hq * pairs}
    if kind == "weights":
        return {"bytes": t * hq * (2.0 * d + 4) + tokens * (kv / 2 + hkv * (8.0 if case["add"] else 4.0)),
                "flops": 2.0 * d * hq * pairs}
    kept = sum(min(p, case["keep"]) for p in P)
    out = kept * (2 * kv if case["fmt"] == "bf16" else 2 * kv + 4.0 * hkv * d)   # 4 bits: read back as rows too
    return {"bytes": 4.0 * tokens * hkv + 8.0 * case["n"] * case["keep"] * hkv + out, "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _inputs(case, seed):
    """Rows N(0, 1) in bf16 as the configurations say; keys with the few strong channels that real
    ones have.  k, v: every token's rows, request after request."""
    P, S = lengths(case)
    hq, hkv, d, kind, n = case["hq"], case["hkv"], case["d"], case["kind"], case["n"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens, r = sum(P) + sum(S), {}
    gain = 1 + 3 * (torch.rand(hkv, d, generator=gen, device="cuda") < 0.04)
    r["k"] = (_normal(gen, tokens, hkv, d) * gain).to(torch.bfloat16)
    r["v"] = _normal(gen, tokens, hkv, d)
    if kind in ("attn", "weights"):
        r["q"] = _normal(gen, sum(S), hq, d)
    L = max(p + s for p, s in zip(P, S))
    if kind == "evict":       # accumulated weights: a few heavy tokens, many light ones, some that got nothing
        w = torch.exp(2 * torch.randn(n, hkv, L, generator=gen, device="cuda"))
        r["w"] = w * (torch.rand(n, hkv, L, generator=gen, device="cuda") > 0.1)
    if kind == "weights":
        r["w"] = torch.exp(torch.randn(n, hkv, L, generator=gen, device="cuda"))
        if not case["add"]:
            r["w"].zero_()
    return r


def _index(case):
    """(lengths [n], new tokens [n], tokens [n, L]: rows of k and v, columns [n, S]: rows of q); past a
    request's end the first row."""
    P, S = lengths(case)
    ln = torch.tensor([p + s for p, s in zip(P, S)], device="cuda")
    sn = torch.tensor(S, device="cuda")
    i = torch.arange(int(max(p + s for p, s in zip(P, S))), device="cuda")
    j = torch.arange(max(max(S), 1), device="cuda")
    tok = torch.where(i < ln[:, None], (ln.cumsum(0) - ln)[:, None] + i, 0)
    col = torch.where(j < sn[:, None], (sn.cumsum(0) - sn)[:, None] + j, 0)
    return ln, sn, tok, col


# ---- the plain forms -----------------------------------------------------------------------------

def _pack(x):
    """bf16 rows [T, H, D] -> (codes [T, H, D / 2], exponents [T, H, D / 32]): 4-bit values."""
    t, h, d = x.shape
    g = x.view(t, h, d // 32, 32)
    top = (g.view(torch.int16).to(torch.int32) & 0x7FFF).amax(3)            # bits of the largest magnitude
    e = (((top + 0x1F) >> 7) - 2).clamp(2, 252) - 127                        # smallest with top <= 7 * 2^e
    a = torch.ldexp(g.float().abs(), -e[..., None])
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code = (code + 8 * (g < 0)).to(torch.uint8).view(t, h, d // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), e.to(torch.int8)


def _unpack(codes, e):
    """The values that 4-bit codes and their exponents stand for, fp32."""
    table = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], dim=-1).long()
    x = table[both].reshape(*e.shape, 32)
    return torch.ldexp(x, e[..., None].to(torch.int32)).flatten(-2)


def _rows(st, what, tok):
    """fp32 K or V rows of tokens `tok` from the cache of the state."""
    if st["case"]["fmt"] == "bf16":
        return st[what][tok].float()
    codes, e = st[what]
    return _unpack(codes[tok], e[tok])


def _scores(case, q, k, ln, sn, col):
    """Scaled scores [n, Hkv, S * G, L], -inf where a column does not see a key."""
    n, L, hkv, d = k.shape
    s, G = col.shape[1], case["hq"] // hkv
    qc = q[col].float().view(n, s, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, s * G, d)
    sc = torch.matmul(qc, k.permute(0, 2, 3, 1).contiguous()).mul_(d ** -0.5)
    pos = (ln - sn)[:, None] + torch.arange(s, device="cuda")               # keys 0..pos are seen
    hidden = torch.arange(L, device="cuda") > pos.repeat_interleave(G, 1)[:, :, None]
    return sc.masked_fill_(hidden[:, None], -math.inf)


def _lse(case, q, k, ln, sn, col):
    """log sum exp of every column's scores as rows [T, Hq]."""
    sc = _scores(case, q, k, ln, sn, col)
    m = sc.amax(3)
    lse = m + sc.sub_(m[..., None]).exp_().sum(3).log()
    return _columns(case, lse[..., None], sn)[..., 0].contiguous()


def _columns(case, x, sn):
    """[n, Hkv, S * G, X] -> the new tokens' rows [T, Hq, X]."""
    n, hkv, c, w = x.shape
    s = c // (case["hq"] // hkv)
    rows = x.view(n, hkv, s, -1, w).permute(0, 2, 1, 3, 4).reshape(n, s, case["hq"], w)
    return rows[torch.arange(s, device="cuda") < sn[:, None]]


def _select(w, ln, keep, first, recent):
    """Kept positions [n, Hkv, keep], ascending, -1 past a request's tokens: the first, the most
    recent, and of the others those of the greatest weight (the lowest position among equals)."""
    n, h, L = w.shape
    i = torch.arange(L, device="cuda")
    held = (i < first) | (i >= (ln - recent)[:, None])
    rank = torch.where(held[:, None], math.inf, w)
    rank = torch.where((i < ln[:, None])[:, None], rank, -math.inf)
    order = torch.sort(rank, dim=2, descending=True, stable=True).indices[:, :, :keep]
    got = torch.where(order < ln[:, None, None], order, L).sort(dim=2).values
    got = torch.nn.functional.pad(got, (0, keep - got.shape[2]), value=L)
    return torch.where(got < L, got, -1).to(torch.int32)


# ---- what a program has in hand, and one pass ----------------------------------------------------

def _engine(case, toks, P, seed):
    """The framework's side: an engine whose cache holds the histories, and the planned batch."""
    import numpy as np
    from paper_2606_21238_amd.engine import PrefillEngine
    n = case["n"]
    blocks = sum(-(-len(t) // 16) for t in toks)
    phys = blocks + 2 * n
    keep = case.get("keep", 0)
    order = np.random.default_rng([seed, 2]).permutation(phys).astype(np.int32)
    eng = PrefillEngine(case["hq"], case["hkv"], case["d"], blocks + n, phys, n, policy="arc", pool_fill=0,
                        initial_order=order, kv_format=case["fmt"], private_blocks=n * -(-keep // 16))
    return eng


def prepare(case, seed):
    P, S = lengths(case)
    st = dict(case=dict(case), **_inputs(case, seed))
    ln, sn, tok, col = _index(case)
    kind, n = case["kind"], case["n"]
    if kind == "weights":
        st["lse"] = _lse(case, st["q"], st["k"][tok].float() if case["fmt"] == "bf16" else _unpack(*_pack(st["k"]))[tok], ln, sn, col)
    if own:
        import numpy as np
        rng = np.random.default_rng([seed, 1])
        toks = [rng.integers(0, VOCAB, p + s, dtype=np.int32) for p, s in zip(P, S)]
        eng = st["eng"] = _engine(case, toks, P, seed)
        # every token was computed and stored before; then the batch is planned over the cached histories
        db = eng.prepare(toks)
        if kind != "store":
            eng.scatter(db, st.pop("k"), st.pop("v"))
        eng.release()
        if kind in ("attn", "weights"):
            plan = db.plan
            plan.cu_q = np.concatenate([[0], np.cumsum(S)]).astype(np.int32)
            plan.prefix_lens = np.array(P, dtype=np.int32)
            plan.slot_mapping = np.concatenate([b[np.arange(p, p + s) // 16] * 16 + np.arange(p, p + s) % 16
                                                for b, p, s in zip(plan.block_tables, P, S)]).astype(np.int32)
            db = eng.upload(plan)
        st["db"] = db
        if kind == "attn":
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda") if case["lse"] else None
        elif kind == "store":
            st["back"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
        elif kind == "evict":
            nb = -(-case["keep"] // 16)
            st["dst"] = eng.num_phys + np.arange(n * nb, dtype=np.int32).reshape(n, nb)
            if case["fmt"] == "mx4":
                slots = (st["dst"][:, :, None] * 16 + np.arange(16)).reshape(n, -1)[:, :case["keep"]]
                st["slots"] = torch.from_numpy(slots.astype(np.int32)).cuda().flatten()
                st["back"] = tuple(torch.empty(n * case["keep"], case["hkv"], case["d"], dtype=torch.bfloat16, device="cuda")
                                   for _ in range(2))
    else:
        st.update(ln=ln, sn=sn, tok=tok, col=col)
        if kind != "store" and case["fmt"] == "mx4":
            st["k"], st["v"] = _pack(st["k"]), _pack(st["v"])
    return st


def _run_own(st):
    case, eng = st["case"], st["eng"]
    kind = case["kind"]
    if kind == "store":
        eng.scatter(st["db"], st["k"], st["v"])
        eng.gather(st["db"].slot_mapping, *st["back"])
        return {"k": st["back"][0], "v": st["back"][1]}
    if kind == "attn":
        eng.attention(st["db"], st["q"], st["out"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]} if case["lse"] else {"out": st["out"]}
    if kind == "weights":
        eng.attention_weights(st["db"], st["q"], st["lse"], st["w"], accumulate=case["add"])
        return {"w": st["w"]}
    kept, kept_w = eng.evict(st["db"], st["w"], case["keep"], st["dst"], n_first=case["first"], n_recent=case["recent"])
    if case["fmt"] == "bf16":
        return {"kept": kept, "w": kept_w, "k": eng.k_pool[eng.num_phys:].view(torch.bfloat16),
                "v": eng.v_pool[eng.num_phys:].view(torch.bfloat16)}
    eng.gather(st["slots"], *st["back"])
    return {"kept": kept, "w": kept_w, "k": st["back"][0], "v": st["back"][1]}


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    kind, ln, sn, tok, col = case["kind"], st["ln"], st["sn"], st["tok"], st["col"]
    if kind == "store":
        return {"k": _unpack(*_pack(st["k"])).to(torch.bfloat16), "v": _unpack(*_pack(st["v"])).to(torch.bfloat16)}
    if kind == "attn":
        sc = _scores(case, st["q"], _rows(st, "k", tok), ln, sn, col)
        m = sc.amax(3)
        p = sc.sub_(m[..., None]).exp_()
        total = p.sum(3)
        v = _rows(st, "v", tok).permute(0, 2, 1, 3).contiguous()
        o = torch.matmul(p, v).div_(total[..., None])
        out = _columns(case, o, sn).to(torch.bfloat16)
        if not case["lse"]:
            return {"out": out}
        return {"out": out, "lse": _columns(case, (m + total.log())[..., None], sn)[..., 0]}
    if kind == "weights":
        n, hkv, L = st["w"].shape
        G, s = case["hq"] // hkv, col.shape[1]
        c = st["lse"][col].view(n, s, hkv, G).permute(0, 2, 1, 3).reshape(n, hkv, s * G)
        p = _scores(case, st["q"], _rows(st, "k", tok), ln, sn, col).sub_(c[..., None]).exp_()
        there = (torch.arange(s, device="cuda") < sn[:, None]).repeat_interleave(G, 1)
        got = p.mul_(there[:, None, :, None]).sum(2)
        st["w"] = st["w"] + got if case["add"] else got
        return {"w": st["w"]}
    kept = _select(st["w"], ln, case["keep"], case["first"], case["recent"])
    there, at = kept >= 0, kept.clamp(min=0).long()
    n, hkv, keep = kept.shape
    kw = st["w"].gather(2, at) * there
    head = torch.arange(hkv, device="cuda")[:, None]
    rows = tok[torch.arange(n, device="cuda")[:, None, None], at]
    if case["fmt"] == "mx4":
        k, v = (_unpack(st[x][0][rows, head], st[x][1][rows, head]).to(torch.bfloat16) for x in "kv")
        k, v = (torch.where(there[..., None], x, 0).transpose(1, 2).reshape(n * keep, hkv, -1) for x in (k, v))
        return {"kept": kept, "w": kw, "k": k, "v": v}
    k, v = (torch.where(there[..., None], st[x][rows, head], 0) for x in "kv")
    k, v = (torch.nn.functional.pad(x, (0, 0, 0, -keep % 16)).unflatten(2, (-1, 16)).transpose(1, 2).flatten(0, 1) for x in (k, v))
    return {"kept": kept, "w": kw, "k": k.contiguous(), "v": v.transpose(2, 3).contiguous()}


# ---- the same values in 64 bits, request by request ----------------------------------------------

def _stored64(x):
    """What the 4-bit cache keeps of bf16 rows, in 64 bits."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    m, k = torch.frexp(top)                                   # top = m * 2^k, m in [0.5, 1)
    e = torch.where(m * 8 > 7, k - 2, k - 3).clamp(-125, 125)
    step = torch.pow(2.0, e.double())
    y = g / step
    lv = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    mid = (lv[1:] + lv[:-1]) / 2
    a = y.abs().contiguous()
    up, down = torch.bucketize(a, mid, right=True), torch.bucketize(a, mid, right=False)
    i = torch.where(up == down, up, up - up % 2)              # a tie goes to the even code
    return (lv[i] * y.sign() * step).flatten(-2)


def exact(case, seed):
    kind = case["kind"]
    if kind == "evict":       # positions, and values that are moved
        return None
    r = _inputs(case, seed)
    if kind == "store":
        return {"k": _stored64(r["k"]), "v": _stored64(r["v"])}
    P, S = lengths(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G = hq // hkv
    if kind == "weights":
        ln, sn, tok, col = _index(case)
        k32 = r["k"].float() if case["fmt"] == "bf16" else _unpack(*_pack(r["k"]))
        given = _lse(case, r["q"], k32[tok], ln, sn, col).double()
        del k32
        w = r["w"].double() if case["add"] else torch.zeros_like(r["w"], dtype=torch.float64)
    else:
        out = torch.empty(sum(S), hq, d, dtype=torch.float64, device="cuda")
        lse = torch.empty(sum(S), hq, dtype=torch.float64, device="cuda")
    at = so = 0
    for n, (p, s) in enumerate(zip(P, S)):
        k, v, q = r["k"][at:at + p + s], r["v"][at:at + p + s], r["q"][so:so + s].double()
        k, v = (k.double(), v.double()) if case["fmt"] == "bf16" else (_stored64(k), _stored64(v))
        hidden = torch.arange(p + s, device="cuda")[None, :] > torch.arange(p, p + s, device="cuda")[:, None]
        for h in range(hq):
            sc = (q[:, h].contiguous() @ k[:, h // G].t().contiguous()) / math.sqrt(d)
            sc.masked_fill_(hidden, -math.inf)
            if kind == "weights":
                w[n, h // G, :p + s] += torch.exp(sc - given[so:so + s, h, None]).sum(0)
                continue
            lse[so:so + s, h] = torch.logsumexp(sc, dim=1)
            out[so:so + s, h] = torch.exp(sc - lse[so:so + s, h, None]) @ v[:, h // G].contiguous()
        at, so = at + p + s, so + s
    if kind == "weights":
        return {"w": w}
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
