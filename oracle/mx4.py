"""The 4-bit KV cache (oracle).  TEST INFRASTRUCTURE ONLY.

K and V rows kept as MXFP4: 32 consecutive dimensions of a token share one scale 2^e and each holds
a sign and one of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Definition, for a group of finite
bf16 values x:

    e    = the smallest integer in [-125, 125] with max|x| <= 7 * 2^e (125 if there is none)
    code = the nearest of the magnitudes to |x| / 2^e, a tie to the even code, at most 6

and a group with an infinity or a NaN reads back as NaN (scale byte 255).  All arithmetic here is
IEEE binary64 on exact values: nearest is decided by comparing distances.

Pool layout MX4 (an interface shared with the library by definition): ``[blocks][Hkv][17 D]`` bytes:
K codes [16][D/2], V codes [2][D/2][8], K scales [16][D/32], V scales [D/32][16]."""

from __future__ import annotations

import numpy as np

from .attention import bf16_to_f64

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(rows_bits):
    """bf16 rows [..., D] -> (codes [..., D] in 0..15, scale bytes [..., D/32])."""
    x = bf16_to_f64(rows_bits)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(g).all(axis=-1)
    g = np.where(bad[..., None], 0.0, g)
    top = np.abs(g).max(axis=-1)
    e = np.full(top.shape, -125)
    for k in range(-124, 126):
        e = np.where(top > 7 * 2.0 ** (k - 1), k, e)
    y = np.abs(g) / 2.0 ** e[..., None].astype(np.float64)
    dist = np.abs(y[..., None] - MAGNITUDES)
    nearest = dist == dist.min(axis=-1, keepdims=True)           # one, or two neighbours of a tie
    i = nearest.argmax(axis=-1)
    i = np.where((nearest.sum(axis=-1) == 2) & (i % 2 == 1), i + 1, i)
    code = i + 8 * np.signbit(g)
    byte = np.where(bad, 255, e + 127)
    return code.reshape(x.shape).astype(np.uint8), byte.astype(np.uint8)


def values(codes, scale_bytes):
    """The values that codes [..., D] and scale bytes [..., D/32] stand for, fp64."""
    c = codes.reshape(*scale_bytes.shape, 32)
    v = MAGNITUDES[c & 7] * np.where(c & 8, -1.0, 1.0) * 2.0 ** (scale_bytes[..., None].astype(np.float64) - 127)
    v = np.where(scale_bytes[..., None] == 255, np.nan, v)
    return v.reshape(codes.shape)


def stored(rows_bits):
    """What the cache keeps of bf16 rows, fp64."""
    return values(*quantise(rows_bits))


def new_pool(num_blocks: int, num_kv_heads: int, head_dim: int, fill: int = 0xFF):
    return np.full((num_blocks, num_kv_heads, 17 * head_dim), fill, dtype=np.uint8)


def _fields(pool):
    """K codes, V codes, K scales and V scales of a pool, as views of its bytes."""
    d = pool.shape[2] // 17
    lead = pool.shape[:2]
    parts = np.split(pool, [8 * d, 16 * d, 16 * d + d // 2], axis=2)
    return (parts[0].reshape(*lead, 16, d // 2), parts[1].reshape(*lead, 2, d // 2, 8),
            parts[2].reshape(*lead, 16, d // 32), parts[3].reshape(*lead, d // 32, 16))


def scatter(pool, k_bits, v_bits, slots) -> None:
    """The 4-bit form of token t's rows ([Hkv, D] bf16 bits) into slot slots[t], token by token."""
    for t, s in enumerate(np.asarray(slots, dtype=np.int64)):
        kp, vp, ks, vs = _fields(pool[s // 16:s // 16 + 1])
        o = int(s % 16)
        code, byte = quantise(k_bits[t])
        kp[0, :, o] = code[:, 0::2] | code[:, 1::2] << 4
        ks[0, :, o] = byte
        code, byte = quantise(v_bits[t])
        vp[0, :, o // 8, :, o % 8] = code[:, 0::2] | code[:, 1::2] << 4
        vs[0, :, :, o] = byte
        pool[s // 16] = np.concatenate([x[0].reshape(pool.shape[1], -1) for x in (kp, vp, ks, vs)], axis=1)


def gather(pool, slots):
    """fp64 K and V [n, Hkv, D] of the slots."""
    kp, vp, ks, vs = _fields(pool)
    s = np.asarray(slots, dtype=np.int64)
    b, o = s // 16, s % 16

    def codes(x):
        return np.stack([x & 15, x >> 4], axis=-1).reshape(*x.shape[:-1], 2 * x.shape[-1])

    k = values(codes(kp[b, :, o]), ks[b, :, o])
    v = values(codes(vp[b, :, o // 8, :, o % 8]), vs[b, :, :, o])
    return k, v
