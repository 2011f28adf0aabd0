"""Pins of the 4-bit cache oracle (oracle/mx4.py): hand-worked groups, the error bound, the pool image."""

from __future__ import annotations

import numpy as np
import pytest

from oracle import mx4
from oracle.attention import bf16_to_f64


def to_bits(x):
    """float values that are exact in bf16 -> bits."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32)
    assert not (b & 0xFFFF).any()
    return (b >> 16).astype(np.uint16)


def group(*head):
    g = np.zeros(32, dtype=np.float32)
    g[: len(head)] = head
    return to_bits(g)


@pytest.mark.parametrize("x,e,want", [
    ((7.0, 6.5, 5.0, 5.0625, 3.5, 2.5, 0.25, 0.75, -1.25, -1.75), 0, (6, 6, 4, 6, 4, 2, 0, 1, -1, -2)),  # ties to even codes
    ((7.03125, 1.0, 0.5, -0.53125), 1, (8, 1, 0, -1)),          # just over 7: the next scale
    ((1.0, 0.25, 0.0625, 0.09375, 0.1875), -2, (1, 0.25, 0, 0.125, 0.25)),   # a step of 1/8
    ((0.0,), -125, (0,)),
    ((2.0 ** -126, -2.0 ** -130), -125, (2.0 ** -126, 0)),      # below the smallest step: zero
    ((3.3895313892515355e38, 2.0 ** 127, 2.0 ** 124), 125, (6 * 2.0 ** 125, 2.0 ** 127, 2.0 ** 124)),  # saturates
])
def test_hand_worked_groups(x, e, want):
    code, byte = mx4.quantise(group(*x))
    assert byte.tolist() == [e + 127]
    v = mx4.values(code, byte)
    assert v[: len(want)].tolist() == list(want) and not v[len(want):].any()


@pytest.mark.parametrize("bad", [0x7F80, 0xFF80, 0x7FC0, 0x7F81])
def test_groups_with_a_non_finite_value_read_back_as_nan(bad):
    g = np.concatenate([group(1.0, 2.0), group(1.0, 2.0)])
    g[5] = bad
    code, byte = mx4.quantise(g)
    assert byte.tolist() == [255, 126]     # 2 <= 7 * 2^-1
    v = mx4.values(code, byte)
    assert np.isnan(v[:32]).all() and v[32:34].tolist() == [1.0, 2.0]


def test_error_is_at_most_half_a_step_and_values_are_exact_in_bf16():
    rng = np.random.default_rng(4)
    bits = rng.integers(0, 0x7F80, (3000, 64)).astype(np.uint16)
    bits[1000:] = (bits[1000:] % 0x300) + 0x3E00          # a narrow range of magnitudes
    bits |= (rng.integers(0, 2, bits.shape) << 15).astype(np.uint16)
    x = bf16_to_f64(bits)
    code, byte = mx4.quantise(bits)
    v = mx4.values(code, byte)
    scale = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=1)
    y = np.abs(x) / scale
    # a magnitude in [2^k, 2^(k+1)) has steps of 2^(k-1), at least 0.5; 6 to 7 rounds to 6
    step = np.maximum(0.5, 2.0 ** np.floor(np.log2(np.maximum(y, 1e-300))) / 2)
    sat = byte.astype(int) - 127 == 125
    ok = np.abs(v - x) <= 0.5 * step * scale
    assert (ok | np.repeat(sat, 32, axis=1) | (y > 6)).all()
    over = (y > 6) & ~np.repeat(sat, 32, axis=1)
    assert (np.abs(v - x)[over] <= scale[over]).all()
    assert not (v.astype(np.float32).view(np.uint32) & 0xFFFF).any() and np.array_equal(v.astype(np.float32), v)
    nz = v[v != 0]
    assert np.abs(nz).min() >= 2.0 ** -126


@pytest.mark.parametrize("d,hkv", [(64, 3), (128, 2)])
def test_pool_image(d, hkv):
    rng = np.random.default_rng(d)
    bits = (rng.standard_normal((2, 40, hkv, d)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    slots = rng.permutation(5 * 16)[:40]
    pool = mx4.new_pool(5, hkv, d)
    mx4.scatter(pool, bits[0], bits[1], slots)
    k, v = mx4.gather(pool, slots)
    assert np.array_equal(k, mx4.stored(bits[0])) and np.array_equal(v, mx4.stored(bits[1]))
    # one value of one token by its place in the bytes
    s, h, i = int(slots[7]), hkv - 1, d - 3
    ck, bk = mx4.quantise(bits[0][7, h])
    cv, bv = mx4.quantise(bits[1][7, h])
    blk, o = pool[s // 16, h], s % 16
    assert (blk[o * d // 2 + i // 2] >> (4 * (i % 2))) & 15 == ck[i]
    assert (blk[8 * d + (o // 8) * 4 * d + (i // 2) * 8 + o % 8] >> (4 * (i % 2))) & 15 == cv[i]
    assert blk[16 * d + o * (d // 32) + i // 32] == bk[i // 32]
    assert blk[16 * d + d // 2 + (i // 32) * 16 + o] == bv[i // 32]
    # slots that no token has keep their bytes
    free = sorted(set(range(80)) - set(slots.tolist()))
    assert (pool[free[0] // 16, 0, (free[0] % 16) * d // 2:][: d // 2] == 0xFF).all()
