"""Pins of the 4-bit cache oracle (oracle/mx4.py) over whole ranges: every code, every bf16 magnitude, the scale
rule beside two others, and a block laid by hand."""

from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import mx4
from oracle.attention import bf16_to_f64
from oracle.qkv import f64_to_bf16_bits

VALUE = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def test_every_code_under_every_scale():
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)
    for byte in range(2, 253):
        v = mx4.values(codes, np.array([byte], np.uint8))
        want = [x * 2.0 ** (byte - 127) for x in VALUE]
        assert v[:16].tolist() == want + [-x for x in want] and np.signbit(v[8:16]).all()
        assert np.array_equal(v[:16], v[16:])


def nearest(y):
    """The code of a magnitude y <= 7: by the borders between neighbours, with what a tie becomes written out."""
    borders = [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6)]
    i = 0
    for k, (b, tie) in enumerate(borders):
        if y > b:
            i = k + 1
        elif y == b:
            i = tie
    return i


@pytest.mark.parametrize("up", [0, 1, 2, 5])
def test_every_magnitude_under_its_own_scale_and_larger_ones(up):
    """A group of x and a neighbour that fixes the scale `up` above the smallest that x alone allows."""
    x = bf16_to_f64(np.arange(0x7F80, dtype=np.uint16))
    e, own = [], []
    for v in x.tolist():
        m, k = math.frexp(v)                                # v = m 2^k, m in [0.5, 1): v <= 7 * 2^(k-3) up to m = 7/8
        own.append(max(-125, k - 3 if m <= 0.875 else k - 2) if v else -125)
        e.append(own[-1] + up)
    keep = [i for i, k in enumerate(e) if k <= 124 or up == 0]
    e = np.minimum(np.array(e)[keep], 125)
    x = x[keep]
    g = np.zeros((len(x), 32))
    g[:, 3] = -x
    if up:
        g[:, 20] = 7 * 2.0 ** e.astype(np.float64)
    code, byte = mx4.quantise(f64_to_bf16_bits(g))
    assert np.array_equal(byte[:, 0], e + 127)
    want = [8 + min(nearest(v / 2.0 ** int(k)), 7) for v, k in zip(x.tolist(), e)]
    assert code[:, 3].tolist() == want
    rest = np.delete(code, [3, 20], axis=1)
    assert not rest.any() and (code[:, 20] == (7 if up else 0)).all()


# Root-mean-square errors in per cent of the values', as documented to a tenth: this rule, the smallest power of two with
# the largest magnitude at most 6 times it, and the largest not over the magnitude divided by 4.
RMS = {"normal": (11.2, 11.5, 11.5), "heavy-tailed": (12.9, 13.9, 13.1), "uniform": (9.9, 9.9, 14.1)}


@pytest.mark.parametrize("name", list(RMS))
def test_rms_error_beside_other_scale_rules(name):
    rng = np.random.default_rng(0)
    n = (40000, 32)
    x = {"normal": lambda: rng.standard_normal(n), "heavy-tailed": lambda: rng.standard_t(4, n),
         "uniform": lambda: rng.uniform(-1, 1, n)}[name]()
    bits = f64_to_bf16_bits(x)
    x = bf16_to_f64(bits)
    top = np.abs(x).max(axis=1)
    got = [np.sqrt(((mx4.stored(bits) - x) ** 2).mean())]
    for e in (np.ceil(np.log2(top / 6)), np.floor(np.log2(top)) - 2):
        y = np.abs(x) / 2.0 ** e[:, None]
        near = np.abs(y[..., None] - np.array(VALUE)).argmin(axis=-1)
        got.append(np.sqrt(((np.array(VALUE)[near] * 2.0 ** e[:, None] - np.abs(x)) ** 2).mean()))
    got = [100 * g / np.sqrt((x ** 2).mean()) for g in got]
    assert got[0] < got[1] and got[0] < got[2]
    assert all(abs(g - want) < 0.1 for g, want in zip(got, RMS[name])), got


def test_a_block_laid_by_hand():
    """Head 1 of block 2, head_dim 64: token 11's bytes at their places (K codes from 0, V codes from 512, K scales from
    1024, V scales from 1056), everything else as it was."""
    k, v = np.zeros((2, 64)), np.zeros((2, 64))
    k[1, [0, 1, 31]] = 1.0, -6.0, 0.5              # 6 <= 7 * 2^0: scale byte 127
    k[1, [32, 63]] = 2.0, 12.0                     # 12 <= 7 * 2^1: 128
    v[1, [4, 5]] = -3.0, 0.75                      # 3 <= 7 * 2^-1: 126, codes of 6 and 1.5
    v[1, [62, 63]] = 0.0625, -0.03125              # 2^-4 <= 7 * 2^-6: 121, codes of 4 and 2
    pool = mx4.new_pool(4, 2, 64, fill=0xA5)
    mx4.scatter(pool, f64_to_bf16_bits(k)[None], f64_to_bf16_bits(v)[None], [2 * 16 + 11])
    want = np.full(17 * 64, 0xA5, np.uint8)
    want[11 * 32:12 * 32] = 0
    want[11 * 32 + 0] = 0xF2                       # -6 (15) over 1 (2)
    want[11 * 32 + 15] = 0x10                      # dimension 31: 0.5 (1)
    want[11 * 32 + 16] = 0x02                      # dimension 32: 2 = 1 * 2
    want[11 * 32 + 31] = 0x70                      # dimension 63: 12 = 6 * 2
    want[512 + 256 + 3 + 8 * np.arange(32)] = 0    # half 1, byte 3 of every pair
    want[512 + 256 + 3 + 8 * 2] = 0x3F             # -3 = -6 / 2 (15), 0.75 = 1.5 / 2 (3)
    want[512 + 256 + 3 + 8 * 31] = 0xC6            # 2^-4 = 4 / 64 (6), -2^-5 = -2 / 64 (12)
    want[1024 + 2 * 11:1024 + 2 * 11 + 2] = 127, 128
    want[1056 + 11], want[1056 + 16 + 11] = 126, 121
    assert np.array_equal(pool[2, 1], want)
    assert (pool[[0, 1, 3]] == 0xA5).all()
    gk, gv = mx4.gather(pool, [2 * 16 + 11])
    assert np.array_equal(gk[0, 1], k[1]) and np.array_equal(gv[0, 1], v[1])


def test_gather_reads_a_block_laid_by_hand():
    pool = mx4.new_pool(1, 1, 64, fill=0)
    b = pool[0, 0]
    b[5 * 32 + 7] = 0x9D                           # K of token 5: dimension 14 is -3 (13), 15 is -0.5 (9)
    b[1024 + 2 * 5] = 130                          # 2^3
    b[512 + 3 * 8 + 5] = 0x27                      # V of token 5: dimension 6 is 6 (7), 7 is 1 (2)
    b[1056 + 5] = 125
    b[1056 + 16 + 5] = 255                         # its second group is NaN
    k, v = mx4.gather(pool, [5])
    want = np.zeros(64)
    want[[14, 15]] = -24.0, -4.0
    assert np.array_equal(k[0, 0], want)
    want = np.r_[np.zeros(32), np.full(32, np.nan)]
    want[[6, 7]] = 1.5, 0.25
    assert np.array_equal(v[0, 0], want, equal_nan=True)
