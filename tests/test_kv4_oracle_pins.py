"""Pins of the 64-bit definitions of the 4-bit cache: rationals, hand-worked rows, brute force."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv4


def _nearest_even(f: Fraction) -> int:
    lo = f.numerator // f.denominator
    rest = f - lo
    return lo + (1 if rest > Fraction(1, 2) or (rest == Fraction(1, 2) and lo % 2) else 0)


@pytest.mark.parametrize("seed", range(4))
def test_codes_are_the_nearest_multiples_in_exact_arithmetic(seed):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((8, 64)) * 10.0 ** rng.integers(-6, 4)).astype(np.float32)
    if seed % 2:
        x = kv4.bf16_round(x).astype(np.float32)
    codes, scales = kv4.quantise(x)
    for r in range(8):
        for g in range(2):
            s = Fraction(float(scales[r, g]))
            for d in range(32 * g, 32 * g + 32):
                want = 0 if s == 0 else max(-7, min(7, _nearest_even(Fraction(float(x[r, d])) / s)))
                assert int(codes[r, d]) - 8 == want


def test_ties_saturation_zeros_and_nan():
    x = np.zeros((1, 32), np.float32)
    codes, scales = kv4.quantise(x)
    assert (codes == 8).all() and scales[0, 0] == 0
    x[0, :7] = [7.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5]  # scale 1: every half is a tie, to the even neighbour
    codes, scales = kv4.quantise(x)
    assert scales[0, 0] == 1 and (codes[0, :7].astype(int) - 8).tolist() == [7, 0, 2, 2, 0, -2, -2]
    x[0, :3] = [1e30, -np.inf, np.nan]
    codes, scales = kv4.quantise(x)
    assert scales[0, 0] == 2048 and codes[0, :3].tolist() == [15, 1, 8]
    assert np.array_equal(kv4.values(codes, scales)[0, :3], [14336.0, -14336.0, 0.0])


@pytest.mark.parametrize("D", [64, 128])
def test_rows_hold_what_was_quantised(D):
    rng = np.random.default_rng(D)
    k, v = (rng.standard_normal((5, D)).astype(np.float32) for _ in range(2))
    rows = kv4.pack_rows(k, v)
    assert rows.shape == (5, D + D // 8)
    for got, x in zip(kv4.unpack_rows(rows), (k, v)):
        assert np.array_equal(got, kv4.values(*kv4.quantise(x)))
        s = np.repeat(kv4.quantise(x)[1].astype(np.float64), 32, -1)
        assert (np.abs(got - x) <= 0.52 * s).all()  # half a step, and the largest element up to 7.03 steps
    # element 2 i in the low half of byte i, keys before values, key scales before value scales
    c = kv4.quantise(k)[0]
    assert rows[2, 3] & 15 == c[2, 6] and rows[2, 3] >> 4 == c[2, 7]
    assert rows[2, D // 2] & 15 == kv4.quantise(v)[0][2, 0]
    assert rows[2, D:D + 2].copy().view(np.float16)[0] == kv4.quantise(k)[1][2, 0]


def test_scales_keep_24_times_themselves_in_fp16():
    x = np.zeros((4096, 32), np.float32)
    x[:, 0] = np.exp(np.random.default_rng(0).uniform(-14, 9.5, 4096))
    s = kv4.quantise(x)[1].astype(np.float64)[:, 0]
    assert np.array_equal((24 * s).astype(np.float16).astype(np.float64), 24 * s)


def test_page_tables_worked_by_hand():
    table = np.full((3, 3), -5, np.int32)
    table[0, 0], table[2, 0] = 9, 4
    got, total, start, slots, position, status = kv4.page_tables([63, 0, 64], [3, 0, 1], [7, 8], table, 6)
    assert got.tolist() == [[9, 7, -5], [-5, -5, -5], [4, 8, -5]]
    assert total.tolist() == [66, 0, 65] and start.tolist() == [0, 3, 3, 4]
    assert slots.tolist() == [9 * 64 + 63, 7 * 64, 7 * 64 + 1, 8 * 64, -1, -1]
    assert position.tolist() == [63, 64, 65, 64, -1, -1]
    assert status.tolist() == [0, 4, 2, 0, 0, 0, 0, 0]
    got, _, start, slots, _, status = kv4.page_tables([63, 0, 64], [3, 0, 1], [7], table, 2)
    assert got[2].tolist() == [4, -1, -5] and start.tolist() == [0, 2, 2, 2] and slots.tolist() == [9 * 64 + 63, 7 * 64]
    assert status.tolist() == [8, 4, 1, 1, 0, 0, 0, 0]


def test_attention_brute_force_and_empty_rows():
    rng = np.random.default_rng(3)
    pool = kv4.pack_rows(rng.standard_normal((3, 2, 64, 64)).astype(np.float32), rng.standard_normal((3, 2, 64, 64)).astype(np.float32))
    q = rng.standard_normal((3, 4, 64))
    table = np.array([[2, 0], [-1, 1]], np.int32)
    out, lse, spread, _, mass = kv4.attention(q, pool, table, [0, 2, 3], [64, 0], 0.125)
    keys = [(2, s) for s in range(64)] + [(0, 0), (0, 1)]
    for t, n in ((0, 65), (1, 66)):
        for j in range(4):
            num, den = np.zeros(64), 0.0
            for page, s in keys[:n]:
                k, v = kv4.unpack_rows(pool[page, j // 2, s])
                e = np.exp(0.125 * float(k @ q[t, j]))
                num, den = num + e * v, den + e
            assert np.allclose(out[t, j], num / den, rtol=1e-12) and np.isclose(lse[t, j], np.log(den), rtol=1e-12)
    assert (np.abs(out[:2]) <= spread[:2] * (1 + 1e-12)).all() and (spread <= mass * (1 + 1e-12)).all()
    assert (out[2] == 0).all() and np.isneginf(lse[2]).all()  # its only page is no page
    idx = np.array([[64, -1, 0], [99, 65, 65], [0, 1, 2]], np.int32)
    out, lse, _, _, _ = kv4.attention(q, pool, table, [0, 2, 3], [64, 0], 0.125, idx)
    k, v = kv4.unpack_rows(pool[0, 0, 1])
    assert np.allclose(out[1, 0], v) and np.isclose(lse[1, 0], 0.125 * float(k @ q[1, 0]) + np.log(2))
