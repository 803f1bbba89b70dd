"""What the tests of the kernels rest on: values that fp16 holds, the quotient by 7, and bounds that a lost unit of keys does not pass."""
import numpy as np
import pytest
import torch

from oracle import kv4

from kv4_bounds import check_tight, definition
from kv4_util import Step


def test_every_value_that_a_code_stands_for_is_exact_in_fp16():
    """For all scales that the writer can leave: fp16 numbers of at most 8 significant bits, up to 2048."""
    half = np.arange(1, 0x6800 + 1, dtype=np.uint16).view(np.float16).astype(np.float64)  # all positive ones up to 2048
    bits = half / 2.0**np.floor(np.log2(half))  # 1 <= bits < 2
    scales = half[bits * 128 == np.round(bits * 128)]
    assert scales[0] == 2.0**-24 and scales[-1] == 2048 and scales.size > 3000
    values = np.arange(-8, 8)[:, None] * scales
    assert np.array_equal(values.astype(np.float16).astype(np.float64), values)
    amax = np.exp(np.random.default_rng(0).uniform(-18, 11, 20000)).astype(np.float32)
    x = np.zeros((20000, 32), np.float32)
    x[:, 0] = amax
    left = kv4.quantise(x)[1].astype(np.float64)[:, 0]
    assert np.isin(left[left > 0], scales).all()


def test_the_quotient_by_seven_from_a_product_and_its_correction():
    """q = RN(a y), y = RN(1 / 7), then RN(q + RN(a - 7 q) y): the quotient rounded once, for all 2^23 significands (a power of two
    changes nothing).  64-bit arithmetic holds each step before its rounding: a - 7 q has a few bits at the end of a's, times 24 of y."""
    a = (np.arange(1 << 23, dtype=np.uint32) | np.uint32(0x3F800000)).view(np.float32)
    y = np.float32(1) / np.float32(7)
    q = a * y
    r = a.astype(np.float64) - 7.0 * q.astype(np.float64)
    assert np.array_equal(r.astype(np.float32).astype(np.float64), r)  # the fused remainder is exact
    quotient = (q.astype(np.float64) + r * np.float64(y)).astype(np.float32)
    assert np.array_equal(quotient, a / np.float32(7))


CASES = [([40000], [1], 16, 1, 128), ([9000], [2], 8, 1, 128), ([3000], [3], 12, 4, 64)]


@pytest.mark.parametrize("ctx,new,Hq,Hkv,D", CASES)
@pytest.mark.parametrize("change", ["none", "lost", "twice"])
def test_a_unit_of_32_keys_lost_or_counted_twice_is_noticed(ctx, new, Hq, Hkv, D, change):
    """The definition itself, rounded as the kernels' results are, passes; one without 32 keys, or with them twice, does not."""
    s = Step(ctx, new, Hq, Hkv, D, seed=3, q_gain=1.5, poison=False)
    ref = definition(s)
    rng = np.random.default_rng(1)
    for unit in rng.integers(0, ctx[0] // 32, 1 if change == "none" else 5):
        times = torch.ones(ctx[0] + new[0], dtype=torch.float64)
        times[32 * unit:32 * unit + 32] = {"none": 1, "lost": 0, "twice": 2}[change]
        got = definition(s, times=[times])
        out, lse = got["out"].bfloat16().double().numpy(), got["lse"].float().double().numpy()
        if change == "none":
            check_tight(s, out, lse, ref=ref)
        else:
            with pytest.raises(AssertionError, match="of its bound"):
                check_tight(s, out, lse, ref=ref)


def test_a_selections_keys_lost_are_noticed():
    s = Step([5000], [6], 8, 1, 64, seed=4, q_gain=1.5, poison=False)
    idx = s.selection(2048)
    ref = definition(s, idx)
    check_tight(s, ref["out"].bfloat16().double().numpy(), ref["lse"].float().double().numpy(), idx, ref=ref)
    short = idx.copy()
    short[:, 640:672] = -1
    got = definition(s, short)
    with pytest.raises(AssertionError, match="of its bound"):
        check_tight(s, got["out"].bfloat16().double().numpy(), got["lse"].float().double().numpy(), idx, ref=ref)


def test_the_definition_agrees_with_the_oracle():
    s = Step([200, 0, 33], [3, 2, 0], 6, 2, 64, seed=12, pad=1)
    for idx in (None, s.selection(50, empty_rows=[1], duplicates=True)):
        r = definition(s, idx)
        out, lse, spread, weight, mass = kv4.attention(s.q, s.pool, s.table, s.start, s.ctx, s.scale, idx)
        for name, want in (("out", out), ("lse", lse), ("spread", spread), ("mass", mass), ("weight", weight)):
            assert np.allclose(r[name][:5].numpy(), want[:5], rtol=1e-11, atol=1e-12), name


def test_the_definition_agrees_with_the_oracle_where_pages_are_missing():
    s = Step([200, 300], [3, 20], 6, 2, 64, seed=13)
    s.table[0, 1], s.table[1, 0], s.table[1, 3] = -1, s.pages + 7, 2**31 - 1
    for cols in (s.table.shape[1], 2):
        s.table = np.ascontiguousarray(s.table[:, :cols])
        for idx in (None, s.selection(50, empty_rows=[1], duplicates=True)):
            r = definition(s, idx)
            for name, want in zip(("out", "lse"), kv4.attention(s.q, s.pool, s.table, s.start, s.ctx, s.scale, idx)):
                assert np.allclose(r[name].numpy(), want, rtol=1e-11, atol=1e-12), name
