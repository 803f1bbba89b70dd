"""Attention over the 4-bit cache where the arguments, not the sizes, are unusual."""
from __future__ import annotations

import numpy as np
import pytest

import kv4_util as ku
from oracle import kv4
from paper_2607_11976_b200 import binding as lt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("max_new", [1, 3, 1000])
def test_a_wrong_max_new_only_costs_time(max_new, D):
    """Requests with more rows than any kernel was launched for are attended all the same."""
    s = ku.Step([100, 3, 700, 0], [1, 40, 100, 260], 16, 2, D, seed=1)
    out, lse = s.run(max_new=max_new)
    s.check(out, lse)


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-12, -1e-12])
@pytest.mark.parametrize("new", [[1, 2], [300, 70]], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_zero_queries_and_tiny_scales_average_the_values(scale, new, D):
    """All weights are equal then, whatever is masked beside them."""
    s = ku.Step([70, 3], new, 8, 2, D, seed=2, pad=1)
    s.scale = scale
    s.q[::2] = 0
    s.q[1::2, :3] = 2.0**-120
    out, lse = s.run(max_new=max(new))
    s.check(out, lse)
    idx = s.selection(40, duplicates=True)
    out, lse = s.run(idx=idx)
    s.check(out, lse, idx)


@pytest.mark.parametrize("gain", [1e3, 1e5, 1e6, 2.5e7])
@pytest.mark.parametrize("new", [[1, 2], [300, 70]], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_scores_far_below_zero(gain, new, D):
    """Tokens that see one key, or few, whose scores are all far from zero: rounding them must not make a weight overflow or vanish.
    (What a token that sees one key gets is that key's value, whatever the score, but for the roundings of weight, value and result.)"""
    s = ku.Step([0, 3], new, 8, 2, D, seed=3, q_gain=gain)
    out, lse = s.run(max_new=max(new))
    s.check(out, lse)
    row = s.pool[s.table[0, 0], :, 0]
    value = kv4.unpack_rows(row)[1]
    assert (np.abs(out[0] - value.repeat(4, 0)) <= (2.0**-8 + 2.0**-10) * np.abs(value).repeat(4, 0)).all()
    idx = s.selection(2)
    out, lse = s.run(idx=idx)
    s.check(out, lse, idx)
    value = value * (idx[0] == 0).any()  # (a row that names nothing it sees gets zeros)
    assert (np.abs(out[0] - value.repeat(4, 0)) <= (2.0**-8 + 2.0**-10) * np.abs(value).repeat(4, 0)).all()


@pytest.mark.parametrize("dtype,Hq,Hkv", [("bf16", 8, 2), ("bf16", 80, 2), ("f32", 8, 2)])
@pytest.mark.parametrize("selected", [False, True])
def test_a_part_of_the_requests(selected, dtype, Hq, Hkv):
    """Tables from the second request on: the first one's rows are left as they were."""
    s = ku.Step([50, 90, 400], [30, 1, 70], Hq, Hkv, 64, dtype, seed=4, pad=2)
    idx = s.selection(60) if selected else None
    n = int(s.new[0])
    s.start, s.ctx, s.new, s.table = s.start[1:], s.ctx[1:], s.new[1:], s.table[1:]
    out, lse = s.run(idx=idx)
    assert (out[:n] == 7.0).all() and (lse[:n] == 7.0).all()
    s.start, s.q, s.T = s.start - n, s.q[n:], s.T - n
    s.check(out[n:], lse[n:], None if idx is None else idx[n:], fused=dtype == "bf16")


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (4, 1, 128)])
@pytest.mark.parametrize("kind", ["slots", "decode", "chunks"])
def test_many_requests(kind, Hq, Hkv, D):
    """Slots that are mostly empty, decoding requests with a few prompts between them, and short chunks: more requests than a CTA
    keeps in mind."""
    rng = np.random.default_rng(5)
    B = 1500
    new = {"slots": np.zeros(B, int), "decode": np.ones(B, int), "chunks": rng.integers(0, 18, B)}[kind]
    if kind != "chunks":
        new[[0, 40, 77, 1029, 1400, B - 1]] = [70, 1, 150, 40, 300, 2]
    ctx = np.where(new > 0, rng.integers(0, 90, B), 0)
    s = ku.Step(ctx, new, Hq, Hkv, D, seed=6)
    out, lse = s.run(max_new=int(new.max()))
    s.check(out, lse, on_gpu_too=True)


@pytest.mark.parametrize("Hq", [8, 40])
def test_many_requests_with_positions_of_their_own(Hq):
    rng = np.random.default_rng(7)
    new = np.zeros(1500, int)
    new[rng.integers(0, 1500, 90)] = 1
    new[[0, 700]] = [0, 9]
    s = ku.Step(np.where(new > 0, rng.integers(0, 200, 1500), 0), new, Hq, 1, 64, seed=8)
    idx = s.selection(70)
    out, lse = s.run(idx=idx)
    s.check(out, lse, idx, on_gpu_too=True)
