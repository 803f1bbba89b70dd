"""Attention over the 4-bit cache: every key of every position counts once.  Bounds that a lost or doubled unit of 32 keys does not
pass (test_kv4_bounds.py), and contexts whose results name the units that were read."""
import numpy as np
import pytest
import torch

from paper_2607_11976_b200 import binding as lt

from kv4_bounds import check_tight
from kv4_util import Step

pytestmark = pytest.mark.gpu


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _tight(s, out, lse, idx=None):
    return check_tight(s, out, lse, idx, sms=_sms(), device="cuda")


DENSE = [
    ([40000], [1], 16, 1, 128),                              # one item over all CTAs, 16 rows
    ([9000], [2], 8, 2, 128),                                # 8 rows a key-value head
    ([9000, 30], [2, 300], 32, 4, 128),                      # few rows and pairs of tiles in one call
    ([20000], [90], 8, 8, 64),                               # a single tile, many CTAs
    ([3000, 500], [700, 401], 16, 2, 128),                   # pairs of tiles, the last ones partly or not at all there
    (np.arange(64) * 61 % 2000, [20] * 64, 16, 4, 128),
    (np.arange(40) * 997 % 3001, [12] * 40, 24, 4, 64),
    ([0], [1500], 12, 4, 64),
    (np.arange(300) * 37 % 1500, [1] * 300, 64, 8, 128),
    (np.arange(700) * 13 % 300, [1] * 700, 8, 2, 64),
    ([333, 20, 0, 64], [4, 3, 1, 1], 16, 2, 128),
    ([31, 63, 64, 65], [1, 1, 1, 1], 24, 8, 64),
]
SELECTED = [  # tokens, query heads, key-value heads, D, topk, context
    (200, 64, 1, 128, 2048, 5000), (333, 48, 1, 64, 700, 900), (90, 300, 1, 64, 333, 600),  # tiles
    (300, 16, 2, 128, 513, 2000), (200, 64, 4, 64, 1024, 1500), (3, 16, 1, 128, 8192, 9000)]  # few rows


@pytest.mark.parametrize("ctx,new,Hq,Hkv,D", DENSE)
def test_attention_within_tight_bounds(ctx, new, Hq, Hkv, D):
    s = Step(ctx, new, Hq, Hkv, D, seed=Hq + D, pad=2, q_gain=1.5)
    _tight(s, *s.run(max_new=max(new)))


@pytest.mark.parametrize("tokens,Hq,Hkv,D,topk,ctx", SELECTED)
def test_attention_topk_within_tight_bounds(tokens, Hq, Hkv, D, topk, ctx):
    s = Step([ctx, ctx // 3], [tokens - tokens // 3, tokens // 3], Hq, Hkv, D, seed=topk, pad=3, q_gain=1.5)
    idx = s.selection(topk, empty_rows=range(7, s.T, 50))
    _tight(s, *s.run(idx=idx), idx)


def _mark(s):
    """Zero queries, so that all weights are equal, and values of zero but for one key of every unit of 32, which has a one in the
    element that is the unit's number modulo D: a result's element counts its units, and lse is the logarithm of the keys' number."""
    s.q[:] = 0
    D = s.D
    for rows in (s.pool, s.clean):
        rows[..., D // 2:D], rows[..., D + D // 16:] = 0x88, 0
        for b in range(s.ctx.size):
            unit = np.arange((int(s.ctx[b] + s.new[b]) + 31) // 32)
            at = 32 * unit + (5 * unit + 3) % 32
            ok = at < int(s.ctx[b] + s.new[b])
            unit, at = unit[ok], at[ok]
            page, d = s.table[b][at // 64], unit % D
            rows[page, :, at % 64, D // 2 + d // 2] = np.where(d % 2, 0x98, 0x89).astype(np.uint8)[:, None]  # code 9: 1
            rows[page, :, at % 64, D + D // 16 + d // 32 * 2 + 1] = 0x3C  # fp16 1.0
    return s


@pytest.mark.parametrize("dtype,path", [("bf16", lt.LT_PATH_AUTO), ("bf16", lt.LT_PATH_GENERIC), ("f32", lt.LT_PATH_AUTO)],
                         ids=["bf16", "bf16-generic", "f32"])
@pytest.mark.parametrize("ctx,new,Hq,Hkv,D", DENSE[:7])
def test_every_unit_of_keys_counts_once(dtype, path, ctx, new, Hq, Hkv, D):
    s = _mark(Step(ctx, new, Hq, Hkv, D, dtype, seed=1, pad=2))
    out, lse = s.run(path, max_new=max(new))
    _tight(s, out, lse)
    for b in range(s.ctx.size):
        n = s.ctx[b] + 1 + np.arange(s.new[b])
        assert np.abs(lse[s.start[b]:s.start[b + 1]] - np.log(n)[:, None]).max() <= 1e-5  # (a key of 40,000: 2.5e-5)


@pytest.mark.parametrize("dtype,path", [("bf16", lt.LT_PATH_AUTO), ("f32", lt.LT_PATH_AUTO)], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens,Hq,Hkv,D,topk,ctx", SELECTED)
def test_every_selected_key_counts_once(dtype, path, tokens, Hq, Hkv, D, topk, ctx):
    s = _mark(Step([ctx, ctx // 3], [tokens - tokens // 3, tokens // 3], Hq, Hkv, D, dtype, seed=2, pad=3))
    idx = s.selection(topk)
    out, lse = s.run(path, idx)
    _tight(s, out, lse, idx)
    last = np.concatenate([s.ctx[b] + np.arange(s.new[b]) for b in range(2)])
    n = ((idx[:last.size] >= 0) & (idx[:last.size] <= last[:, None])).sum(1)
    assert np.abs(lse[:last.size] - np.log(n)[:, None]).max() <= 1e-5


def test_results_repeat_bit_for_bit():
    for i, (ctx, new, Hq, Hkv, D) in enumerate(DENSE[:6]):
        s = Step(ctx, new, Hq, Hkv, D, seed=i, q_gain=1.5)
        (o, l), idx = s.run(), s.selection(300)
        oi, li = s.run(idx=idx)
        for _ in range(4):
            for (a, b), (c, d) in ((s.run(), (o, l)), (s.run(idx=idx), (oi, li))):
                assert np.array_equal(a, c) and np.array_equal(b, d)
