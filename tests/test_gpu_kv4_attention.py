"""Attention over the 4-bit cache against its definition in 64 bits, on every path."""
import numpy as np
import pytest
import torch

from paper_2607_11976_b200 import binding as lt

from kv4_util import Step

pytestmark = pytest.mark.gpu

PATHS = [("bf16", lt.LT_PATH_AUTO), ("bf16", lt.LT_PATH_GENERIC), ("f32", lt.LT_PATH_AUTO)]
IDS = ["bf16", "bf16-generic", "f32"]

# contexts, tokens added, query heads, key-value heads, head size
SHAPES = [
    ([0], [1], 1, 1, 64),                               # one token sees itself
    ([0], [1], 8, 1, 128),
    ([31], [1], 8, 8, 128),                             # ends at a unit of 32 keys, one head each
    ([63, 64, 65], [1, 1, 1], 12, 4, 64),               # around a page
    ([500], [1], 64, 4, 128),                           # 16 heads a key-value head
    ([130, 0, 7, 1000], [1, 1, 1, 1], 40, 8, 128),      # 5 heads a key-value head
    ([333, 20], [4, 3], 16, 2, 128),                    # drafted tokens
    ([90, 0, 200], [0, 5, 2], 6, 2, 64),                # a request that adds nothing
    ([17], [40], 24, 8, 64),
    ([100, 0], [33, 70], 8, 2, 128),                    # short chunks
    ([2000], [2], 66, 2, 64),                           # 33 heads a key-value head
    ([64], [1], 128, 1, 128),
]


@pytest.mark.parametrize("dtype,path", PATHS, ids=IDS)
@pytest.mark.parametrize("ctx,new,Hq,Hkv,D", SHAPES)
def test_attention(dtype, path, ctx, new, Hq, Hkv, D):
    s = Step(ctx, new, Hq, Hkv, D, dtype, seed=len(ctx) + Hq, pad=3, q_gain=1.5)
    out, lse = s.run(path)
    s.check(out, lse, fused=dtype == "bf16" and path != lt.LT_PATH_GENERIC)


@pytest.mark.parametrize("dtype,path", PATHS, ids=IDS)
@pytest.mark.parametrize("ctx,new,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("topk", [1, 31, 96, 600])
def test_attention_topk(dtype, path, ctx, new, Hq, Hkv, D, topk):
    s = Step(ctx, new, Hq, Hkv, D, dtype, seed=topk + Hq, pad=2, q_gain=1.5)
    idx = s.selection(topk, empty_rows=range(0, s.T, 5))
    out, lse = s.run(path, idx)
    s.check(out, lse, idx, fused=dtype == "bf16" and path != lt.LT_PATH_GENERIC, n_most=topk)


@pytest.mark.parametrize("dtype,path", PATHS, ids=IDS)
def test_scales_far_apart_and_peaked_scores(dtype, path):
    s = Step([700, 90], [3, 1], 16, 2, 128, dtype, seed=4, q_gain=4.0, loud=True)
    fused = dtype == "bf16" and path != lt.LT_PATH_GENERIC
    s.check(*s.run(path), fused=fused)
    idx = s.selection(64, duplicates=True)
    s.check(*s.run(path, idx), idx, fused=fused)


@pytest.mark.parametrize("dtype,path", PATHS, ids=IDS)
def test_tables_with_pages_that_are_none(dtype, path):
    s = Step([300, 200, 50], [2, 1, 40], 8, 2, 64, dtype, seed=6)
    s.table[0, 1], s.table[1, :], s.table[2, 1] = -1, s.pages + 5, 2**31 - 1
    fused = dtype == "bf16" and path != lt.LT_PATH_GENERIC
    s.check(*s.run(path), fused=fused)
    idx = s.selection(70)
    s.check(*s.run(path, idx), idx, fused=fused)
    s.table = np.ascontiguousarray(s.table[:, :2])  # positions beyond the table
    s.check(*s.run(path), fused=fused)
    s.check(*s.run(path, idx), idx, fused=fused)
