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


def test_the_two_references_agree():
    from oracle import kv4
    s = Step([200, 0, 33], [3, 2, 0], 6, 2, 64, seed=12, pad=1)
    for idx in (None, s.selection(50, empty_rows=[1], duplicates=True)):
        for a, b in zip(s.reference_on_gpu(idx), kv4.attention(s.q, s.pool, s.table, s.start, s.ctx, s.scale, idx)):
            assert np.allclose(a, b, rtol=1e-11, atol=1e-12, equal_nan=True)


# Sizes at which a CTA has several items and many units of keys of each, ends in the middle of one and begins in the middle of another.
LONG = [
    (np.arange(64) * 61 % 2000, [20] * 64, 16, 4, 128),      # 80 rows a request: tiles of 128 rows
    (np.arange(40) * 997 % 3001, [12] * 40, 24, 4, 64),
    ([3000, 500], [700, 401], 16, 2, 128),                   # pairs of tiles, the last ones partly or not at all there
    ([0], [1500], 12, 4, 64),                                # the first chunk of a prompt
    (np.arange(300) * 37 % 1500, [1] * 300, 64, 8, 128),     # decoding
    (np.arange(700) * 13 % 300, [1] * 700, 8, 2, 64),        # more requests than a CTA has threads
    ([40000], [1], 16, 1, 128),                              # one item over all CTAs
    ([9000, 30], [2, 300], 32, 4, 128),                      # both kernels in one call
]


@pytest.mark.parametrize("ctx,new,Hq,Hkv,D", LONG)
@pytest.mark.parametrize("max_new", ["right", "unknown"])
def test_attention_over_several_items_per_cta(ctx, new, Hq, Hkv, D, max_new):
    s = Step(ctx, new, Hq, Hkv, D, seed=Hq + D, pad=5, q_gain=1.5)
    out, lse = s.run(max_new=max(new) if max_new == "right" else 0)
    s.check(out, lse, on_gpu_too=True)


@pytest.mark.parametrize("tokens,Hq,Hkv,D,topk,ctx", [
    (200, 64, 1, 128, 2048, 5000), (333, 48, 1, 64, 700, 900), (150, 128, 1, 128, 1000, 3000), (90, 300, 1, 64, 333, 600),  # tiles
    (300, 16, 2, 128, 513, 2000), (200, 64, 4, 64, 1024, 1500)])                                                          # few rows
def test_attention_topk_over_several_items_per_cta(tokens, Hq, Hkv, D, topk, ctx):
    s = Step([ctx, 0, ctx // 3], [tokens // 2, tokens // 4, tokens - tokens // 2 - tokens // 4], Hq, Hkv, D, seed=topk, pad=3, q_gain=1.5)
    idx = s.selection(topk, empty_rows=range(7, s.T, 50))
    out, lse = s.run(idx=idx)
    s.check(out, lse, idx, on_gpu_too=True)


@pytest.mark.parametrize("repeat", range(3))
def test_results_do_not_vary(repeat):
    """The same call again, beside other work: the same bits."""
    s = Step([4000, 100, 900], [130, 9, 1], 32, 2, 128, seed=repeat, q_gain=1.5)
    idx = s.selection(600)
    first, again = [s.run(), s.run(idx=idx)], []
    noise = torch.randn(4096, 4096, device="cuda")
    for _ in range(5):
        noise = noise @ noise / 64
        again += [s.run(), s.run(idx=idx)]
    for i, (o, l) in enumerate(again):
        assert np.array_equal(o, first[i % 2][0]) and np.array_equal(l, first[i % 2][1])
