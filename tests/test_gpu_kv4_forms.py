"""The calls of the 4-bit cache at sizes that launch every form of their kernels: four heads to a CTA, tables that take several turns of the
grid, and every bf16 number as the largest of a group."""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2607_11976_b200 import binding as lt

from kv4_util import Step, on_gpu
from test_gpu_kv4_cache import _append_read, _tables

pytestmark = pytest.mark.gpu


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# The fp32 kernel takes four heads to a CTA from tokens x Hkv x ceil(group / 4) = twice the SMs on.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(16, 4), (20, 4), (36, 4), (12, 4), (1, 1)])  # groups of 4, 5, 9, 3 and 1
def test_fp32_attention_of_many_tokens(dtype, D, Hq, Hkv):
    per = Hkv * -(-(Hq // Hkv) // 4)
    tokens = -(-2 * _sms() // per) + 20
    s = Step([90, 0], [tokens - 30, 30], Hq, Hkv, D, dtype, seed=Hq, pad=2, q_gain=1.5)
    s.check(*s.run(lt.LT_PATH_GENERIC), fused=False, on_gpu_too=True)
    idx = s.selection(70, empty_rows=range(0, s.T, 9))
    s.check(*s.run(lt.LT_PATH_GENERIC, idx), idx, fused=False, n_most=70, on_gpu_too=True)


@pytest.mark.parametrize("less", [1, 0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fp32_attention_around_the_change_of_form(dtype, less):
    s = Step([100], [2 * _sms() - less], 4, 1, 128, dtype, seed=less, q_gain=1.5)
    s.check(*s.run(lt.LT_PATH_GENERIC), fused=False, on_gpu_too=True)
    idx = s.selection(33)
    s.check(*s.run(lt.LT_PATH_GENERIC, idx), idx, fused=False, n_most=33, on_gpu_too=True)


def _first_steps(ctx, new, pad, cols=None, T=None):
    ctx, new = np.asarray(ctx), np.asarray(new)
    per, old = -(-(ctx + new) // 64), -(-ctx // 64)
    order = np.random.default_rng(len(ctx)).permutation(int(per.sum()) + 4).astype(np.int32)
    table = np.full((len(ctx), cols or int(per.max())), -1, np.int32)
    at = 0
    for b in range(len(ctx)):
        table[b, :old[b]] = order[at:at + old[b]]
        at += old[b]
    T = T or int(new.sum()) + pad
    got, want = _tables(ctx, new, order[at:], table, T), kv4.page_tables(ctx, new, order[at:], table, T)
    for name, g, w in zip(("page_table", "total_len", "query_start", "slot_map", "position", "status"), got, want):
        assert np.array_equal(g, w), name


# A turn of the grid is 1024 tokens, or fresh pages, for every SM.
@pytest.mark.parametrize("B,new_hi,pad", [(701, 1024, 333), (1100, 600, 0), (1, 300_000, 5), (3, 200, 400_000), (2, 152_000, 152_000)])
def test_tables_of_several_turns_of_the_grid(B, new_hi, pad):
    rng = np.random.default_rng(B)
    new = rng.integers(0, new_hi + 1, B)
    new[-1] = new_hi
    _first_steps(rng.integers(0, 900, B), new, pad)


def test_fresh_pages_of_several_turns_of_the_grid():
    """Ten million tokens announced, a hundred rows for them: the pages are dealt out all the same, and the step reported as too long."""
    _first_steps([100, 0, 64], [5, 10_000_000, 300_000], 0, T=100)


def test_every_bf16_number_as_the_largest_of_a_group():
    """Infinities, NaN, numbers beyond the largest scale, scales below fp16's normal range, and zeros; the others are fractions of it (ties
    between codes among them) or, beside what is not finite, ordinary numbers."""
    bits = np.arange(1 << 16, dtype=np.uint32) << 16
    with np.errstate(invalid="ignore", over="ignore"):
        top = bits.view(np.float32)
        rng = np.random.default_rng(0)
        part = rng.integers(-14, 15, (1 << 16, 31)) / 14 * np.where(rng.random((1 << 16, 31)) < 0.5, 1, rng.random((1 << 16, 31)))
        rest = np.where(np.isfinite(top)[:, None], np.nan_to_num(top.astype(np.float64))[:, None] * part, rng.standard_normal((1 << 16, 31)) * 3e3)
    x = np.concatenate([top[:, None], kv4.bf16_round(rest).astype(np.float32)], 1)
    x = np.take_along_axis(x, rng.permuted(np.tile(np.arange(32), (1 << 16, 1)), axis=1), 1).reshape(-1, 2, 1, 64)
    k, v = np.ascontiguousarray(x[:, 0]), np.ascontiguousarray(x[:, 1])
    T = k.shape[0]
    slots = rng.permutation(T).astype(np.int32)
    pool, outs = _append_read("bf16", T, 1, 64, slots, T // 64, k, v, False)
    with np.errstate(invalid="ignore"):
        want = kv4.pack_rows(k, v)
    assert np.array_equal(pool[slots // 64, :, slots % 64], want)
    assert all(np.isfinite(o).all() for o in outs["f32"])


def test_bf16_append_of_extreme_values():
    """The f32 test's values where bf16 has them: both ways of quantising a group side by side in a row."""
    x = np.zeros((4, 1, 128), np.float32)
    x[0, 0, :8] = [1e30, -1e30, np.inf, -np.inf, np.nan, 1.0, 20000.0, 9000.0]
    x[0, 0, 32:40] = [1e-9, -1e-9, 3e-8, 0, 0, 0, 0, 0]
    x[0, 0, 64:68] = [1.0, -0.5, 0.25, 7.0]
    x[1, 0, :4] = [4.1e-7, -2e-7, 1e-7, 5.9e-8]
    x[1, 0, 32:36] = [14336.0, -14335.0, 1024.0, 1023.0]  # the largest that the short way takes
    x[1, 0, 64:66] = [14400.0, 1.0]                       # the next bf16 number
    x[1, 0, 96:98] = [4.2724609375e-4, 2.1e-4]            # scale 2^-14
    x[2, 0, :2] = [np.nan, np.nan]
    x[2, 0, 32:64] = -np.inf
    x[3, 0, 0::2], x[3, 0, 1::2] = -0.0, np.float32(1.17e-38)
    x = kv4.bf16_round(np.nan_to_num(x, nan=0, posinf=0, neginf=0)).astype(np.float32) + np.where(np.isfinite(x), 0, x).astype(np.float32)
    slots = np.array([5, 70, 1, 63], np.int32)
    pool, outs = _append_read("bf16", 4, 1, 128, slots, 2, x, x[::-1].copy(), False)
    assert np.array_equal(pool[slots // 64, 0, slots % 64], kv4.pack_rows(x[:, 0], x[::-1, 0]))
    assert all(np.isfinite(o).all() for o in outs["f32"])
