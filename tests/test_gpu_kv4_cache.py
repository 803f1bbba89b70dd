"""Block tables, and the 4-bit cache's writer and reader, bit for bit against their definitions."""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2607_11976_b200 import binding as lt

from kv4_util import DT, on_gpu

pytestmark = pytest.mark.gpu


def _tables(ctx, new, free, table, T):
    B = len(ctx)
    g = dict(ctx=on_gpu(np.asarray(ctx, np.int32)), new=on_gpu(np.asarray(new, np.int32)), free=on_gpu(np.asarray(free, np.int32)),
             table=on_gpu(np.asarray(table, np.int32)))
    total, start, slots, position, status = (torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (B, B + 1, T, T, 8))
    lt.lt_page_tables(g["ctx"], g["new"], g["free"], g["table"], total, start, slots, position, status)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (g["table"], total, start, slots, position, status)]


@pytest.mark.parametrize("B,new_hi,ctx_hi,pad,short_pages,short_cols,short_T", [
    (1, 1, 0, 0, 0, 0, 0), (1, 1, 63, 0, 0, 0, 0), (1, 200, 64, 3, 0, 0, 0), (7, 0, 500, 2, 0, 0, 0), (64, 1, 4000, 0, 0, 0, 0),
    (33, 700, 300, 100, 0, 0, 0), (1024, 5, 300, 0, 0, 0, 0), (1025, 5, 300, 1, 0, 0, 0), (2500, 90, 900, 7, 0, 0, 0),
    (40, 300, 300, 5, 9, 0, 0), (40, 300, 300, 0, 0, 3, 0), (40, 300, 300, 0, 0, 0, 777), (1500, 70, 10, 0, 100, 1, 5000)])
def test_page_tables(B, new_hi, ctx_hi, pad, short_pages, short_cols, short_T):
    rng = np.random.default_rng(B + new_hi)
    ctx, new = rng.integers(0, ctx_hi + 1, B), rng.integers(0, new_hi + 1, B)
    new[-1] = new_hi
    per, old = -(-(ctx + new) // 64), -(-ctx // 64)
    cols = max(int(per.max()) + 1 - 2 * short_cols, 1)
    order = rng.permutation(int(per.sum()) + 4).astype(np.int32)
    table = np.full((B, cols), -1, np.int32)
    at = 0
    for b in range(B):
        n = min(old[b], cols)
        table[b, :n] = order[at:at + n]
        at += n
    free = order[at:][:max(int((per - old).sum()) + 2 - short_pages, 0)]
    T = max(int(new.sum()) + pad - short_T, 1)
    got, want = _tables(ctx, new, free, table, T), kv4.page_tables(ctx, new, free, table, T)
    for name, g, w in zip(("page_table", "total_len", "query_start", "slot_map", "position", "status"), got, want):
        assert np.array_equal(g, w), name


def test_page_tables_negative_lengths_missing_pages_and_no_free_list():
    table = np.full((4, 2), -1, np.int32)
    table[0, 0] = 3
    args = ([10, -5, 70, 2], [2, 3, 1, -9], [], table, 9)
    for g, w in zip(_tables(*args), kv4.page_tables(*args)):
        assert np.array_equal(g, w)


def test_tables_advance_over_steps():
    """Ten steps in a row, each one's total_len the next one's context_len: all live slots stay distinct."""
    rng = np.random.default_rng(5)
    B, cols = 6, 9
    free = rng.permutation(80).astype(np.int32)
    table, ctx, used = np.full((B, cols), -1, np.int32), np.zeros(B, np.int32), set()
    for step in range(10):
        new = rng.integers(0, 58, B).astype(np.int32)
        T = max(int(new.sum()), 1)
        table, total, start, slots, position, status = _tables(ctx, new, free, table, T)
        free, ctx = free[status[2]:], total
        assert status[0] == 0 and not used & set(slots[:start[-1]].tolist())
        used |= set(slots[:start[-1]].tolist())
    assert len(used) == int(ctx.sum())


def _append_read(dtype, T, Hkv, D, slots, pages, k, v, fused_projection):
    pool = torch.full((pages, Hkv, 64, D + D // 8), 0xA5, dtype=torch.uint8, device="cuda")
    if fused_projection:  # rows of q, k and v side by side
        qkv = torch.zeros(T, 4 * Hkv, D, dtype=DT[dtype], device="cuda")
        gk, gv = qkv[:, 2 * Hkv:3 * Hkv], qkv[:, 3 * Hkv:]
        gk.copy_(on_gpu(k, DT[dtype]))
        gv.copy_(on_gpu(v, DT[dtype]))
    else:
        gk, gv = on_gpu(k, DT[dtype]), on_gpu(v, DT[dtype])
    lt.lt_kv4_append(dtype, gk, gv, on_gpu(slots), pool)
    outs = {}
    for out_type in ("f32", "bf16"):
        ko, vo = (torch.full((T, Hkv, D), 7.0, dtype=DT[out_type], device="cuda") for _ in range(2))
        lt.lt_kv4_read(out_type, pool, on_gpu(slots), ko, vo)
        outs[out_type] = ko.float().cpu().numpy(), vo.float().cpu().numpy()
    return pool.cpu().numpy(), outs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hkv,D,strided", [(1, 1, 64, False), (1, 8, 128, True), (2, 3, 64, True), (63, 1, 128, False), (65, 2, 64, False),
                                             (300, 5, 128, True), (4099, 8, 128, False), (5000, 7, 64, True)])
def test_append_and_read(dtype, T, Hkv, D, strided):
    rng = np.random.default_rng(T + D)
    k = (rng.standard_normal((T, Hkv, D)) * np.exp(rng.uniform(-12, 4, (T, Hkv, 1)))).astype(np.float32)
    v = rng.standard_normal((T, Hkv, D)).astype(np.float32)
    v[0, 0, :32] = 0
    k[T // 2, -1] = np.round(k[T // 2, -1] * 2) / 2  # ties
    k[T // 2, -1, 0::32] = 7.0
    if dtype == "bf16":
        k, v = kv4.bf16_round(k).astype(np.float32), kv4.bf16_round(v).astype(np.float32)
    pages = T // 64 + 3
    slots = rng.permutation(pages * 64)[:T].astype(np.int32)
    if T > 4:
        slots[rng.integers(0, T, T // 5)] = -1
        slots[3] = pages * 64  # beyond the pool
    pool, outs = _append_read(dtype, T, Hkv, D, slots, pages, k, v, strided)
    want = np.full_like(pool, 0xA5)
    ok = (slots >= 0) & (slots < pages * 64)
    want[slots[ok] // 64, :, slots[ok] % 64] = kv4.pack_rows(k, v)[ok]
    assert np.array_equal(pool, want)
    for i, x in enumerate((k, v)):
        exact = kv4.values(*kv4.quantise(x)) * ok[:, None, None]
        assert np.array_equal(outs["f32"][i].astype(np.float64), exact)
        assert np.array_equal(outs["bf16"][i].astype(np.float64), kv4.bf16_round(exact))


def test_append_of_extreme_values():
    x = np.zeros((4, 1, 64), np.float32)
    x[0, 0, :8] = [1e30, -1e30, np.inf, -np.inf, np.nan, 1.0, 20000.0, 9000.0]
    x[0, 0, 32:40] = [1e-9, -1e-9, 3e-8, 0, 0, 0, 0, 0]
    x[1, 0, :4] = [4.1e-7, -2e-7, 1e-7, 5.9e-8]  # scales in fp16's subnormal range
    x[1, 0, 32:36] = [14336.0, -14335.0, 1024.0, 1023.0]
    x[2, 0, :2] = [np.nan, np.nan]
    x[3, 0, 0::2], x[3, 0, 1::2] = -0.0, np.float32(1.17e-38)
    slots = np.array([5, 70, 1, 63], np.int32)
    pool, outs = _append_read("f32", 4, 1, 64, slots, 2, x, x[::-1].copy(), False)
    assert np.array_equal(pool[slots // 64, 0, slots % 64], kv4.pack_rows(x[:, 0], x[::-1, 0]))
    assert np.isfinite(outs["f32"][0]).all()


def test_read_takes_a_slot_any_number_of_times_and_on_another_stream():
    rng = np.random.default_rng(9)
    rows = kv4.pack_rows(*(rng.standard_normal((2, 2, 64, 128)).astype(np.float32) for _ in range(2)))
    slots = np.array([7, 7, 127, 7, -1, 0, 128, -2**31], np.int32)
    pool, s = on_gpu(rows), on_gpu(slots)
    ko, vo = (torch.full((8, 2, 128), 7.0, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lt.lt_kv4_read("f32", pool, s, ko, vo)
    side.synchronize()
    ok = (slots >= 0) & (slots < 128)
    k, v = kv4.unpack_rows(rows[np.where(ok, slots, 0) // 64, :, np.where(ok, slots, 0) % 64])
    assert np.array_equal(ko.cpu().numpy(), k * ok[:, None, None]) and np.array_equal(vo.cpu().numpy(), v * ok[:, None, None])


def test_pool_beyond_four_gigabytes():
    """Rows whose byte offset passes 32 bits."""
    pages = (5 << 30) // lt.lt_kv4_page_bytes(1, 64)
    pool = lt.alloc_kv4_pool(pages, 1, 64)
    rng = np.random.default_rng(11)
    k, v = (rng.standard_normal((6, 1, 64)).astype(np.float32) for _ in range(2))
    slots = np.array([0, pages * 64 - 1, pages * 32, 64 * (2**32 // 4608) + 5, 64 * (2**31 // 4608) + 1, 77], np.int32)
    lt.lt_kv4_append("f32", on_gpu(k), on_gpu(v), on_gpu(slots), pool)
    ko, vo = (torch.empty((6, 1, 64), device="cuda") for _ in range(2))
    lt.lt_kv4_read("f32", pool, on_gpu(slots), ko, vo)
    assert np.array_equal(ko.double().cpu().numpy(), kv4.values(*kv4.quantise(k)))
    assert np.array_equal(vo.double().cpu().numpy(), kv4.values(*kv4.quantise(v)))
