"""The definition of attention over the 4-bit cache with torch's 64-bit operations, and bounds on the bf16 kernels' error that count
each of their roundings, near enough that 32 keys lost or counted twice show.

What the cache's rows stand for is exact in fp16 (test_kv4_bounds.py), so neither kernel rounds keys or values.  Per key, with
w = |scale| sum_d |q_d k_d| and u = 2^-23 (a tensor core's product adds 17 numbers, each cut off at the last of 24 bits of the largest):
  few rows   a group of 32 elements begins at -8 sum q and takes two products over u_d = 1 .. 15: every number in it is at most
             M = max(8 sum |q_d|, 15 max |q_d|), so it is off by 2 * 17 u M, and what it begins with by 10 roundings of u / 2 of 8 sum |q_d|;
             times the group's scale and |scale|, summed over the groups that is w8.  The sum over the groups in fp32: 4 roundings of w.
  many rows  D / 16 products of exact factors: 8 * 17 u w.
  both       the exponent |y| under 64 of a probability that counts, in fp32 (64 * 2^-24), ex2.approx (2^-22) and up to 40 changes of the maximum
             or joins, each an ex2.approx: under 2^-16 in all; each shift or maximum held in fp32: 16 roundings of w.
so a key's probability is off by the factor e^ds, ds = max(w8, 136 u w) + 24 u w + 2^-16.
  lse        ds weighted by the probabilities, to first order (ds^2 bounds what is left), the sum of n' positive numbers in fp32 (n' 2^-24, n' the
             most keys of a run of work) and the fp32 result: log2 and the maximum, times ln 2.
  out        numerator and denominator move by ds, each probability by 2^-11 for fp16 (2^-36 of the largest if subnormal there), the numerator's
             products by n' / 16 * 17 u, all of sum p |v|; the result by 2^-8 of itself (a half step of bf16).
"""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv4

U = 2.0**-23


def definition(step, idx=None, device="cpu", times=None):
    """out, lse and what the bounds need, as torch float64 [T, Hq(, D)]; NaN where a row is nobody's.  times: how often each position of
    a request counts (a float64 tensor per request, default once)."""
    T, Hq, D, Hkv, group = step.T, step.Hq, step.D, step.Hkv, step.Hq // step.Hkv
    def wide(a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device)
    kv = [wide(x) for x in kv4.unpack_rows(step.clean)]  # [pages, Hkv, 64, D]
    scales = wide(np.ascontiguousarray(step.clean[..., D:D + D // 16]).view(np.float16).astype(np.float64))  # of keys
    q = wide(step.q)
    rows = dict(dtype=torch.float64, device=device)
    r = dict(out=torch.full((T, Hq, D), float("nan"), **rows), spread=torch.zeros(T, Hq, D, **rows), mass=torch.zeros(T, Hq, D, **rows),
             lse=torch.full((T, Hq), float("nan"), **rows), ds_mean=torch.zeros(T, Hq, **rows), ds_max=torch.zeros(T, Hq, **rows),
             weight=torch.zeros(T, Hq, **rows))
    for b in range(step.ctx.size):
        t0, t1, ctx = int(step.start[b]), int(step.start[b + 1]), int(step.ctx[b])
        if t1 == t0:
            continue
        at = torch.arange(min(ctx + t1 - t0, 64 * step.table.shape[1]), device=device)
        page = wide(step.table[b].astype(np.int64))[at // 64]
        there = (page >= 0) & (page < kv[0].shape[0])
        page = torch.where(there, page, 0)
        last = ctx + torch.arange(t1 - t0, device=device)
        if idx is None:
            count = (at[None] <= last[:, None]).double()
        else:
            i = wide(idx[t0:t1].astype(np.int64))
            ok = (i >= 0) & (i <= last[:, None]) & (i < at.numel())
            count = torch.zeros(t1 - t0, at.numel(), **rows)
            count.scatter_add_(1, torch.where(ok, i, 0), ok.double())
        count = count * there
        if times is not None:
            count = count * times[b].to(device)
        for h in range(Hkv):
            k, v = (x[page, h, at % 64] for x in kv)
            hs = slice(h * group, (h + 1) * group)
            x = q[t0:t1, hs]
            size = abs(step.scale)
            s = step.scale * torch.einsum("tgd,nd->tgn", x, k) + torch.log(count)[:, None]
            lse = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[..., None]).nan_to_num(0.0)
            parts = x.abs().reshape(*x.shape[:-1], D // 32, 32)
            m = torch.maximum(8 * parts.sum(-1), 15 * parts.amax(-1)) * 34 * U + parts.sum(-1) * 8 * 10 * U / 2
            w = size * torch.einsum("tgd,nd->tgn", x.abs(), k.abs())
            w8 = size * torch.einsum("tgi,ni->tgn", m, scales[page, h, at % 64])
            ds = torch.maximum(w8, 136 * U * w) + 24 * U * w + 2.0**-16
            ds = ds * (count > 0)[:, None]
            r["out"][t0:t1, hs], r["spread"][t0:t1, hs], r["lse"][t0:t1, hs] = p @ v, p @ v.abs(), lse
            r["mass"][t0:t1, hs] = (count @ v.abs())[:, None]
            r["ds_mean"][t0:t1, hs], r["ds_max"][t0:t1, hs] = (p * ds).sum(-1), ds.amax(-1)
            r["weight"][t0:t1, hs] = (w * (count > 0)[:, None]).amax(-1)
    return r


def keys_of_a_run(step, idx, sms):
    """Most keys of one row that pass through one set of accumulators: work is cut evenly over the CTAs, in the measure of rows of 8 (other
    items are larger and fewer), keys rounded up to 128 and 256 more for an item."""
    keys = step.ctx.astype(np.int64) + step.new if idx is None else np.where(step.new > 0, idx.shape[1], 0)
    heads = step.Hq // step.Hkv
    items = -(-step.new.astype(np.int64) * heads // 8) if idx is None else step.new.astype(np.int64) * -(-heads // 8)
    return int(min(keys.max(), ((keys + 512) * items * step.Hkv).sum() // sms + 512))


def check_tight(step, out, lse, idx=None, ref=None, sms=148, device="cpu"):
    """Asserts that out and lse (numpy) are within the bounds above; returns the largest shares of them."""
    r = definition(step, idx, device) if ref is None else ref
    end, n = int(step.start[-1]), keys_of_a_run(step, idx, sms)
    r = {name: x[:end].cpu().numpy() for name, x in r.items()}
    empty = np.isneginf(r["lse"])
    assert np.array_equal(np.isneginf(lse[:end]), empty), "rows that see nothing"
    want = np.where(empty, 0.0, r["lse"])
    ltol = r["ds_mean"] + r["ds_max"]**2 + n * 2.0**-24 + 2.0**-22 * (np.abs(want) + r["weight"] + 32)
    lshare = np.abs(np.where(empty, 0.0, lse[:end]) - want) / ltol
    assert lshare.max() <= 1, f"lse: {lshare.max():.2f} of its bound"
    rel = 2 * r["ds_max"] + 2.0**-11 + n * (17 * U / 16 + 2.0**-24)
    ref_out = np.nan_to_num(r["out"])
    tol = rel[..., None] * r["spread"] + 2.0**-36 * r["mass"] + 2.0**-8 * (1 + rel[..., None]) * np.abs(ref_out) + 1e-30
    share = np.abs(out[:end] - ref_out) / tol
    assert share.max() <= 1, f"out: {share.max():.2f} of its bound"
    return float(lshare.max()), float(share.max())
