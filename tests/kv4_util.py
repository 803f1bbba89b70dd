"""Inputs, calls and tolerances of the tests of the 4-bit key-value cache."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv4
from paper_2607_11976_b200 import binding as lt

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def on_gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


class Step:
    """Requests of ctx[b] cached and new[b] added tokens over a pool of random rows, pages in random order.  Rows of the pool that no
    token sees hold NaN and infinite scales (`poison`); their codes are random."""

    def __init__(self, ctx, new, Hq, Hkv, D, dtype="bf16", seed=0, pad=0, q_gain=1.0, spare_pages=2, poison=True, loud=False):
        rng = np.random.default_rng(seed)
        self.ctx, self.new = np.asarray(ctx, np.int32), np.asarray(new, np.int32)
        self.Hq, self.Hkv, self.D, self.dtype, self.pad = Hq, Hkv, D, dtype, pad
        B = self.ctx.size
        total = self.ctx + self.new
        per = -(-total // 64)
        self.max_pages = max(int(per.max()), 1)
        self.pages = int(per.sum()) + spare_pages
        order = rng.permutation(self.pages)
        self.table = np.full((B, self.max_pages), -1, np.int32)
        at = 0
        for b in range(B):
            self.table[b, :per[b]] = order[at:at + per[b]]
            at += per[b]
        k = rng.standard_normal((self.pages, Hkv, 64, D)).astype(np.float32)
        v = rng.standard_normal((self.pages, Hkv, 64, D)).astype(np.float32)
        if loud:  # scales that differ a great deal between positions and groups
            k *= np.exp(rng.uniform(-3, 1.5, (self.pages, Hkv, 64, D // 32, 1))).repeat(32, -1).reshape(k.shape).astype(np.float32)
            v *= np.exp(rng.uniform(-6, 6, (self.pages, Hkv, 64, D // 32, 1))).repeat(32, -1).reshape(k.shape).astype(np.float32)
        self.clean = kv4.pack_rows(k, v)
        self.pool = self.clean.copy()
        if poison:
            seen = np.zeros((self.pages, 64), bool)
            for b in range(B):
                p = np.arange(total[b] if self.new[b] else 0)
                seen[self.table[b, p // 64], p % 64] = True
            bad = np.array([np.nan, np.inf, -np.inf, 6e4], np.float16)
            for j in range(D // 16):
                self.pool[..., D + 2 * j:D + 2 * j + 2][np.broadcast_to(~seen[:, None], self.pool.shape[:3])] = bad[j % 4:j % 4 + 1].view(np.uint8)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.T = int(self.start[-1]) + pad
        q = (q_gain * rng.standard_normal((self.T, Hq, D))).astype(np.float32)
        self.q = kv4.bf16_round(q) if dtype == "bf16" else q.astype(np.float64)
        self.scale = float(np.float32(D**-0.5))
        self.rng = rng

    def selection(self, topk, empty_rows=(), duplicates=False):
        """idx [T, topk] as an indexer leaves it: distinct visible positions, padded with -1; further entries out of sight."""
        idx = np.full((self.T, topk), -1, np.int32)
        for b in range(self.ctx.size):
            for t in range(self.start[b], self.start[b + 1]):
                last = self.ctx[b] + t - self.start[b]
                got = self.rng.permutation(last + 1)[:topk]
                idx[t, :got.size] = got
                if got.size < topk and t % 2:
                    idx[t] = self.rng.permutation(idx[t])  # padding anywhere
                if t % 3 == 0:
                    idx[t, self.rng.integers(topk)] = last + 1 + self.rng.integers(200)  # not visible
                if duplicates:
                    idx[t, topk // 2:] = idx[t, :topk - topk // 2]
        for t in empty_rows:
            idx[t] = -1
        return idx

    def tensors(self):
        return dict(q=on_gpu(self.q, DT[self.dtype]), pool=on_gpu(self.pool), table=on_gpu(self.table), start=on_gpu(self.start),
                    ctx=on_gpu(self.ctx))

    def run(self, path=lt.LT_PATH_AUTO, idx=None, max_new=0, want_lse=True, q=None, grid=0):
        g = self.tensors()
        q = g["q"] if q is None else q
        out = torch.full((self.T, self.Hq, self.D), 7.0, dtype=DT[self.dtype], device="cuda")
        lse = torch.full((self.T, self.Hq), 7.0, device="cuda") if want_lse else None
        ws = torch.full((lt.lt_kv4_attention_workspace_bytes(self.dtype, self.T, self.ctx.size, self.Hq, self.Hkv, self.D),), 0xFF,
                        dtype=torch.uint8, device="cuda")
        tun = lt.Tunables(path=path, grid=grid)
        if idx is None:
            lt.lt_kv4_attention(self.dtype, q, g["pool"], g["table"], g["start"], g["ctx"], self.scale, out, lse, ws, max_new, tun)
        else:
            lt.lt_kv4_attention_topk(self.dtype, q, g["pool"], g["table"], g["start"], g["ctx"], on_gpu(idx), self.scale, out, lse, ws, tun)
        torch.cuda.synchronize()
        assert lt.lt_read_status(ws) == [0] * 8, "a wait ran out or an index check failed"
        return out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()

    def reference_on_gpu(self, idx=None):
        """kv4.attention(...) with torch's 64-bit operations, for sizes that the CPU would take minutes for."""
        T, Hq, D, Hkv = self.T, self.Hq, self.D, self.Hkv
        group = Hq // Hkv
        kv = [on_gpu(x) for x in kv4.unpack_rows(self.clean)]  # [pages, Hkv, 64, D] each
        q = on_gpu(self.q)
        out, spread = (torch.full((T, Hq, D), float("nan"), dtype=torch.float64, device="cuda") for _ in range(2))
        mass, lse = torch.zeros_like(out), torch.full((T, Hq), float("nan"), dtype=torch.float64, device="cuda")
        weight = torch.zeros_like(lse)
        for b in range(self.ctx.size):
            t0, t1, ctx = int(self.start[b]), int(self.start[b + 1]), int(self.ctx[b])
            if t1 == t0:
                continue
            at = torch.arange(ctx + t1 - t0, device="cuda")
            page = on_gpu(self.table[b].astype(np.int64))[at // 64]
            last = ctx + torch.arange(t1 - t0, device="cuda")
            if idx is not None:
                i = on_gpu(idx[t0:t1].astype(np.int64))
                ok = (i >= 0) & (i <= last[:, None])
                count = torch.zeros(t1 - t0, at.numel(), dtype=torch.float64, device="cuda")
                count.scatter_add_(1, torch.where(ok, i, 0), ok.double())
            else:
                count = (at[None] <= last[:, None]).double()
            for h in range(Hkv):
                k, v = (x[page, h, at % 64] for x in kv)
                hs = slice(h * group, (h + 1) * group)
                x = q[t0:t1, hs]
                s = self.scale * torch.einsum("tgd,nd->tgn", x, k) + torch.log(count)[:, None]
                lse[t0:t1, hs] = torch.logsumexp(s, -1)
                p = torch.exp(s - lse[t0:t1, hs, None]).nan_to_num(0.0)
                out[t0:t1, hs], spread[t0:t1, hs] = p @ v, p @ v.abs()
                mass[t0:t1, hs] = (count @ v.abs())[:, None]
                weight[t0:t1, hs] = (abs(self.scale) * torch.einsum("tgd,nd->tgn", x.abs(), k.abs()) * (count > 0)[:, None]).amax(-1)
        return [x.cpu().numpy() for x in (out, lse, spread, weight, mass)]

    def check(self, out, lse, idx=None, fused=True, n_most=None, on_gpu_too=False):
        """Against the 64-bit definition, within what the roundings on the way can do.

        Fused path.  A score is a sum of exact products accumulated in fp32 over codes offset by 8 (u, begun at -8 sum q):
        no more than 64 |q_d| s per element pass through an accumulator, in at most 4 roundings of 2^-22 each; the tiled
        form instead rounds key values, of 12 significant bits, to fp16 (2^-11 of scale * sum |q k|).  So a score is off by
        at most ds = weight * (2^-11 + 64 * 4 * 2^-22) where weight >= scale * sum |q k|; |code| >= 1 for most elements but not
        for all, which the factor 4 on the second term covers.  A probability is then off by the factor e^ds, by 2^-11 for its
        rounding to fp16, and the value by 2^-11 for its own; numerator and denominator both move: 2 ds + 2 * 2^-11, with 2^-20
        for sums and exponentials, of spread = sum p |v|.  Small probabilities are subnormal in
        fp16, times 2^11 as they are held relative to a maximum that is at most the largest: their rounding is not relative but up to
        2^-25, so 2^-36 of the largest each, which shows in an element whose code is 0 at every key that matters (2^-36 mass,
        mass = sum |v|; the largest probability is at most the sum).
        The result is rounded to bf16 (2^-8 of itself).
        fp32 path: ds = weight * (D + 8) 2^-24, sums of n terms, and a result rounded to 2^-24."""
        if on_gpu_too:
            ref, ref_lse, spread, weight, mass = self.reference_on_gpu(idx)
        else:
            ref, ref_lse, spread, weight, mass = kv4.attention(self.q, self.pool, self.table, self.start, self.ctx, self.scale, idx)
        end = int(self.start[-1])
        assert np.array_equal(out[end:], np.full_like(out[end:], 7.0)), "rows behind the last request were written"
        if fused:
            ds = weight * (2.0**-11 + 4 * 256 * 2.0**-22)
            rel, last, sums, lost = 2 * ds + 2 * 2.0**-11 + 2.0**-20, 2.0**-8, 2.0**-20, 2.0**-36
        else:
            n = n_most or int((self.ctx + self.new).max())
            ds = weight * (self.D + 8) * 2.0**-24
            rel, last, sums = 2 * ds + (n + 64) * 2.0**-24, 2.0**-24 if self.dtype == "f32" else 2.0**-8, (n + 64) * 2.0**-24
            lost = 0.0
        with np.errstate(invalid="ignore"):
            tol = rel[..., None] * spread + last * (1 + rel[..., None]) * np.abs(ref) + lost * mass + 1e-30
            err = np.abs(out - ref)
        bad = ~(err[:end] <= tol[:end])
        assert not bad.any(), f"{bad.sum()} of {bad.size} off; worst {np.nanmax(err[:end] / tol[:end]):.2f} of the tolerance, first at {np.argwhere(bad)[0]}"
        if lse is not None:
            assert np.array_equal(lse[end:], np.full_like(lse[end:], 7.0))
            empty = np.isneginf(ref_lse[:end])
            assert np.array_equal(np.isneginf(lse[:end]), empty)
            ltol = ds[:end] + sums + 2.0**-23 * (np.abs(np.where(empty, 0, ref_lse[:end])) + weight[:end] + 32)
            lerr = np.abs(np.where(empty, 0, lse[:end]) - np.where(empty, 0, ref_lse[:end]))
            assert (lerr <= ltol).all(), f"lse off by {np.max(lerr / ltol):.2f} of the tolerance"
        return float(np.nanmax(err[:end] / tol[:end])) if end else 0.0
