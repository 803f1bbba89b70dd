"""A serving step as it is used: tables, append, the indexer's selection over its own paged keys, attention; eager, captured and replayed."""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2607_11976_b200 import binding as lt

from kv4_util import Step, on_gpu

pytestmark = pytest.mark.gpu

H, DI = 64, 128  # the indexer's heads


class Server:
    """B requests over a pool of pages; the indexer's keys lie in a pool of their own under the same page numbers."""

    def __init__(self, B, T, max_pages, pages, Hq, Hkv, D, topk, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.B, self.T, self.Hq, self.Hkv, self.D, self.topk, self.pages, self.max_pages = B, T, Hq, Hkv, D, topk, pages, max_pages
        i32 = dict(dtype=torch.int32, device="cuda")
        self.g, self.scale = g, D**-0.5
        self.pool = lt.alloc_kv4_pool(pages, Hkv, D)
        self.pool.random_(0, 256, generator=g)  # whatever lay there: NaN scales among it
        self.keys = torch.zeros(pages * 64, DI, dtype=torch.bfloat16, device="cuda")
        self.free = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((B, max_pages), -1, **i32)
        self.ctx, self.new, self.total = (torch.zeros(B, **i32) for _ in range(3))
        self.start, self.status = torch.zeros(B + 1, **i32), torch.zeros(8, **i32)
        self.slots, self.position = torch.zeros(T, **i32), torch.zeros(T, **i32)
        self.kv = torch.zeros(T, 2, Hkv, D, dtype=torch.bfloat16, device="cuda")
        self.q = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device="cuda")
        self.out, self.out_sparse = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.lse, self.lse_sparse = (torch.zeros(T, Hq, device="cuda") for _ in range(2))
        self.idx = torch.full((T, topk), -1, **i32)
        self.ws = torch.empty(lt.lt_kv4_attention_workspace_bytes("bf16", T, B, Hq, Hkv, D), dtype=torch.uint8, device="cuda")

    def feed(self, new):
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        for t in (self.kv, self.q):
            t.copy_(torch.randn(t.shape, generator=self.g, device="cuda"))

    def call(self):
        lt.lt_page_tables(self.ctx, self.new, self.free, self.table, self.total, self.start, self.slots, self.position, self.status)
        lt.lt_kv4_append("bf16", self.kv[:, 0], self.kv[:, 1], self.slots, self.pool)
        lt.lt_kv4_attention("bf16", self.q, self.pool, self.table, self.start, self.ctx, self.scale, self.out, self.lse, self.ws)
        lt.lt_kv4_attention_topk("bf16", self.q, self.pool, self.table, self.start, self.ctx, self.idx, self.scale, self.out_sparse,
                                 self.lse_sparse, self.ws)

    def advance(self):
        used = int(self.status[2])
        self.free = torch.cat([self.free[used:], self.free[:used]])
        self.ctx.copy_(self.total)


class Mirror(Step):
    """The server's state as a Step, for its tolerances."""

    def __init__(self, s, ctx, new, pool):
        self.ctx, self.new, self.Hq, self.Hkv, self.D, self.dtype = ctx, new, s.Hq, s.Hkv, s.D, "bf16"
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T, self.pool, self.clean, self.table = s.T, pool, pool, s.table.cpu().numpy()
        self.q, self.scale = s.q.double().cpu().numpy(), s.scale


def _check(s, ctx, new, kv_log):
    """Outputs against 64-bit attention over what the requests were fed, quantised by the oracle."""
    start = np.concatenate([[0], np.cumsum(new)])
    pool = np.full(tuple(s.pool.shape), 0x5A, np.uint8)
    table = s.table.cpu().numpy()
    for b, rows in enumerate(kv_log):
        k, v = np.concatenate([r[:, 0] for r in rows]), np.concatenate([r[:, 1] for r in rows])
        assert k.shape[0] == ctx[b] + new[b]
        at = np.arange(k.shape[0])
        pool[table[b][at // 64], :, at % 64] = kv4.pack_rows(k, v)
    m = Mirror(s, np.asarray(ctx, np.int32), np.asarray(new, np.int32), pool)
    end = int(start[-1])
    for out, lse, idx in ((s.out, s.lse, None), (s.out_sparse, s.lse_sparse, s.idx.cpu().numpy())):
        o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
        o[end:], l[end:] = 7.0, 7.0  # (padding keeps what an earlier step left there)
        m.check(o, l, idx)


def _rows_fed(s, new):
    kv, at, fed = s.kv.float().cpu().numpy(), 0, []
    for n in new:
        fed.append(kv[at:at + n])
        at += n
    return fed


def test_steps_with_the_indexers_selection():
    """A prompt in chunks, then decoding: the indexer selects over its own paged keys by the same table."""
    s = Server(B=3, T=160, max_pages=40, pages=130, Hq=16, Hkv=2, D=128, topk=256, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    ctx, log = np.zeros(3, int), [[], [], []]
    for new in ([150, 0, 10], [100, 37, 23], [150, 0, 9], [0, 150, 1], [1, 1, 1], [4, 1, 0]):
        s.feed(new)
        iq = torch.randn(s.T, H, DI, generator=g, device="cuda").to(torch.bfloat16)
        iw = torch.randn(s.T, H, generator=g, device="cuda")
        ik = torch.randn(s.T, DI, generator=g, device="cuda").to(torch.bfloat16)
        s.idx.fill_(-1)
        s.call()  # (tables first: the indexer needs the pages; its result goes into the second call)
        start = np.concatenate([[0], np.cumsum(new)])
        ok = s.slots >= 0
        s.keys[s.slots[ok].long()] = ik[ok]
        for b in range(3):
            N = int(ctx[b] + new[b])
            if new[b] == 0:
                continue
            k = min(s.topk, N)
            rows = slice(int(start[b]), int(start[b + 1]))
            got = torch.full((new[b], k), -1, dtype=torch.int32, device="cuda")
            ws = torch.empty(lt.lt_indexer_topk_paged_workspace_bytes("bf16", new[b], N, H, DI, k), dtype=torch.uint8, device="cuda")
            lt.lt_indexer_topk_paged("bf16", iq[rows].contiguous(), iw[rows].contiguous(), s.keys, None, s.table[b].contiguous(), N, k,
                                     int(ctx[b]), got, None, ws)
            s.idx[rows, :k] = got
        s.call()
        torch.cuda.synchronize()
        assert s.status.tolist()[:2] == [0, sum(new)] and lt.lt_read_status(s.ws)[0] == 0
        for b, rows in enumerate(_rows_fed(s, new)):
            log[b].append(rows)
        _check(s, ctx, new, log)
        ctx = ctx + new
        s.advance()


def test_a_captured_step_follows_the_lengths():
    """One graph, replayed with other lengths, other tokens and other selections: the bits of eager calls."""
    s, e = (Server(B=4, T=200, max_pages=30, pages=140, Hq=16, Hkv=2, D=64, topk=64, seed=9) for _ in range(2))
    for x in (s, e):
        x.feed([1, 1, 1, 1])
        x.call()  # eager once: loads the kernels
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.call()
    free = s.free.clone()
    rng = np.random.default_rng(1)
    for x in (s, e):
        x.ctx.zero_()
        x.table.fill_(-1)
    for new in ([150, 1, 3, 40], [1, 1, 1, 1], [0, 180, 0, 2], [60, 60, 60, 20], [3, 2, 1, 0]):
        idx = torch.from_numpy(rng.integers(-1, 300, (200, 64)).astype(np.int32)).cuda()
        for x in (s, e):
            x.feed(new)
            x.idx.copy_(idx)
            x.out.fill_(3.0), x.out_sparse.fill_(3.0)
        graph.replay()
        e.call()
        torch.cuda.synchronize()
        for name in ("table", "slots", "position", "start", "total", "status", "out", "lse", "out_sparse", "lse_sparse"):
            assert torch.equal(getattr(s, name), getattr(e, name)), (new, name)
        used = int(e.status[2])
        for x in (s, e):
            x.ctx.copy_(x.total)
        free = torch.cat([free[used:], free[:used]])
        s.free.copy_(free), e.free.copy_(free)


def test_calls_on_two_streams_with_a_workspace_each():
    a, b = Step([700, 90, 2000], [1, 40, 2], 16, 2, 128, seed=1), Step([300, 1500], [90, 1], 32, 4, 128, seed=2)
    want = [a.run(), b.run()]
    got = []
    for s in (a, b):
        t = s.tensors()
        got.append(dict(s=s, t=t, out=torch.full((s.T, s.Hq, s.D), 7.0, dtype=torch.bfloat16, device="cuda"),
                        lse=torch.full((s.T, s.Hq), 7.0, device="cuda"), stream=torch.cuda.Stream(),
                        ws=torch.empty(lt.lt_kv4_attention_workspace_bytes("bf16", s.T, s.ctx.size, s.Hq, s.Hkv, s.D), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for x in got:
            s, t = x["s"], x["t"]
            lt.lt_kv4_attention("bf16", t["q"], t["pool"], t["table"], t["start"], t["ctx"], s.scale, x["out"], x["lse"], x["ws"], stream=x["stream"])
    torch.cuda.synchronize()
    for x, (o, l) in zip(got, want):
        assert np.array_equal(x["out"].double().cpu().numpy(), o) and np.array_equal(x["lse"].double().cpu().numpy(), l)


def test_strided_queries_no_lse_and_a_negative_or_zero_scale():
    s = Step([130, 500], [3, 60], 8, 2, 64, seed=5)
    wide = torch.zeros(s.T, 12, 64, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10] = on_gpu(s.q, torch.bfloat16)
    o, l = s.run(q=wide[:, 2:10])
    s.check(o, l)
    o2, none = s.run(q=wide[:, 2:10], want_lse=False)
    assert none is None and np.array_equal(o, o2)
    idx = s.selection(40)
    for scale in (-0.11, 0.0):
        s.scale = float(np.float32(scale))
        s.check(*s.run())
        s.check(*s.run(idx=idx), idx)


def test_large_and_tiny_queries():
    for gain in (1e4, 1e-6, 0.0):
        s = Step([100], [40], 8, 2, 64, seed=6, q_gain=gain)
        s.scale = float(np.float32(0.125 / max(gain, 1e-6)))
        s.check(*s.run())
        idx = s.selection(33)
        s.check(*s.run(idx=idx), idx)


def test_fewer_ctas_give_results_within_the_same_bounds():
    for new in ([1, 2, 1], [30, 2, 70]):
        s = Step([700, 90, 3000], new, 16, 2, 128, seed=8)
        for grid in (1, 3, 50):
            s.check(*s.run(grid=grid), on_gpu_too=True)


def test_lengths_beyond_the_table():
    """A context longer than the table reaches, up to the largest number: the tokens see what the table holds."""
    for ctx in (700, 1 << 30, 2**31 - 1):
        for new in (1, 60):
            s = Step([400], [new], 8, 2, 64, seed=11, poison=False)
            s.table = np.ascontiguousarray(s.table[:, :5])
            s.ctx[0] = ctx
            out, lse = s.run()
            s.ctx[0] = 319 + 60  # all tokens beyond the table's 320 positions
            s.check(out, lse)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right():
    s = Step([6000], [300], 16, 2, 128, seed=7)
    t = s.tensors()
    out, lse = torch.empty(s.T, 16, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(s.T, 16, device="cuda")
    ws = torch.empty(lt.lt_kv4_attention_workspace_bytes("bf16", s.T, 1, 16, 2, 128), dtype=torch.uint8, device="cuda")

    def call(limit_us):
        lt.lt_kv4_attention("bf16", t["q"], t["pool"], t["table"], t["start"], t["ctx"], s.scale, out, lse, ws, 300, lt.Tunables(wait_limit_us=limit_us))
        return lt.lt_read_status(ws)

    assert call(1)[0] == lt.LT_STATUS_TIMEOUT  # some wait of the first keys' way through the kernel takes longer than that
    assert call(0) == [0] * 8
    s.check(out.double().cpu().numpy(), lse.double().cpu().numpy(), on_gpu_too=True)


def test_pool_beyond_four_gigabytes():
    """Pages whose byte offset passes 32 bits, both kernels and both forms."""
    D, Hkv = 128, 4
    s = Step([500, 70], [2, 50], 16, Hkv, D, seed=10)
    page = lt.lt_kv4_page_bytes(Hkv, D)
    pages = (5 << 30) // page
    pool = lt.alloc_kv4_pool(pages, Hkv, D)
    far = np.random.default_rng(0).permutation(np.arange(pages - 400, pages))[:s.pages]
    far[0], far[-1] = pages - 1, 2**32 // page + 1
    pool[torch.from_numpy(far).cuda()] = on_gpu(s.pool)
    table = np.where(s.table >= 0, far[np.clip(s.table, 0, None)], -1).astype(np.int32)
    ws = torch.empty(lt.lt_kv4_attention_workspace_bytes("bf16", s.T, 2, 16, Hkv, D), dtype=torch.uint8, device="cuda")
    t, idx = s.tensors(), s.selection(64)
    for sel in (None, idx):
        out, lse = torch.full((s.T, 16, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((s.T, 16), 7.0, device="cuda")
        if sel is None:
            lt.lt_kv4_attention("bf16", t["q"], pool, on_gpu(table), t["start"], t["ctx"], s.scale, out, lse, ws)
        else:
            lt.lt_kv4_attention_topk("bf16", t["q"], pool, on_gpu(table), t["start"], t["ctx"], on_gpu(sel), s.scale, out, lse, ws)
        s.check(out.double().cpu().numpy(), lse.double().cpu().numpy(), sel)
