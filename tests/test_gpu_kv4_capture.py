"""Calls of the 4-bit cache captured and replayed, and beside other work of the library: every form gives the bits of an eager call by itself."""
import numpy as np
import pytest
import torch

from paper_2607_11976_b200 import binding as lt

from kv4_util import DT, Step
from test_gpu_kv4_step import DI, H, Server

pytestmark = pytest.mark.gpu


class Call:
    """One attention call with buffers of its own."""

    def __init__(self, s, topk=0, path=lt.LT_PATH_AUTO, max_new=0):
        self.s, self.path, self.max_new, self.t = s, path, max_new, s.tensors()
        self.idx = torch.from_numpy(s.selection(topk)).cuda() if topk else None
        self.out = torch.full((s.T, s.Hq, s.D), 7.0, dtype=DT[s.dtype], device="cuda")
        self.lse = torch.full((s.T, s.Hq), 7.0, device="cuda")
        self.ws = torch.empty(lt.lt_kv4_attention_workspace_bytes(s.dtype, s.T, s.ctx.size, s.Hq, s.Hkv, s.D), dtype=torch.uint8, device="cuda")

    def __call__(self, stream=None):
        s, t, tun = self.s, self.t, lt.Tunables(path=self.path)
        args = (s.dtype, t["q"], t["pool"], t["table"], t["start"], t["ctx"])
        if self.idx is None:
            lt.lt_kv4_attention(*args, s.scale, self.out, self.lse, self.ws, self.max_new, tun, stream)
        else:
            lt.lt_kv4_attention_topk(*args, self.idx, s.scale, self.out, self.lse, self.ws, tun, stream)

    def results(self):
        return self.out.clone(), self.lse.clone()


# queries' type, new tokens, query heads, key-value heads, selected positions, path
FORMS = [("bf16", [3, 1], 16, 2, 0, lt.LT_PATH_AUTO), ("bf16", [90, 300], 16, 2, 0, lt.LT_PATH_AUTO), ("bf16", [3, 1], 16, 2, 70, lt.LT_PATH_FUSED),
         ("bf16", [40, 30], 64, 1, 200, lt.LT_PATH_FUSED), ("bf16", [40, 30], 16, 2, 0, lt.LT_PATH_GENERIC), ("f32", [3, 1], 16, 2, 0, lt.LT_PATH_AUTO),
         ("f32", [40, 30], 16, 2, 70, lt.LT_PATH_AUTO)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,new,Hq,Hkv,topk,path", FORMS)
def test_every_form_replays_with_other_lengths_and_queries(dtype, new, Hq, Hkv, topk, path, D):
    call = Call(Step([700, 90], new, Hq, Hkv, D, dtype, seed=1, pad=2, q_gain=1.5), topk, path)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    g = torch.Generator(device="cuda").manual_seed(2)
    for ctx in ([700, 90], [100, 89], [0, 1], [699, 0]):
        call.t["ctx"].copy_(torch.tensor(ctx, dtype=torch.int32))
        call.t["q"].copy_(torch.randn(call.t["q"].shape, generator=g, device="cuda"))
        call.out.fill_(7.0), call.lse.fill_(7.0), call.ws.fill_(0xFF)
        graph.replay()
        got = call.results()
        call.out.fill_(7.0), call.lse.fill_(7.0), call.ws.fill_(0xFF)
        call()
        for a, b in zip(got, call.results()):
            assert torch.equal(a, b), ctx
        assert lt.lt_read_status(call.ws) == [0] * 8


def test_a_sparse_step_in_two_graphs_with_the_indexer_between_them():
    """The indexer's lengths come from the host: what stands before and behind it is captured, the indexer is called."""
    s, e = (Server(B=2, T=60, max_pages=20, pages=50, Hq=16, Hkv=2, D=128, topk=128, seed=3) for _ in range(2))

    def tables(x):
        lt.lt_page_tables(x.ctx, x.new, x.free, x.table, x.total, x.start, x.slots, x.position, x.status)
        lt.lt_kv4_append("bf16", x.kv[:, 0], x.kv[:, 1], x.slots, x.pool)

    def attend(x):
        lt.lt_kv4_attention_topk("bf16", x.q, x.pool, x.table, x.start, x.ctx, x.idx, x.scale, x.out_sparse, x.lse_sparse, x.ws)

    def select(x, iq, iw, ik, ctx, new):
        ok = x.slots >= 0
        x.keys[x.slots[ok].long()] = ik[ok]
        x.idx.fill_(-1)
        at = 0
        for b in range(2):
            N, rows = ctx[b] + new[b], slice(at, at + new[b])
            at += new[b]
            if new[b] == 0:
                continue
            k = min(x.topk, N)
            got = torch.empty(new[b], k, dtype=torch.int32, device="cuda")
            ws = torch.empty(lt.lt_indexer_topk_paged_workspace_bytes("bf16", new[b], N, H, DI, k), dtype=torch.uint8, device="cuda")
            lt.lt_indexer_topk_paged("bf16", iq[rows].contiguous(), iw[rows].contiguous(), x.keys, None, x.table[b].contiguous(), N, k, ctx[b], got, None, ws)
            x.idx[rows, :k] = got

    for x in (s, e):
        x.feed([1, 1])
        tables(x), attend(x)
    torch.cuda.synchronize()
    before, behind = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(before):
        tables(s)
    with torch.cuda.graph(behind):
        attend(s)
    for x in (s, e):
        x.ctx.zero_(), x.table.fill_(-1)
    g = torch.Generator(device="cuda").manual_seed(4)
    ctx, free = [0, 0], s.free.clone()
    for new in ([50, 10], [1, 59], [40, 0], [2, 1], [1, 1]):
        iq, iw, ik = (torch.randn(shape, generator=g, device="cuda").to(t) for shape, t in
                      (((60, H, DI), torch.bfloat16), ((60, H), torch.float32), ((60, DI), torch.bfloat16)))
        for x in (s, e):
            x.feed(new)
            x.out_sparse.fill_(3.0), x.lse_sparse.fill_(3.0)
        before.replay()
        select(s, iq, iw, ik, ctx, new)
        behind.replay()
        tables(e)
        select(e, iq, iw, ik, ctx, new)
        attend(e)
        torch.cuda.synchronize()
        for name in ("table", "slots", "position", "start", "total", "status", "idx", "out_sparse", "lse_sparse"):
            assert torch.equal(getattr(s, name), getattr(e, name)), (new, name)
        assert s.status[0] == 0
        last = torch.cat([torch.arange(c, c + n) for c, n in zip(ctx, new)]).cuda()
        assert torch.equal((s.idx[:last.numel()] >= 0).sum(1), torch.clamp(last + 1, max=s.topk))  # the lengths of this step
        used = int(s.status[2])
        free = torch.cat([free[used:], free[:used]])
        for x in (s, e):
            x.ctx.copy_(x.total), x.free.copy_(free)
        ctx = [c + n for c, n in zip(ctx, new)]


def test_calls_of_several_kinds_at_once():
    """Pairs of tiles, selections by single tiles, few rows and the indexer on streams of their own, all of which share out an SM's tensor
    memory and shared memory among them."""
    calls = [Call(Step([3000, 500], [700, 401], 16, 2, 128, seed=1, q_gain=1.5)), Call(Step([2000], [150], 64, 1, 128, seed=2, q_gain=1.5), 700),
             Call(Step([900, 40], [30, 20], 16, 4, 64, seed=3, q_gain=1.5)), Call(Step([9000, 30, 4000], [2, 1, 1], 16, 4, 128, seed=4, q_gain=1.5))]
    g = torch.Generator(device="cuda").manual_seed(5)
    T, N, k = 256, 20000, 512
    q, w, x = (torch.randn(shape, generator=g, device="cuda").to(t) for shape, t in
               (((T, H, DI), torch.bfloat16), ((T, H), torch.float32), ((N, DI), torch.bfloat16)))
    idx, ws = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(
        lt.lt_indexer_topk_workspace_bytes("bf16", T, N, H, DI, k), dtype=torch.uint8, device="cuda")

    def index(stream=None):
        lt.lt_indexer_topk_ex("bf16", q, w, x, None, k, N - T, idx, None, ws, stream=stream)

    want = []
    for c in calls:
        c()
        want.append(c.results())
    index()
    want_idx = idx.clone()
    idx.fill_(-7)
    for c in calls:
        c.out.fill_(7.0), c.lse.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(len(calls) + 1)]
    for _ in range(15):
        for c, stream in zip(calls, streams):
            c(stream)
        index(streams[-1])
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert torch.equal(c.out[:int(c.s.start[-1])], w[0][:int(c.s.start[-1])]) and torch.equal(c.lse, w[1])
        assert lt.lt_read_status(c.ws) == [0] * 8
    assert torch.equal(idx, want_idx)
