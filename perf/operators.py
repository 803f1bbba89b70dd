"""A serving step over a key-value cache held in 4 bits, operator by operator: what is measured of each, its plain form
in elementary torch operations, and the same results in 64 bits.

  tables      lt_page_tables: block tables, slot map and positions of a step from the requests' lengths
  cache       lt_kv4_append + lt_kv4_read: rows of keys and values quantised into their slots, and read back
  attention   lt_kv4_attention: causal attention of ragged requests over their pages of the cache
  topk        lt_kv4_attention_topk: the same over the positions that an indexer selected for each token

The cache holds, for every page of 64 tokens and every key-value head, 64 rows of D + D / 8 bytes: D / 2 bytes of key
codes, D / 2 of value codes, then D / 32 key scales and D / 32 value scales in fp16.  A code is a nibble u (the even
element of a byte in its low half) that stands for (u - 8) * scale of its group of 32 elements.  The scale of a group is
its largest magnitude / 7 rounded to bf16, held in fp16, at most 2048; the code is the nearest integer to x / scale (ties
to even) within [-7, 7], plus 8; a group whose scale is 0 has all codes 8.
"""
import math

import torch

own = False

PAGE = 64   # tokens of a page
GROUP = 32  # elements that share a scale


def listed():
    return [
        # one decode step of an ordinary batch: every request adds a token, most stay within their last page
        dict(name="tables_step", op="tables", B=64, new_lo=1, new_hi=1, ctx_hi=32768, pad=0),
        # a scheduler that admits many prompts at once, in a buffer of fixed size
        dict(name="tables_admit", op="tables", B=701, new_lo=1, new_hi=1024, ctx_hi=8192, pad=333),
        # the keys and values of one decode step
        dict(name="cache_step", op="cache", dtype="bf16", T=64, Hkv=8, D=128, skip=0),
        # a large prefill chunk, some of its tokens without a slot
        dict(name="cache_chunk", op="cache", dtype="bf16", T=65536, Hkv=8, D=128, skip=57),
        # one token of one request: the smallest call there is, latency counts
        dict(name="attention_one", op="attention", dtype="bf16", B=1, new_lo=1, new_hi=1, ctx_lo=4096, ctx_hi=4096, Hq=32, Hkv=8, D=128, pad=0),
        # an ordinary decode step of a ragged batch
        dict(name="attention_step", op="attention", dtype="bf16", B=64, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=32768, Hq=64, Hkv=8, D=128, pad=0),
        # one token at the longest context
        dict(name="attention_1m", op="attention", dtype="bf16", B=1, new_lo=1, new_hi=1, ctx_lo=1048575, ctx_hi=1048575, Hq=64, Hkv=8, D=128, pad=0),
        # prefill chunks, drafted tokens and decoding requests in one padded batch, small heads
        dict(name="attention_mixed", op="attention", dtype="bf16", B=9, new_lo=1, new_hi=512, ctx_lo=0, ctx_hi=4096, Hq=32, Hkv=4, D=64, pad=77),
        # a chunk of a long prompt
        dict(name="attention_chunk", op="attention", dtype="bf16", B=1, new_lo=2048, new_hi=2048, ctx_lo=30720, ctx_hi=30720, Hq=32, Hkv=4, D=128, pad=0),
        # drafted tokens of a small model verified in fp32
        dict(name="attention_f32", op="attention", dtype="f32", B=4, new_lo=4, new_hi=4, ctx_lo=1000, ctx_hi=2000, Hq=16, Hkv=2, D=128, pad=0),
        # sparse attention of a decode step over the indexer's 2048 positions
        dict(name="topk_step", op="topk", dtype="bf16", B=32, new_lo=1, new_hi=1, ctx_lo=32768, ctx_hi=65536, Hq=64, Hkv=8, D=128, topk=2048, pad=0),
        # sparse attention of a prefill chunk, all query heads on one key-value head
        dict(name="topk_chunk", op="topk", dtype="bf16", B=1, new_lo=1024, new_hi=1024, ctx_lo=64512, ctx_hi=64512, Hq=64, Hkv=1, D=128, topk=2048, pad=0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "cache", "attention", "attention", "attention", "topk", "topk"])
    if op == "tables":
        return dict(op=op, B=_log_int(rng, 1, 701), new_lo=rng.choice([0, 1]), new_hi=_log_int(rng, 1, 1024), ctx_hi=_log_int(rng, 1, 32768), pad=rng.choice([0, 0, 100]))
    if op == "cache":
        T = _log_int(rng, 1, 65536)
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), T=T, Hkv=rng.choice([1, 2, 3, 4, 8]), D=rng.choice([64, 128]), skip=rng.choice([0, 0, T // 9]))
    Hkv = rng.choice([1, 2, 4, 8])
    D = rng.choice([64, 128, 128])
    kind = rng.choice(["step", "step", "draft", "chunk", "f32"])
    c = dict(op=op, dtype="f32" if kind == "f32" else "bf16", B=1, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0, Hq=Hkv * rng.choice([1, 3, 4, 5, 8, 8, 16]), Hkv=Hkv, D=D)
    if kind == "step":
        c["B"], c["ctx_hi"] = _log_int(rng, 1, 64), _log_int(rng, 16, 32768)
    elif kind == "draft":
        c["B"], c["ctx_hi"], c["new_lo"], c["new_hi"] = _log_int(rng, 1, 16), _log_int(rng, 64, 16384), 0, rng.randint(2, 8)
    elif kind == "chunk":
        c["B"], c["ctx_hi"], c["new_hi"] = _log_int(rng, 1, 8), _log_int(rng, 1, 8192), _log_int(rng, 16, 512 if op == "attention" else 128)
    else:
        c["B"], c["ctx_hi"], c["new_hi"], c["Hq"] = _log_int(rng, 1, 4), _log_int(rng, 1, 1024), rng.randint(1, 4), min(c["Hq"], 16 - 16 % Hkv)
    if op == "topk":
        c["topk"] = _log_int(rng, 1, 2048)
    c["pad"] = rng.choice([0, 0, 13])
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _lengths(case, g):
    """(tokens in the cache before the step, tokens of the step) of every request, on the host."""
    B = case["B"]

    def between(lo, hi, jitter):
        # spread evenly over the range, both ends among them, in random order
        x = torch.linspace(0, 1, B, dtype=torch.float64) if B > 1 else torch.ones(1, dtype=torch.float64)
        if jitter and B > 2:
            x[1:-1] += (torch.rand(B - 2, generator=g, dtype=torch.float64) - 0.5) / B
        return torch.round(lo + (hi - lo) * x).long()[torch.randperm(B, generator=g)]

    ctx = between(case.get("ctx_lo", 0), case["ctx_hi"], True)
    new = between(case["new_lo"], case["new_hi"], False)  # the step's tokens are as many whatever the seed
    if int(new.sum()) == 0:
        new[0] = 1
    return ctx, new


def _quantised(x, wide=None):
    """Codes (float, -7 .. 7) and scales of x [..., D]; the quotient is taken in `wide` (32 bits decide for bf16 values)."""
    x = x.float()
    groups = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    scale = (groups.abs().amax(-1, keepdim=True) / 7.0).bfloat16().float().clamp(max=2048.0).half()
    s = scale.to(wide or torch.float32)
    code = torch.where(s > 0, torch.round(groups.to(s.dtype) / s.clamp(min=2.0**-24)).clamp(-7, 7), torch.zeros_like(s)).float()
    return code, scale


def _rows(k, v):
    """The cache's rows (uint8 [..., D + D / 8]) of keys and values [..., D]."""
    parts = []
    scales = []
    for x in (k, v):
        code, scale = _quantised(x)
        u = (code + 8).to(torch.uint8).reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
        parts.append(u[..., 0] | (u[..., 1] << 4))
        scales.append(scale.squeeze(-1).contiguous().view(torch.uint8))
    return torch.cat(parts + scales, -1)


def _make_pool(pages, Hkv, D, g, dev):
    """A pool whose rows hold quantised keys and values: keys with a few channels larger than the others."""
    pool = torch.empty(pages, Hkv, PAGE, D + D // 8, dtype=torch.uint8, device=dev)
    loud = 1.0 + 3.0 * (torch.rand(Hkv, 1, D, generator=g, device=dev) < 0.04)
    step = max(1, (1 << 27) // (Hkv * PAGE * D))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        k = torch.randn(n, Hkv, PAGE, D, generator=g, device=dev) * loud
        v = torch.randn(n, Hkv, PAGE, D, generator=g, device=dev)
        pool[p:p + n] = _rows(k.bfloat16(), v.bfloat16())
    return pool


def prepare(case, seed):
    dev = "cuda"
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=dev).manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "cache":
        T, Hkv, D, dt = case["T"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
        pages = (T + PAGE - 1) // PAGE + 3
        loud = 1.0 + 3.0 * (torch.rand(1, Hkv, D, generator=g, device=dev) < 0.04)
        # the two thirds of a fused projection's rows that hold keys and values
        kv = torch.randn(T, 2, Hkv, D, generator=g, device=dev)
        kv[:, 0] *= loud
        st["kv"] = kv.to(dt)
        slots = torch.randperm(pages * PAGE, generator=g, device=dev)[:T].sort().values.to(torch.int32)
        if case["skip"]:
            slots[torch.randperm(T, generator=g, device=dev)[:case["skip"]]] = -1
        st["slots"] = slots
        st["pool"] = torch.zeros(pages, Hkv, PAGE, D + D // 8, dtype=torch.uint8, device=dev)
        st["k_out"] = torch.zeros(T, Hkv, D, dtype=dt, device=dev)
        st["v_out"] = torch.zeros(T, Hkv, D, dtype=dt, device=dev)
        return st
    ctx, new = _lengths(case, host)
    B, total = case["B"], int(new.sum())
    T = total + case["pad"]
    per = (ctx + new + PAGE - 1) // PAGE
    old = (ctx + PAGE - 1) // PAGE
    max_pages = (case["ctx_hi"] + case["new_hi"] + PAGE - 1) // PAGE + 1
    pages = int(per.sum()) + 5
    order = torch.randperm(pages, generator=host)
    first = torch.cumsum(per, 0) - per
    column = torch.arange(max_pages)[None]
    table = torch.where(column < per[:, None], order[(first[:, None] + column).clamp(max=pages - 1)], -1)
    i32 = dict(dtype=torch.int32, device=dev)
    st["ctx"], st["new"] = ctx.to(**i32), new.to(**i32)
    if case["op"] == "tables":
        # the pages in use are the front of the order, the free ones its back
        st["free"] = order.flip(0)[:int((per - old).sum()) + 3].to(**i32)
        taken = torch.cumsum(old, 0) - old
        st["table"] = torch.where(column < old[:, None], order[(taken[:, None] + column).clamp(max=pages - 1)], -1).to(**i32)
        st["total"], st["start"] = torch.zeros(B, **i32), torch.zeros(B + 1, **i32)
        st["slots"], st["position"] = torch.zeros(T, **i32), torch.zeros(T, **i32)
        st["status"] = torch.zeros(8, **i32)
        return st
    Hq, Hkv, D, dt = case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    st["table"] = table.to(**i32)
    st["pool"] = _make_pool(pages, Hkv, D, g, dev)
    st["start"] = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(new, 0)]).to(**i32)
    st["q"] = (1.5 * torch.randn(T, Hq, D, generator=g, device=dev)).to(dt)
    st["scale"] = 1.0 / math.sqrt(D)
    st["out"] = torch.zeros(T, Hq, D, dtype=dt, device=dev)
    st["lse"] = torch.zeros(T, Hq, dtype=torch.float32, device=dev)
    st["most_new"], st["most_keys"] = int(new.max()), int((ctx + new).max())
    if case["op"] == "topk":
        # what adjacent tokens select they share in large part; tokens that see fewer positions have their rows padded with -1
        k, width = case["topk"], max(case["topk"], int((ctx + new).max()))
        request = torch.repeat_interleave(torch.arange(B), new)
        sees = (ctx[request] + torch.arange(total) - (torch.cumsum(new, 0) - new)[request] + 1).to(dev)
        common = torch.rand(B, width, generator=g, device=dev)
        st["idx"] = torch.full((T, k), -1, **i32)
        for t in range(0, total, 256):
            e = min(total, t + 256)
            score = common[request[t:e].to(dev)] + 0.3 * torch.rand(e - t, width, generator=g, device=dev)
            score = score.masked_fill(torch.arange(width, device=dev)[None] >= sees[t:e, None], -1.0)
            best = score.topk(k, 1)
            st["idx"][t:e] = torch.where(best.values >= 0, best.indices, -1).to(torch.int32)
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _tables_plain(st):
    ctx, new, free, table = st["ctx"].long(), st["new"].long(), st["free"].long(), st["table"].long()
    B, T, max_pages = ctx.numel(), st["slots"].numel(), table.shape[1]
    total = ctx + new
    start = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    old, per = (ctx + PAGE - 1) // PAGE, (total + PAGE - 1) // PAGE
    first = torch.cumsum(per - old, 0) - (per - old)
    column = torch.arange(max_pages, device=ctx.device)[None]
    fresh = (column >= old[:, None]) & (column < per[:, None])
    table = torch.where(fresh, free[(first[:, None] + column - old[:, None]).clamp(0, free.numel() - 1)], table)
    token = torch.arange(T, device=ctx.device)
    request = torch.searchsorted(start[1:], token, right=True).clamp(max=B - 1)
    position = ctx[request] + token - start[request]
    slot = table[request, (position // PAGE).clamp(0, max_pages - 1)] * PAGE + position % PAGE
    real = token < start[-1]
    status = torch.zeros(8, dtype=torch.int64, device=ctx.device)
    status[1], status[2] = start[-1], (per - old).sum()
    minus = torch.full_like(token, -1)
    got = (table, total, start, torch.where(real, slot, minus), torch.where(real, position, minus), status)
    return tuple(x.to(torch.int32) for x in got)


def _cache_plain(st):
    kv, slots = st["kv"], st["slots"].long()
    code, scale = _quantised(kv, torch.float64 if kv.dtype == torch.float32 else torch.float32)
    values = (code * scale.float()).reshape(kv.shape) * (slots >= 0).float()[:, None, None, None]
    values = values.to(kv.dtype)
    return values[:, 0].contiguous(), values[:, 1].contiguous()


def _decoded(rows, D):
    """Keys and values (fp32) of cache rows uint8 [..., D + D / 8]."""
    codes = rows[..., :D].reshape(*rows.shape[:-1], 2, D // 2)
    codes = torch.stack([codes & 15, codes >> 4], -1).reshape(*rows.shape[:-1], 2, D // GROUP, GROUP).float() - 8.0
    scales = rows[..., D:].contiguous().view(torch.float16).reshape(*rows.shape[:-1], 2, D // GROUP, 1).float()
    kv = (codes * scales).reshape(*rows.shape[:-1], 2, D)
    return kv[..., 0, :], kv[..., 1, :]


def _softmax_plain(q, k, v, sees, scale):
    """q [..., R, D] over k, v [..., N, D] where `sees` holds; rows that see nothing give 0 and -inf."""
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(~sees, -math.inf)
    most = s.amax(-1, keepdim=True)
    most = torch.where(most == -math.inf, torch.zeros_like(most), most)
    p = s.sub_(most).exp_()
    norm = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / norm.clamp(min=1e-38)
    return o, (most + torch.log(norm)).squeeze(-1)


def _tokens(st):
    """Per token of the step: its request and its position in it; per request padded token numbers."""
    start = st["start"].long()
    total = st["q"].shape[0] - st["case"]["pad"]
    token = torch.arange(total, device=start.device)
    request = torch.searchsorted(start[1:], token, right=True)
    return token, request, st["ctx"].long()[request] + token - start[request]


def _attention_plain(st):
    c, q, start, ctx = st["case"], st["q"], st["start"].long(), st["ctx"].long()
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    R, P = st["most_new"], (st["most_keys"] + PAGE - 1) // PAGE
    new = start[1:] - start[:-1]
    row = torch.arange(R, device=q.device)
    token = (start[:-1, None] + row).clamp(max=q.shape[0] - 1)                              # [B, R]
    pages = st["pool"][st["table"].long()[:, :P].clamp(min=0)]                              # [B, P, Hkv, 64, row]
    k, v = _decoded(pages.transpose(1, 2).reshape(B, Hkv, P * PAGE, -1), D)
    qb = q.float()[token].reshape(B, R, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * R, D)
    last = (ctx[:, None] + row)[:, None, :].expand(B, Hq // Hkv, R).reshape(B, 1, -1, 1)
    sees = torch.arange(P * PAGE, device=q.device) <= last
    o, lse = _softmax_plain(qb, k, v, sees, st["scale"])
    o = o.reshape(B, Hq, R, D).transpose(1, 2)[row[None] < new[:, None]]                     # [tokens, Hq, D]
    lse = lse.reshape(B, Hq, R).transpose(1, 2)[row[None] < new[:, None]]
    out, out_lse = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"])
    out[:o.shape[0]], out_lse[:o.shape[0]] = o.to(out.dtype), lse
    return out, out_lse


def _topk_plain(st):
    c, q = st["case"], st["q"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    token, request, position = _tokens(st)
    idx = st["idx"].long()[:token.numel()]
    sees = (idx >= 0) & (idx <= position[:, None])
    at = idx.clamp(min=0)
    page = st["table"].long()[request[:, None], (at // PAGE).clamp(max=st["table"].shape[1] - 1)].clamp(min=0)
    rows = st["pool"][page, :, at % PAGE].transpose(1, 2)                                    # [tokens, Hkv, topk, row]
    k, v = _decoded(rows, D)
    qb = q.float()[:token.numel()].reshape(-1, Hkv, Hq // Hkv, D)
    o, lse = _softmax_plain(qb, k, v, sees[:, None, None], st["scale"])
    out, out_lse = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"])
    out[:token.numel()], out_lse[:token.numel()] = o.reshape(-1, Hq, D).to(out.dtype), lse.reshape(-1, Hq)
    return out, out_lse


PLAIN = {"tables": _tables_plain, "cache": _cache_plain, "attention": _attention_plain, "topk": _topk_plain}


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _call(st):
    """The calls that a user makes of the framework's operators."""
    from paper_2607_11976_b200 import binding as lt
    c = st["case"]
    if c["op"] == "tables":
        lt.lt_page_tables(st["ctx"], st["new"], st["free"], st["table"], st["total"], st["start"], st["slots"], st["position"], st["status"])
        return st["table"], st["total"], st["start"], st["slots"], st["position"], st["status"]
    if c["op"] == "cache":
        lt.lt_kv4_append(c["dtype"], st["kv"][:, 0], st["kv"][:, 1], st["slots"], st["pool"])
        lt.lt_kv4_read(c["dtype"], st["pool"], st["slots"], st["k_out"], st["v_out"])
        return st["k_out"], st["v_out"]
    if "workspace" not in st:  # once per program
        size = lt.lt_kv4_attention_workspace_bytes(c["dtype"], st["q"].shape[0], c["B"], c["Hq"], c["Hkv"], c["D"])
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    if c["op"] == "attention":
        lt.lt_kv4_attention(c["dtype"], st["q"], st["pool"], st["table"], st["start"], st["ctx"], st["scale"], st["out"], st["lse"], st["workspace"], max_new=c["new_hi"])
    else:
        lt.lt_kv4_attention_topk(c["dtype"], st["q"], st["pool"], st["table"], st["start"], st["ctx"], st["idx"], st["scale"], st["out"], st["lse"], st["workspace"])
    return st["out"], st["lse"]


def run(st):
    return _call(st) if own else PLAIN[st["case"]["op"]](st)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "cache":
        values = case["T"] * case["Hkv"] * case["D"] * 2
        size = 2 if case["dtype"] == "bf16" else 4
        # read, quantised, written to the cache, read there, written out
        return {"bytes": values * (2 * size + 2 * 9 / 16) + 8 * case["T"], "flops": 4 * values}
    ctx, new = _lengths(case, torch.Generator().manual_seed(0))
    total = int(new.sum())
    if case["op"] == "tables":
        fresh = int(((ctx + new + PAGE - 1) // PAGE - (ctx + PAGE - 1) // PAGE).sum())
        return {"bytes": 4 * (case["B"] * 5 + 2 * fresh + 2 * (total + case["pad"])), "flops": 0}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    row = D + D // 8
    q_and_out = total * Hq * (D * 2 * (2 if case["dtype"] == "bf16" else 4) + 4)
    if case["op"] == "attention":
        pairs = float((new.double() * ctx + new.double() * (new + 1) / 2).sum())
        keys = float((ctx + new)[new > 0].sum())
        return {"bytes": keys * Hkv * row + q_and_out, "flops": pairs * Hq * D * 4}
    request = torch.repeat_interleave(torch.arange(case["B"]), new)
    sees = ctx[request] + torch.arange(total) - (torch.cumsum(new, 0) - new)[request] + 1
    pairs = float(sees.clamp(max=case["topk"]).sum())
    # a request's tokens share its cache: no more than its keys have to come from memory
    keys = float(torch.minimum((ctx + new).double(), torch.zeros(case["B"], dtype=torch.float64).index_add_(0, request, sees.clamp(max=case["topk"]).double())).sum())
    return {"bytes": keys * Hkv * row + 4 * pairs + q_and_out, "flops": pairs * Hq * D * 4}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------------
def _exact_values(x):
    """What the cache keeps of x [..., D], in 64 bits: the nearest multiple of the group's scale, found among all of them."""
    D = x.shape[-1]
    flat = x.double().reshape(-1, GROUP)
    out = torch.empty_like(flat)
    multiples = torch.arange(-7, 8, dtype=torch.float64, device=x.device)
    for at in range(0, flat.shape[0], 1 << 18):
        f = flat[at:at + (1 << 18)]
        s = (f.abs().max(1).values.float() / 7.0).to(torch.bfloat16).double().clamp(max=2048.0)
        s = s.to(torch.float16).double()[:, None]
        best, far = torch.zeros_like(f), torch.full_like(f, math.inf)
        for m in multiples:
            d = (f - m * s).abs()
            nearer = (d < far) | ((d == far) & (m % 2 == 0))  # a tie goes to the even one
            best, far = torch.where(nearer, m * s, best), torch.where(nearer, d, far)
        out[at:at + (1 << 18)] = best
    return out.reshape(*x.shape[:-1], D)


def _exact_rows(rows, D):
    """Keys and values in 64 bits of cache rows [n, D + D / 8], nibble by nibble."""
    n = rows.shape[0]
    value = torch.arange(16, dtype=torch.float64, device=rows.device) - 8
    halves = []
    for j in range(2):
        b = rows[:, j * D // 2:(j + 1) * D // 2].long()
        x = torch.empty(n, D, dtype=torch.float64, device=rows.device)
        x[:, 0::2], x[:, 1::2] = value[b % 16], value[b // 16]
        scale = rows[:, D + j * D // 16:D + (j + 1) * D // 16].contiguous().view(torch.float16).double()
        halves.append(x * scale.repeat_interleave(GROUP, 1))
    return halves


def exact(case, seed):
    if case["op"] == "tables":
        return None  # whole numbers
    st = prepare(case, seed)
    if case["op"] == "cache":
        kv = _exact_values(st["kv"])
        kv[st["slots"] < 0] = 0
        return kv[:, 0], kv[:, 1]
    Hq, Hkv, D, scale = case["Hq"], case["Hkv"], case["D"], st["scale"]
    group = Hq // Hkv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    start, ctx = st["start"].tolist(), st["ctx"].tolist()

    def attend(t0, t1, h, k, v, hidden):
        q = st["q"][t0:t1, h * group:(h + 1) * group].double()
        s = torch.einsum("rgd,nd->rgn", q, k) * scale
        s[hidden[:, None, :].expand_as(s)] = -math.inf
        lse[t0:t1, h * group:(h + 1) * group] = torch.logsumexp(s, -1)
        out[t0:t1, h * group:(h + 1) * group] = torch.einsum("rgn,nd->rgd", torch.softmax(s, -1).nan_to_num(0.0), v)

    for b in range(case["B"]):
        n = ctx[b] + start[b + 1] - start[b]
        if start[b + 1] == start[b]:
            continue
        table = st["table"][b].long()
        position = torch.arange(n, device="cuda")
        page, offset = table[position // PAGE], position % PAGE
        for h in range(Hkv):
            k, v = _exact_rows(st["pool"][page, h, offset], D)
            if case["op"] == "attention":
                step = max(1, (1 << 28) // (group * n))
                for t in range(start[b], start[b + 1], step):
                    e = min(start[b + 1], t + step)
                    mine = ctx[b] + torch.arange(t, e, device="cuda") - start[b]
                    attend(t, e, h, k, v, position[None] > mine[:, None])
            else:
                for t in range(start[b], start[b + 1]):
                    i = st["idx"][t].long()
                    i = i[(i >= 0) & (i <= ctx[b] + t - start[b])]
                    attend(t, t + 1, h, k[i], v[i], torch.zeros(1, i.numel(), dtype=torch.bool, device="cuda"))
    return out, lse
