"""The cache operators of windowed serving, and the sizes they are measured at.

Three operators share one paged key-value cache (pages of 64 tokens, keys then
values as [kv head][token][d] in bf16, found through a page table):

  append   norm of queries and keys for each head (optional), position rotation,
           and the new keys and values written into the cache; one row is one token
  decode   attention of one new token of each request over the cached positions
           it sees: the last `window` ones and the first `sinks` ones
  prefill  the same attention for the rows of prompts (or chunks of prompts),
           each row at its own position

The head layouts are those of the model shapes in configs.py.  A window of the
largest context is attention over everything.
"""
import math

import torch

own = False

PAGE = 64


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def listed():
    return [
        # one request's next token through an 8B-shaped layer: latency is all there is
        dict(name="append_1", op="append", rows=1, requests=1, Hq=32, Hkv=8, d=128, dtype="f32", norm=False, ctx=1088),
        # a decode step of eight requests with 70B heads, each at its own position
        dict(name="append_8", op="append", rows=8, requests=8, Hq=64, Hkv=8, d=128, dtype="bf16", norm=False, ctx=4352),
        # a prefill chunk of two prompts through a layer with norms of queries and keys
        dict(name="append_chunk", op="append", rows=1999, requests=2, Hq=64, Hkv=8, d=128, dtype="bf16", norm=True,
             ctx=4096),
        # a long prompt with one kv head per query head, in fp32 as the framework's activations are
        dict(name="append_long", op="append", rows=8191, requests=1, Hq=40, Hkv=40, d=128, dtype="f32", norm=False,
             ctx=8192),
        # one request at batch 1 over everything it has cached (the 8B decode workload)
        dict(name="decode_1", op="decode", batch=1, ctx_lo=1088, ctx_hi=1088, Hq=32, Hkv=8, d=128, dtype="f32",
             window=1088, sinks=0),
        # eight requests of 128 to 4352 tokens (the batched 70B workload), the cache bounded by a window
        dict(name="decode_8", op="decode", batch=8, ctx_lo=128, ctx_hi=4352, Hq=64, Hkv=8, d=128, dtype="f32",
             window=1024, sinks=4),
        # a serving batch with long contexts behind a 4096-token window
        dict(name="decode_64", op="decode", batch=64, ctx_lo=1000, ctx_hi=32768, Hq=64, Hkv=8, d=128, dtype="bf16",
             window=4096, sinks=64),
        # few requests over very long contexts, all of it visible: the split over the length has to fill the card
        dict(name="decode_long", op="decode", batch=4, ctx_lo=60001, ctx_hi=131072, Hq=32, Hkv=8, d=128, dtype="bf16",
             window=131072, sinks=0),
        # a short follow-up turn behind a kept conversation: few rows, latency counts
        dict(name="prefill_turn", op="prefill", rows=33, prompts=1, first=1055, Hq=32, Hkv=8, d=128, dtype="f32",
             window=512, sinks=4),
        # four prompts of 512 tokens, 70B heads, everything visible (the prefill workload)
        dict(name="prefill_4x512", op="prefill", rows=2048, prompts=4, first=0, even=True, Hq=64, Hkv=8, d=128,
             dtype="f32", window=512, sinks=0),
        # ragged prompts of a continuous batch, one kv head per query head
        dict(name="prefill_ragged", op="prefill", rows=5003, prompts=6, first=700, Hq=40, Hkv=40, d=128, dtype="bf16",
             window=1024, sinks=4),
        # the second half of a 16k prompt behind a 4096-token window
        dict(name="prefill_long", op="prefill", rows=8192, prompts=1, first=8192, Hq=32, Hkv=8, d=128, dtype="bf16",
             window=4096, sinks=4),
    ]


HEADS = [(4, 2, 64), (8, 2, 64), (20, 4, 64), (12, 4, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "prefill"])
    Hq, Hkv, d = rng.choice(HEADS)
    dtype = rng.choice(["f32", "bf16"])
    heads = dict(Hq=Hq, Hkv=Hkv, d=d, dtype=dtype)
    if op == "append":
        rows = _log(rng, 1, 8191)
        requests = rng.randint(1, min(rows, 16))
        return dict(op=op, rows=rows, requests=requests, norm=rng.random() < 0.5, ctx=rows + _log(rng, 1, 4096), **heads)
    window, sinks = _log(rng, 16, 8192), rng.choice([0, 0, 1, 4, 16, 64, 100])
    if op == "decode":
        batch = _log(rng, 1, 64)
        hi = _log(rng, 16, 131072)
        if rng.random() < 0.4:
            window = hi
        # at most the cached bytes that the longest listed case reads
        while batch * min(hi, window + sinks) * Hkv * d > 4 * 95000 * 8 * 128:
            batch, hi, window = max(1, batch // 2), max(1, hi * 2 // 3), max(16, window * 2 // 3)
        while batch * hi * Hkv * d > 4 * 131072 * 8 * 128 * 2:  # the cache that has to be laid out
            hi = hi * 2 // 3
        return dict(op=op, batch=batch, ctx_lo=rng.randint(1, hi), ctx_hi=hi, window=window, sinks=sinks, **heads)
    rows = _log(rng, 1, 8192)
    prompts = rng.randint(1, min(rows, 8))
    first = rng.choice([0, _log(rng, 1, 8192)])
    if rng.random() < 0.4:
        window = first + rows
    # at most the products of the longest listed case, and its score matrix in the plain form
    while (rows * min(first + rows, window + sinks) * Hq * d > 8192 * 4096 * 32 * 128
           or rows * (first + rows) * Hq > 8192 * 16384 * 32):
        rows, first = max(prompts, rows * 2 // 3), first * 2 // 3
    return dict(op=op, rows=rows, prompts=prompts, first=first, window=window, sinks=sinks, **heads)


# --------------------------------------------------------------------------
# what a case stands for, from its values alone
# --------------------------------------------------------------------------
def _split(total, parts, even):
    """`total` rows cut into `parts` runs of at least one row: equal, or growing with the index."""
    if even:
        ends = [total * (i + 1) // parts for i in range(parts)]
    else:
        weight = parts * (parts + 1) // 2
        ends = [(i + 1) + (total - parts) * ((i + 1) * (i + 2) // 2) // weight for i in range(parts)]
    return [e - s for s, e in zip([0] + ends[:-1], ends)]


def _contexts(case):
    """Context lengths of a decode case: spread evenly from ctx_lo to ctx_hi, out of order."""
    B, lo, hi = case["batch"], case["ctx_lo"], case["ctx_hi"]
    lens = [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]
    return [lens[(b * 7 + 3) % B] if B % 7 else lens[b] for b in range(B)]


def _prompts(case):
    """(rows, first position) of each prompt of a prefill case."""
    n = case["prompts"]
    lens = _split(case["rows"], n, case.get("even", False))
    return [(l, case["first"] * (i + 1) // n) for i, l in enumerate(lens)]


def _visible(pos, window, sinks):
    """How many cached positions a query at position `pos` sees."""
    return min(pos + 1, window + sinks)


def work(case):
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "append":
        T = case["rows"]
        elems = T * (Hq + 2 * Hkv) * d
        rotated = T * (Hq + Hkv) * d
        return {"bytes": elems * es + T * Hq * d * es + T * 2 * Hkv * d * 2 + T * 8,
                "flops": rotated * (3 + (4 if case["norm"] else 0))}
    if case["op"] == "decode":
        seen = sum(_visible(n - 1, case["window"], case["sinks"]) for n in _contexts(case))
        return {"bytes": seen * 2 * Hkv * d * 2 + case["batch"] * Hq * d * es * 2, "flops": 4 * seen * Hq * d}
    window, sinks = case["window"], case["sinks"]
    seen = read = 0
    for rows, first in _prompts(case):
        seen += sum(_visible(first + t, window, sinks) for t in range(rows))
        read += min(first + rows, rows - 1 + window + sinks)  # cached positions that some row of the prompt sees
    return {"bytes": read * 2 * Hkv * d * 2 + case["rows"] * Hq * d * es * 2, "flops": 4 * seen * Hq * d}


# --------------------------------------------------------------------------
# what a user's program has in hand
# --------------------------------------------------------------------------
def _cache(gen, dev, requests, positions, Hkv, d):
    """A filled cache of one layer with its pages scattered, and its page table."""
    pages = max(1, -(-positions // PAGE))
    order = torch.randperm(requests * pages, generator=gen, device=dev).view(requests, pages)
    kv = torch.empty(requests * pages, 2, Hkv, PAGE, d, dtype=torch.bfloat16, device=dev)
    kv.normal_(generator=gen)
    return kv, order


def _sink_direction(gen, dev, kv, order, Hkv, d, first_tokens):
    """Keys of the first tokens lie along a direction that the queries share, as in trained models."""
    u = torch.randn(Hkv, d, generator=gen, device=dev)
    n = min(first_tokens, PAGE)
    if n:
        kv[order[:, 0], 0, :, :n, :] = (0.5 * kv[order[:, 0], 0, :, :n, :].float() + 0.6 * u[:, None, :]).bfloat16()
    return u


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    G = Hq // Hkv
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    page_bytes = 2 * Hkv * PAGE * d * 2
    s = dict(op=case["op"], Hq=Hq, Hkv=Hkv, d=d, dtype=dt, page_bytes=page_bytes)
    if own:
        from paper_2512_21835_gb300 import loip
        s["loip"] = loip

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    if case["op"] == "append":
        T, R = case["rows"], case["requests"]
        lens = _split(T, R, False)
        kv, order = _cache(gen, dev, R, case["ctx"], Hkv, d)
        first = [(case["ctx"] - l) * (r + 1) // R for r, l in enumerate(lens)]
        s.update(qkv=(1.5 * torch.randn(T, (Hq + 2 * Hkv) * d, generator=gen, device=dev)).to(dt),
                 positions=ints([first[r] + t for r, l in enumerate(lens) for t in range(l)]),
                 row_req=ints([r for r, l in enumerate(lens) for _ in range(l)]),
                 g_q=None, g_k=None, eps=1e-6, theta=500000.0, q_out=torch.empty(T, Hq * d, dtype=dt, device=dev))
        if case["norm"]:
            s.update(g_q=(1 + 0.02 * torch.randn(d, generator=gen, device=dev)).bfloat16(),
                     g_k=(1 + 0.02 * torch.randn(d, generator=gen, device=dev)).bfloat16())
    elif case["op"] == "decode":
        lens = _contexts(case)
        kv, order = _cache(gen, dev, case["batch"], max(lens), Hkv, d)
        u = _sink_direction(gen, dev, kv, order, Hkv, d, case["sinks"])
        q = torch.randn(case["batch"], Hkv, G, d, generator=gen, device=dev) + 0.5 * u[None, :, None, :]
        s.update(q=q.reshape(case["batch"], Hq * d).to(dt), ctx_lens=ints(lens), max_ctx=max(lens),
                 o=torch.empty(case["batch"], Hq * d, dtype=dt, device=dev))
        if own:  # the workspace that a program keeps beside its buffers, zeroed once
            need = loip.loip_k_window_attention_scratch_bytes(case["batch"], Hq, Hkv, d, case["window"], case["sinks"],
                                                              max(lens))
            s["scratch"] = torch.zeros(need, dtype=torch.uint8, device=dev)
    else:
        runs = _prompts(case)
        M, n = case["rows"], len(runs)
        ends = [f + l for l, f in runs]
        kv, order = _cache(gen, dev, n, max(ends), Hkv, d)
        u = _sink_direction(gen, dev, kv, order, Hkv, d, case["sinks"])
        q = torch.randn(M, Hkv, G, d, generator=gen, device=dev) + 0.5 * u[None, :, None, :]
        starts = [sum(l for l, _ in runs[:i]) for i in range(n + 1)]
        s.update(q=q.reshape(M, Hq * d).to(dt), row_starts=ints(starts), first_pos=ints([f for _, f in runs]),
                 max_ctx=max(ends), longest=max(l for l, _ in runs),
                 o=torch.empty(M, Hq * d, dtype=dt, device=dev))
        if own:
            need = loip.loip_k_window_prefill_scratch_bytes(M, n, Hq, Hkv, d, case["window"], case["sinks"], max(ends))
            s["scratch"] = torch.zeros(need, dtype=torch.uint8, device=dev)
    s.update(kv=kv, pages=order, page_offsets=order.to(torch.int64) * page_bytes, max_pages=order.shape[1],
             window=case.get("window"), sinks=case.get("sinks"))
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["op"]](state)


def _own_append(s):
    s["loip"].loip_k_qk_append(s["qkv"], s["g_q"], s["g_k"], s["Hq"], s["Hkv"], s["d"], s["eps"], s["theta"],
                               s["positions"], s["row_req"], s["q_out"], s["kv"], s["page_offsets"], s["max_pages"],
                               PAGE, 0, s["page_bytes"])
    return [s["q_out"], s["kv"]]


def _own_decode(s):
    s["loip"].loip_k_window_attention(s["q"], s["kv"], s["page_offsets"], s["max_pages"], s["ctx_lens"], s["Hq"],
                                      s["Hkv"], s["d"], PAGE, 0, s["page_bytes"], s["window"], s["sinks"],
                                      s["max_ctx"], s["scratch"], s["o"])
    return s["o"]


def _own_prefill(s):
    s["loip"].loip_k_window_prefill(s["q"], s["kv"], s["page_offsets"], s["max_pages"], s["row_starts"],
                                    s["first_pos"], s["Hq"], s["Hkv"], s["d"], PAGE, 0, s["page_bytes"], s["window"],
                                    s["sinks"], s["max_ctx"], s["scratch"], s["o"])
    return s["o"]


_own = {"append": _own_append, "decode": _own_decode, "prefill": _own_prefill}


def _plain_append(s):
    Hq, Hkv, d, T = s["Hq"], s["Hkv"], s["d"], s["qkv"].shape[0]
    x = s["qkv"].float().view(T, Hq + 2 * Hkv, d)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if s["g_q"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s["eps"]) * s["g_q"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s["eps"]) * s["g_k"].float()
    # the angle is a product of a position and a frequency: 32 bits do not hold its turns, so it is formed in 64
    i = torch.arange(d // 2, device=x.device, dtype=torch.float64)
    angle = s["positions"].double()[:, None] * s["theta"] ** (-2.0 * i / d)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(y):
        a, b = y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)

    pos = s["positions"].long()
    page, slot = s["pages"][s["row_req"].long(), pos // PAGE], pos % PAGE
    s["kv"][page, 0, :, slot] = turn(k).bfloat16()
    s["kv"][page, 1, :, slot] = v.bfloat16()
    return [turn(q).reshape(T, Hq * d).to(s["dtype"]), s["kv"]]


def _plain_decode(s):
    Hq, Hkv, d, B = s["Hq"], s["Hkv"], s["d"], s["q"].shape[0]
    n = s["ctx_lens"].long()[:, None]
    j = torch.arange(min(s["max_ctx"], s["window"] + s["sinks"]), device=n.device)[None, :]
    pos = torch.where(j < s["sinks"], j, j + (n - s["window"] - s["sinks"]).clamp(min=0))
    seen = pos < n
    pos = pos.clamp(max=s["max_ctx"] - 1)
    page, slot = s["pages"].gather(1, pos // PAGE), pos % PAGE
    k, v = s["kv"][page, 0, :, slot].float(), s["kv"][page, 1, :, slot].float()  # [B, seen, Hkv, d]
    q = s["q"].float().view(B, Hkv, Hq // Hkv, d)
    a = torch.einsum("bhgd,bjhd->bhgj", q, k) / math.sqrt(d)
    a = a.masked_fill(~seen[:, None, None, :], -math.inf)
    p = torch.exp(a - a.amax(-1, keepdim=True))
    o = torch.einsum("bhgj,bjhd->bhgd", p, v) / p.sum(-1, keepdim=True)
    return o.reshape(B, Hq * d).to(s["dtype"])


def _plain_prefill(s):
    Hq, Hkv, d, M = s["Hq"], s["Hkv"], s["d"], s["q"].shape[0]
    start, first = s["row_starts"].long(), s["first_pos"].long()
    t = torch.arange(s["longest"], device=start.device)
    rows = (start[:-1, None] + t[None]).clamp(max=M - 1)  # [prompts, longest]: padded with rows that are dropped
    q = s["q"].float().view(M, Hkv, Hq // Hkv, d)[rows]
    j = torch.arange(s["max_ctx"], device=start.device)
    kv = s["kv"][s["pages"][:, j // PAGE], :, :, j % PAGE].float()  # [prompts, ctx, 2, Hkv, d]
    a = torch.einsum("nthgd,njhd->nhgtj", q, kv[:, :, 0]) / math.sqrt(d)
    pos = (first[:, None] + t[None])[:, :, None]
    seen = (j <= pos) & ((j < s["sinks"]) | (j > pos - s["window"]))
    a = a.masked_fill_(~seen[:, None, None], -math.inf)
    p = a.sub_(a.amax(-1, keepdim=True)).exp_()
    o = torch.einsum("nhgtj,njhd->nthgd", p, kv[:, :, 1]) / p.sum(-1).permute(0, 3, 1, 2)[..., None]
    live = torch.arange(M, device=start.device)
    n = torch.searchsorted(start[1:], live, right=True)
    return o[n, live - start[n]].reshape(M, Hq * d).to(s["dtype"])


_plain = {"append": _plain_append, "decode": _plain_decode, "prefill": _plain_prefill}


# --------------------------------------------------------------------------
# the definition, in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, d = s["Hq"], s["Hkv"], s["d"]
    G = Hq // Hkv
    if case["op"] == "append":
        x = s["qkv"].double()
        T = x.shape[0]
        turns = torch.tensor([[math.pow(s["theta"], -2.0 * i / d)] for i in range(d // 2)], dtype=torch.float64,
                             device=x.device) @ s["positions"].double()[None, :]
        z = torch.polar(torch.ones_like(turns), turns).T[:, None, :]  # [T, 1, d/2]: e^(i pos theta^(-2i/d))
        kv = s["kv"].double()

        def heads(lo, n, gain):
            y = x[:, lo * d:(lo + n) * d].reshape(T, n, d)
            if gain is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + s["eps"]) * gain.double()
            w = torch.complex(y[..., :d // 2], y[..., d // 2:]) * z
            return torch.cat([w.real, w.imag], dim=-1)

        q, k = heads(0, Hq, s["g_q"]), heads(Hq, Hkv, s["g_k"])
        v = x[:, (Hq + Hkv) * d:].reshape(T, Hkv, d)
        where = s["pages"][s["row_req"].long(), (s["positions"] // PAGE).long()]
        kv[where, 0, :, (s["positions"] % PAGE).long()] = k
        kv[where, 1, :, (s["positions"] % PAGE).long()] = v
        return [q.reshape(T, Hq * d), kv]

    # attention, one request and kv head at a time: queries `rows` at positions `pos`
    if case["op"] == "decode":
        runs = [(b, 1, n - 1) for b, n in enumerate(_contexts(case))]
    else:
        runs, row = [], 0
        for l, f in _prompts(case):
            runs.append((row, l, f))
            row += l
    q = s["q"].view(-1, Hkv, G, d)
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for r, (row, rows, first) in enumerate(runs):
        n = first + rows
        for h in range(Hkv):
            mine = s["kv"][s["pages"][r, :-(-n // PAGE)]]
            K = mine[:, 0, h].reshape(-1, d)[:n].double()
            V = mine[:, 1, h].reshape(-1, d)[:n].double()
            for lo in range(0, rows, 1024):  # rows are independent: a bounded piece of them at a time
                hi = min(rows, lo + 1024)
                i = first + torch.arange(lo, hi, device=q.device)[:, None]
                j = torch.arange(n, device=q.device)[None, :]
                hidden = (j > i) | ((j >= case["sinks"]) & (i - j >= case["window"]))
                a = q[row + lo:row + hi, h].double().reshape(-1, d) @ K.T * d ** -0.5
                a = a.view(hi - lo, G, n).masked_fill(hidden[:, None, :], -math.inf)
                out[row + lo:row + hi, h] = (torch.softmax(a, -1).view(-1, n) @ V).view(hi - lo, G, d)
    return out.reshape(-1, Hq * d)
