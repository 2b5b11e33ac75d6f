"""The operators of an 8-bit key-value cache, and the sizes they are measured at.

A row of the cache (a token's key or value of one kv head, d elements) is d / 32 blocks of 32
elements.  A block has an exponent byte E and 32 code bytes, sign and 7-bit magnitude m:

  value = +-m 2^(E - 133),  m = rint(|x| 2^(133 - E)),
  E the smallest (and 8 at least) for which no magnitude of the block exceeds 127

so that an element is off by half a step at most, and every value is a bf16 number.  E is at most
253: a block that holds something that is not finite, or 127.5 2^120 (1.7e38) or more, is stored
with E = 255, which stands for NaN in all its elements (as 254 would).  Pages of 64 tokens are
found through a page table; a layer's part of a page is [kv head][4 granules], a granule (16
tokens, 33 d bytes) is the codes of the keys [16][d], those of the values [16][d], the exponents
of the keys [16][d / 32] and those of the values.  The 16-byte piece c of token t's codes lies at
c ^ (t d / 128 % (d / 16)) in its row.

  store    norm of queries and keys for each head (optional), position rotation, the new keys
           and values quantised into the cache; then what the cache holds for them is read back
  read     rows of the cache as bf16 or fp32 numbers
  decode   attention of one new token of each request over the cached positions it
           sees: the last `window` ones and the first `sinks` ones
  prefill  the same attention for the rows of prompts (or chunks of prompts), each row
           at its own position

The head layouts are those of the model shapes in configs.py.  A window of the largest context is
attention over everything.
"""
import math

import torch

own = False

PAGE, GRANULE, BLOCK = 64, 16, 32


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def listed():
    return [
        # one request's next token through an 8B-shaped layer: latency is all there is
        dict(name="store_1", op="store", rows=1, requests=1, Hq=32, Hkv=8, d=128, dtype="f32", norm=False, ctx=640),
        # a prefill chunk of three prompts through a layer with norms of queries and keys
        dict(name="store_chunk", op="store", rows=1501, requests=3, Hq=64, Hkv=8, d=128, dtype="bf16", norm=True,
             ctx=2048),
        # a long prompt with one kv head per query head, in fp32 as the framework's activations are
        dict(name="store_long", op="store", rows=8191, requests=1, Hq=40, Hkv=40, d=128, dtype="f32", norm=False,
             ctx=8192),
        # the prefix of one request, to be kept elsewhere
        dict(name="read_prefix", op="read", rows=1087, requests=1, Hq=32, Hkv=8, d=128, dtype="bf16"),
        # a serving batch's whole cache of a layer, to be moved
        dict(name="read_batch", op="read", rows=100003, requests=9, Hq=64, Hkv=8, d=128, dtype="bf16"),
        # one request at batch 1 over everything it has cached (the end of the 8B decode workload)
        dict(name="decode_1", op="decode", batch=1, ctx_lo=640, ctx_hi=640, Hq=32, Hkv=8, d=128, dtype="f32",
             window=640, sinks=0),
        # eight requests of 128 to 4352 tokens (the batched 70B workload), everything visible
        dict(name="decode_8", op="decode", batch=8, ctx_lo=128, ctx_hi=4352, Hq=64, Hkv=8, d=128, dtype="f32",
             window=4352, sinks=0),
        # a serving batch with long contexts behind a 4096-token window
        dict(name="decode_96", op="decode", batch=96, ctx_lo=1000, ctx_hi=32768, Hq=64, Hkv=8, d=128, dtype="bf16",
             window=4096, sinks=64),
        # few requests over very long contexts, all of it visible: the split over the length has to fill the card
        dict(name="decode_long", op="decode", batch=5, ctx_lo=60001, ctx_hi=131072, Hq=32, Hkv=8, d=128, dtype="bf16",
             window=131072, sinks=0),
        # a short follow-up turn behind a kept conversation: few rows, latency counts
        dict(name="prefill_turn", op="prefill", rows=47, prompts=1, first=1041, Hq=32, Hkv=8, d=128, dtype="f32",
             window=1088, sinks=0),
        # ragged prompts of a continuous batch, one kv head per query head, each behind what it has cached
        dict(name="prefill_ragged", op="prefill", rows=4999, prompts=7, first=900, Hq=40, Hkv=40, d=128, dtype="bf16",
             window=1024, sinks=4),
        # the last chunk of a 16k prompt, all of it visible
        dict(name="prefill_long", op="prefill", rows=8192, prompts=1, first=8192, Hq=32, Hkv=8, d=128, dtype="bf16",
             window=16384, sinks=0),
    ]


HEADS = [(4, 2, 64), (8, 2, 64), (20, 4, 64), (12, 4, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "read", "decode", "prefill"])
    Hq, Hkv, d = rng.choice(HEADS)
    dtype = rng.choice(["f32", "bf16"])
    heads = dict(Hq=Hq, Hkv=Hkv, d=d, dtype=dtype)
    if op == "store":
        rows = _log(rng, 1, 8191)
        requests = rng.randint(1, min(rows, 16))
        return dict(op=op, rows=rows, requests=requests, norm=rng.random() < 0.5, ctx=rows + _log(rng, 1, 4096), **heads)
    if op == "read":
        rows = _log(rng, 16, 100003)
        while rows * Hkv * d * (3 if dtype == "bf16" else 5) > 100003 * 8 * 128 * 3:
            rows = rows * 2 // 3
        return dict(op=op, rows=rows, requests=rng.randint(1, min(rows, 16)), **heads)
    window, sinks = _log(rng, 16, 8192), rng.choice([0, 0, 1, 4, 16, 64, 100])
    if op == "decode":
        batch = _log(rng, 1, 96)
        hi = _log(rng, 16, 131072)
        if rng.random() < 0.4:
            window = hi
        # at most the cached bytes that the longest listed case reads
        while batch * min(hi, window + sinks) * Hkv * d > 5 * 95000 * 8 * 128:
            batch, hi, window = max(1, batch // 2), max(1, hi * 2 // 3), max(16, window * 2 // 3)
        while batch * hi * Hkv * d > 5 * 131072 * 8 * 128 * 2:  # the cache that has to be laid out
            hi = hi * 2 // 3
        return dict(op=op, batch=batch, ctx_lo=rng.randint(1, hi), ctx_hi=hi, window=window, sinks=sinks, **heads)
    rows = _log(rng, 1, 8192)
    prompts = rng.randint(1, min(rows, 8))
    first = rng.choice([0, _log(rng, 1, 8192)])
    if rng.random() < 0.4:
        window = first + rows
    # at most a part of the products of the longest listed case, and of its score matrix in the plain form
    while (rows * min(first + rows, window + sinks) * Hq * d > 8192 * 4096 * 32 * 128
           or rows * (first + rows) * Hq > 8192 * 12288 * 32):
        rows, first = max(prompts, rows * 2 // 3), first * 2 // 3
    return dict(op=op, rows=rows, prompts=prompts, first=first, window=window, sinks=sinks, **heads)


# --------------------------------------------------------------------------
# what a case stands for, from its values alone
# --------------------------------------------------------------------------
def _split(total, parts):
    """`total` rows cut into `parts` runs of at least one row, growing with the index."""
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
    return [(l, case["first"] * (i + 1) // n) for i, l in enumerate(_split(case["rows"], n))]


def work(case):
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    es = 4 if case["dtype"] == "f32" else 2
    held = 2 * Hkv * (d + d // BLOCK)  # cached bytes of a token
    if case["op"] == "store":
        T = case["rows"]
        return {"bytes": T * ((Hq + 2 * Hkv) * d * es + Hq * d * es + held + 2 * Hkv * d * 2 + 8),
                "flops": T * (Hq + Hkv) * d * (3 + (4 if case["norm"] else 0)) + T * 2 * Hkv * d * 2}
    if case["op"] == "read":
        return {"bytes": case["rows"] * (held + 2 * Hkv * d * es + 8), "flops": case["rows"] * 2 * Hkv * d}
    window, sinks = case["window"], case["sinks"]
    if case["op"] == "decode":
        seen = sum(min(n, window + sinks) for n in _contexts(case))
        return {"bytes": seen * held + case["batch"] * Hq * d * es * 2, "flops": 4 * seen * Hq * d}
    seen = read = 0
    for rows, first in _prompts(case):
        seen += sum(min(first + t + 1, window + sinks) for t in range(rows))
        read += min(first + rows, rows - 1 + window + sinks)  # cached positions that some row of the prompt sees
    return {"bytes": read * held + case["rows"] * Hq * d * es * 2, "flops": 4 * seen * Hq * d}


# --------------------------------------------------------------------------
# the cache's bytes, with elementary operations
# --------------------------------------------------------------------------
def _pieces(kv, is_v, d):
    """The codes of the keys or values of a cache [pages, kv heads, 4, 33 d] as [pages, kv heads, 4, 16, pieces, 16]."""
    return kv[..., is_v * GRANULE * d:(is_v + 1) * GRANULE * d].unflatten(-1, (GRANULE, d // 16, 16))


def _exponents(kv, is_v, d):
    at, n = 2 * GRANULE * d + is_v * GRANULE * (d // BLOCK), d // BLOCK
    return kv[..., at:at + GRANULE * n].unflatten(-1, (GRANULE, n))


def _place(slot, d):
    """Where the 16-byte pieces of a token's row lie: [..., pieces]."""
    c = torch.arange(d // 16, device=slot.device)
    return c ^ (slot * d // 128 % (d // 16))[..., None]


def _encode(x):
    """Codes [..., d] and exponents [..., d / 32] of rows of fp32 or fp64 numbers.  Powers of two scale exactly."""
    b = x.unflatten(-1, (-1, BLOCK))
    most = b.abs().amax(-1, keepdim=True)
    _, e = torch.frexp(torch.where(most.isfinite(), most, 1.0))  # most = f 2^e with f in [1/2, 1)
    E = e + 126
    E = (E + (torch.ldexp(most, 133 - E) >= 127.5)).clamp(min=8)
    bad = ~most.isfinite() | (E > 253)
    E = torch.where(bad, 255, E)
    m = torch.where(bad, 0.0, torch.ldexp(torch.where(bad, 0.0, b), 133 - E).round())
    codes = m.abs().to(torch.uint8) | ((m < 0).to(torch.uint8) << 7)
    return codes.flatten(-2), E.squeeze(-1).to(torch.uint8)


def _decode(codes, exps):
    """fp32 numbers of codes [..., d] and exponents [..., d / 32]."""
    m = (codes & 127).float()
    m = torch.where(codes > 127, -m, m)
    step = ((exps.int().clamp(min=7) - 6) << 23).view(torch.float32)  # the fp32 number 2^(E - 133)
    step = torch.where(exps >= 254, math.nan, step)
    return (m.unflatten(-1, (-1, BLOCK)) * step[..., None]).flatten(-2)


def _held(s, page, slot):
    """Keys and values (fp32 [..., kv heads, d]) that the cache holds at (page, slot)."""
    d, g, t = s["d"], slot // GRANULE, slot % GRANULE
    place = _place(t, d)

    def rows(is_v):
        codes = _pieces(s["kv"], is_v, d)[page[..., None], :, g[..., None], t[..., None], place]  # [..., pieces, kv heads, 16]
        codes = codes.transpose(-2, -3).flatten(-2)
        return _decode(codes, _exponents(s["kv"], is_v, d)[page, :, g, t])

    return rows(0), rows(1)


# --------------------------------------------------------------------------
# what a user's program has in hand
# --------------------------------------------------------------------------
def _cache(gen, dev, requests, positions, Hkv, d, sinks=0):
    """A filled cache of one layer with its pages scattered, its page table, and the directions along which the
    keys of the first tokens lie (the queries share them, as in trained models)."""
    pages = max(1, -(-positions // PAGE))
    n = requests * pages
    order = torch.randperm(n, generator=gen, device=dev).view(requests, pages)
    u = torch.randn(Hkv, d, generator=gen, device=dev)
    kv = torch.empty(n, Hkv, PAGE // GRANULE, 33 * d, dtype=torch.uint8, device=dev)
    t = torch.arange(GRANULE, device=dev)
    place = _place(t, d)
    first = torch.zeros(n, dtype=torch.bool, device=dev)
    first[order[:, 0]] = True
    early = (torch.arange(PAGE, device=dev) < sinks).view(PAGE // GRANULE, GRANULE, 1)
    step = max(1, (64 << 20) // (Hkv * PAGE * d))
    for lo in range(0, n, step):  # a bounded piece of the pages at a time
        part = kv[lo:lo + step]
        for is_v in (0, 1):
            x = torch.randn(part.shape[0], Hkv, PAGE // GRANULE, GRANULE, d, generator=gen, device=dev)
            if not is_v and sinks:
                lie = first[lo:lo + step, None, None, None, None] & early
                x = torch.where(lie, 0.5 * x + 0.6 * u[:, None, None, :], x)
            codes, exps = _encode(x)
            _pieces(part, is_v, d)[:, :, :, t[:, None], place] = codes.unflatten(-1, (-1, 16))
            _exponents(part, is_v, d).copy_(exps)
    return kv, order, u


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    G = Hq // Hkv
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    page_bytes = Hkv * (PAGE // GRANULE) * 33 * d
    s = dict(op=case["op"], Hq=Hq, Hkv=Hkv, d=d, dtype=dt, page_bytes=page_bytes)
    if own:
        from paper_2512_21835_gb300 import loip
        s["loip"] = loip

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    if case["op"] in ("store", "read"):
        T, R = case["rows"], case["requests"]
        lens = _split(T, R)
        ctx = case["ctx"] if case["op"] == "store" else max(lens)
        kv, order, _ = _cache(gen, dev, R, ctx, Hkv, d)
        first = [(ctx - l) * (r + 1) // R if case["op"] == "store" else 0 for r, l in enumerate(lens)]
        s.update(positions=torch.cat([torch.arange(f, f + l, dtype=torch.int32, device=dev) for f, l in zip(first, lens)]),
                 row_req=torch.repeat_interleave(torch.arange(R, dtype=torch.int32, device=dev),
                                                 torch.tensor(lens, device=dev)))
        if case["op"] == "read":
            s["kv_out"] = torch.empty(T, 2 * Hkv * d, dtype=dt, device=dev)
        else:
            s.update(qkv=(1.5 * torch.randn(T, (Hq + 2 * Hkv) * d, generator=gen, device=dev)).to(dt),
                     g_q=None, g_k=None, eps=1e-6, theta=500000.0, q_out=torch.empty(T, Hq * d, dtype=dt, device=dev),
                     # what is read back is exact in bf16
                     kv_out=torch.empty(T, 2 * Hkv * d, dtype=torch.bfloat16, device=dev))
            if case["norm"]:
                s.update(g_q=(1 + 0.02 * torch.randn(d, generator=gen, device=dev)).bfloat16(),
                         g_k=(1 + 0.02 * torch.randn(d, generator=gen, device=dev)).bfloat16())
    elif case["op"] == "decode":
        lens = _contexts(case)
        kv, order, u = _cache(gen, dev, case["batch"], max(lens), Hkv, d, case["sinks"])
        q = torch.randn(case["batch"], Hkv, G, d, generator=gen, device=dev) + 0.5 * u[None, :, None, :]
        s.update(q=q.reshape(case["batch"], Hq * d).to(dt), ctx_lens=ints(lens), max_ctx=max(lens),
                 o=torch.empty(case["batch"], Hq * d, dtype=dt, device=dev))
        if own:  # the workspace that a program keeps beside its buffers, zeroed once
            need = loip.loip_k_window_attention_q8_scratch_bytes(case["batch"], Hq, Hkv, d, case["window"],
                                                                 case["sinks"], max(lens))
            s["scratch"] = torch.zeros(need, dtype=torch.uint8, device=dev)
    else:
        runs = _prompts(case)
        M, n = case["rows"], len(runs)
        ends = [f + l for l, f in runs]
        kv, order, u = _cache(gen, dev, n, max(ends), Hkv, d, case["sinks"])
        q = torch.randn(M, Hkv, G, d, generator=gen, device=dev) + 0.5 * u[None, :, None, :]
        starts = [sum(l for l, _ in runs[:i]) for i in range(n + 1)]
        s.update(q=q.reshape(M, Hq * d).to(dt), row_starts=ints(starts), first_pos=ints([f for _, f in runs]),
                 max_ctx=max(ends), longest=max(l for l, _ in runs),
                 o=torch.empty(M, Hq * d, dtype=dt, device=dev))
        if own:
            need = loip.loip_k_window_prefill_q8_scratch_bytes(M, n, Hq, Hkv, d, case["window"], case["sinks"],
                                                               max(ends))
            s["scratch"] = torch.zeros(need, dtype=torch.uint8, device=dev)
    s.update(kv=kv, pages=order, page_offsets=order.to(torch.int64) * page_bytes, max_pages=order.shape[1],
             window=case.get("window"), sinks=case.get("sinks"))
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["op"]](state)


def _own_read(s):
    s["loip"].loip_k_cache_read_q8(s["kv"], s["page_offsets"], s["max_pages"], s["positions"], s["row_req"], s["Hkv"],
                                   s["d"], PAGE, 0, s["page_bytes"], s["kv_out"])
    return s["kv_out"]


def _own_store(s):
    s["loip"].loip_k_qk_append_q8(s["qkv"], s["g_q"], s["g_k"], s["Hq"], s["Hkv"], s["d"], s["eps"], s["theta"],
                                  s["positions"], s["row_req"], s["q_out"], s["kv"], s["page_offsets"],
                                  s["max_pages"], PAGE, 0, s["page_bytes"])
    return [s["q_out"], _own_read(s)]


def _own_decode(s):
    s["loip"].loip_k_window_attention_q8(s["q"], s["kv"], s["page_offsets"], s["max_pages"], s["ctx_lens"], s["Hq"],
                                         s["Hkv"], s["d"], PAGE, 0, s["page_bytes"], s["window"], s["sinks"],
                                         s["max_ctx"], s["scratch"], s["o"])
    return s["o"]


def _own_prefill(s):
    s["loip"].loip_k_window_prefill_q8(s["q"], s["kv"], s["page_offsets"], s["max_pages"], s["row_starts"],
                                       s["first_pos"], s["Hq"], s["Hkv"], s["d"], PAGE, 0, s["page_bytes"],
                                       s["window"], s["sinks"], s["max_ctx"], s["scratch"], s["o"])
    return s["o"]


_own = {"store": _own_store, "read": _own_read, "decode": _own_decode, "prefill": _own_prefill}


def _plain_read(s):
    pos = s["positions"].long()
    k, v = _held(s, s["pages"][s["row_req"].long(), pos // PAGE], pos % PAGE)
    return torch.cat([k, v], dim=1).flatten(1).to(s["kv_out"].dtype)


def _plain_store(s):
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
    page, g, t = s["pages"][s["row_req"].long(), pos // PAGE], pos % PAGE // GRANULE, pos % GRANULE

    def put(y, is_v):
        codes, exps = _encode(y)
        pieces = codes.unflatten(-1, (-1, 16)).transpose(1, 2)  # [rows, pieces, kv heads, 16]
        _pieces(s["kv"], is_v, d)[page[:, None], :, g[:, None], t[:, None], _place(t, d)] = pieces
        _exponents(s["kv"], is_v, d)[page, :, g, t] = exps

    put(turn(k), 0)
    put(v, 1)
    return [turn(q).reshape(T, Hq * d).to(s["dtype"]), _plain_read(s)]


def _plain_decode(s):
    Hq, Hkv, d, B = s["Hq"], s["Hkv"], s["d"], s["q"].shape[0]
    n = s["ctx_lens"].long()[:, None]
    j = torch.arange(min(s["max_ctx"], s["window"] + s["sinks"]), device=n.device)[None, :]
    pos = torch.where(j < s["sinks"], j, j + (n - s["window"] - s["sinks"]).clamp(min=0))
    seen = pos < n
    pos = pos.clamp(max=s["max_ctx"] - 1)
    k, v = _held(s, s["pages"].gather(1, pos // PAGE), pos % PAGE)  # [B, seen, Hkv, d]
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
    k, v = _held(s, s["pages"][:, j // PAGE], (j % PAGE).expand(start.numel() - 1, -1))  # [prompts, ctx, Hkv, d]
    a = torch.einsum("nthgd,njhd->nhgtj", q, k).div_(math.sqrt(d))
    pos = (first[:, None] + t[None])[:, :, None]
    seen = (j <= pos) & ((j < s["sinks"]) | (j > pos - s["window"]))
    a = a.masked_fill_(~seen[:, None, None], -math.inf)
    p = a.sub_(a.amax(-1, keepdim=True)).exp_()
    o = torch.einsum("nhgtj,njhd->nthgd", p, v) / p.sum(-1).permute(0, 3, 1, 2)[..., None]
    live = torch.arange(M, device=start.device)
    n = torch.searchsorted(start[1:], live, right=True)
    return o[n, live - start[n]].reshape(M, Hq * d).to(s["dtype"])


_plain = {"store": _plain_store, "read": _plain_read, "decode": _plain_decode, "prefill": _plain_prefill}


# --------------------------------------------------------------------------
# the definition, in 64 bits
# --------------------------------------------------------------------------
def _exact_rows(s, pages, pos, head, is_v):
    """fp64 rows [n, d] of one kv head at `pos`, each byte looked up by its address."""
    Hkv, d = s["Hkv"], s["d"]
    dev = pos.device
    bytes_ = s["kv"].view(-1)
    value = torch.tensor([c if c < 128 else 128 - c for c in range(256)], dtype=torch.float64, device=dev)
    step = torch.tensor([2.0 ** (E - 133) for E in range(254)] + 2 * [math.nan], dtype=torch.float64, device=dev)
    start = ((pages * Hkv + head) * 4 + pos % 64 // 16) * (33 * d)
    t, i = (pos % 16)[:, None], torch.arange(d, device=dev)[None, :]
    code = start[:, None] + is_v * 16 * d + t * d + ((i // 16) ^ (t * d // 128 % (d // 16))) * 16 + i % 16
    exp = start[:, None] + 32 * d + is_v * (d // 2) + t * (d // 32) + i // 32
    return value[bytes_[code].long()] * step[bytes_[exp].long()]


def _exact_rounded(y):
    """fp64 numbers to what 32 of them share an exponent for, by halving and doubling steps."""
    b = y.reshape(*y.shape[:-1], -1, 32)
    most = b.abs().amax(-1, keepdim=True)
    step = torch.full_like(most, 2.0 ** -125)
    while bool((over := most / step >= 127.5).any()):
        step = torch.where(over, 2 * step, step)
    return (torch.round(b / step) * step).reshape(y.shape)


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, d = s["Hq"], s["Hkv"], s["d"]
    G = Hq // Hkv
    if case["op"] == "read":
        pos = s["positions"].long()
        pages = s["pages"][s["row_req"].long(), pos // 64]
        heads = [_exact_rows(s, pages, pos, h, is_v) for is_v in (0, 1) for h in range(Hkv)]
        return torch.stack(heads, dim=1).reshape(pos.numel(), -1)
    if case["op"] == "store":
        x = s["qkv"].double()
        T = x.shape[0]
        turns = torch.tensor([[math.pow(s["theta"], -2.0 * i / d)] for i in range(d // 2)], dtype=torch.float64,
                             device=x.device) @ s["positions"].double()[None, :]
        z = torch.polar(torch.ones_like(turns), turns).T[:, None, :]  # [T, 1, d/2]: e^(i pos theta^(-2i/d))

        def heads(lo, n, gain):
            y = x[:, lo * d:(lo + n) * d].reshape(T, n, d)
            if gain is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + s["eps"]) * gain.double()
            w = torch.complex(y[..., :d // 2], y[..., d // 2:]) * z
            return torch.cat([w.real, w.imag], dim=-1)

        q, k = heads(0, Hq, s["g_q"]), heads(Hq, Hkv, s["g_k"])
        v = x[:, (Hq + Hkv) * d:].reshape(T, Hkv, d)
        return [q.reshape(T, Hq * d), torch.cat([_exact_rounded(k), _exact_rounded(v)], dim=1).reshape(T, -1)]

    # attention, one request and kv head at a time: queries `rows` at positions `pos`
    if case["op"] == "decode":
        runs = [(b, 1, n - 1) for b, n in enumerate(_contexts(case))]
    else:
        runs, row = [], 0
        for l, f in _prompts(case):
            runs.append((row, l, f))
            row += l
    window, sinks = case["window"], case["sinks"]
    q = s["q"].view(-1, Hkv, G, d)
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for r, (row, rows, first) in enumerate(runs):
        n = first + rows
        j = torch.arange(n, device=q.device)
        j = j[(j < sinks) | (j > first - window)]  # what the first row or a later one sees
        for h in range(Hkv):
            pages = s["pages"][r][j // 64]
            K, V = _exact_rows(s, pages, j, h, 0), _exact_rows(s, pages, j, h, 1)
            for lo in range(0, rows, 1024):  # rows are independent: a bounded piece of them at a time
                hi = min(rows, lo + 1024)
                i = first + torch.arange(lo, hi, device=q.device)[:, None]
                hidden = (j[None, :] > i) | ((j[None, :] >= sinks) & (i - j[None, :] >= window))
                a = q[row + lo:row + hi, h].double().reshape(-1, d) @ K.T * d ** -0.5
                a = a.view(hi - lo, G, -1).masked_fill(hidden[:, None, :], -math.inf)
                out[row + lo:row + hi, h] = (torch.softmax(a, -1).view(-1, j.numel()) @ V).view(hi - lo, G, d)
    return out.reshape(-1, Hq * d)
