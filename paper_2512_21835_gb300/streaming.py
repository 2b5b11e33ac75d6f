"""Windowed generation with a bounded cache: the windowed-serving operators together.

    python -m paper_2512_21835_gb300.streaming [--model tiny] [--prompt N] [--new N]
                                               [--window N] [--sinks N] [--chunk N] [--batch N]
                                               [--cache bf16|q8]

A cache behind a sliding window with sinks stops growing, so its pages can be
recycled instead of pushing weights off the device as a growing cache does.  Each
layer appends its new tokens (loip_k_qk_append) and attends behind the window:
prompts in chunks (loip_k_window_prefill), then one token per request and step
(loip_k_window_attention).  A page that holds neither sinks nor positions that a later
token sees goes back to the pool; its page-table entry is not read again.  With
cache="q8" the cache holds 8 bits per element (loip_k_qk_append_q8 and the attentions
of that name), in 33/64 of the memory.

Weights are resident and generated (the shapes of configs.MODELS); up to 8 requests.
"""
from __future__ import annotations

import argparse
import time

import numpy as np

from . import configs

PAGE = 64


class PagePool:
    """Pages of a cache shared by several requests, and their page table (host side)."""

    def __init__(self, n_pages: int, requests: int, max_ctx: int, page_bytes: int):
        self.page_bytes, self.max_ctx = page_bytes, max_ctx
        self.max_pages = -(-max_ctx // PAGE)
        self.free = list(range(n_pages - 1, -1, -1))
        self.table = np.zeros((requests, self.max_pages), dtype=np.int64)  # byte offsets; 0 where no page is held
        self.held = [dict() for _ in range(requests)]  # page index in the request -> page of the pool
        self.most = 0

    def extend(self, request: int, first: int, last: int) -> None:
        """Pages for the positions first .. last of a request.  (The last page may have room past max_ctx, but
        the attention reads no key there.)"""
        if last >= self.max_ctx:
            raise ValueError(f"position {last} of request {request}: the context is {self.max_ctx} tokens")
        for i in range(first // PAGE, last // PAGE + 1):
            if i in self.held[request]:
                continue
            if not self.free:
                raise MemoryError(f"the page pool is exhausted at position {first} of request {request}")
            page = self.free.pop()
            self.held[request][i] = page
            self.table[request, i] = page * self.page_bytes
        self.most = max(self.most, sum(len(h) for h in self.held))

    def retire(self, request: int, next_pos: int, window: int, sinks: int) -> int:
        """Takes back the pages that no query at `next_pos` or later sees; returns how many."""
        gone = [i for i in self.held[request]
                if i * PAGE >= sinks and (i + 1) * PAGE <= next_pos - window + 1]
        for i in gone:
            self.free.append(self.held[request].pop(i))
            self.table[request, i] = 0
        return len(gone)


def pages_of_a_request(window: int, sinks: int, max_ctx: int, chunk: int) -> int:
    """Pages that the window, the sinks and a chunk can touch, and no more than the context has."""
    return min(-(-sinks // PAGE) + (window + chunk) // PAGE + 2, -(-max_ctx // PAGE))


class WindowedDecoder:
    """Greedy decoding of a resident model behind a sliding window with sinks."""

    def __init__(self, model: dict, batch: int, window: int, sinks: int, max_ctx: int, chunk: int = 256,
                 n_pages: int | None = None, seed: int = configs.WEIGHT_SEED, cache: str = "bf16"):
        import torch

        from . import build, loip
        build.build()
        self.torch, self.L = torch, loip
        if cache not in ("bf16", "q8"):
            raise ValueError(f"the cache is bf16 or q8, not {cache}")
        kind = "_q8" if cache == "q8" else ""
        self.append, self.attend, self.attend_chunk = (
            getattr(loip, f + kind) for f in ("loip_k_qk_append", "loip_k_window_attention", "loip_k_window_prefill"))
        m = self.m = dict(model)
        self.window, self.sinks, self.max_ctx, self.chunk = window, sinks, max_ctx, chunk
        H, F, d = m["hidden"], m["ffn"], m["head_dim"]
        self.qd, self.kvd = m["n_heads"] * d, m["n_kv_heads"] * d

        def gen(shape, tid, kind=0):
            t = torch.empty(shape, dtype=torch.int16, device="cuda")
            loip.loip_k_generate(t, 0, seed, tid, kind)
            return t

        self.embed, self.lm_head = gen((m["vocab"], H), 1), gen((m["vocab"], H), 2)
        self.g_final = gen((H,), 3, 1)
        self.layers = []
        for l in range(m["n_layers"]):
            t = 16 + 16 * l
            w = dict(g_attn=gen((H,), t, 1), wo=gen((H, self.qd), t + 4), g_mlp=gen((H,), t + 5, 1),
                     wg=gen((F, H), t + 6), wu=gen((F, H), t + 7), wd=gen((H, F), t + 8), g_q=None, g_k=None,
                     wqkv=torch.cat([gen((self.qd, H), t + 1), gen((self.kvd, H), t + 2), gen((self.kvd, H), t + 3)]))
            if m.get("qk_norm"):
                w.update(g_q=gen((d,), t + 9, 1), g_k=gen((d,), t + 10, 1))
            self.layers.append(w)
        # a page holds every layer's keys and values of 64 tokens
        self.layer_page_bytes = (loip.loip_k_cache_q8_layer_bytes(m["n_kv_heads"], d) if cache == "q8"
                                 else 2 * m["n_kv_heads"] * PAGE * d * 2)
        page_bytes = m["n_layers"] * self.layer_page_bytes
        if n_pages is None:
            n_pages = batch * pages_of_a_request(window, sinks, max_ctx, chunk)
        self.pool = PagePool(n_pages, batch, max_ctx, page_bytes)
        self.kv = torch.empty(n_pages * page_bytes, dtype=torch.uint8, device="cuda")
        heads = (m["n_heads"], m["n_kv_heads"], d, window, sinks, max_ctx)
        need = max(getattr(loip, f"loip_k_window_attention{kind}_scratch_bytes")(batch, *heads),
                   getattr(loip, f"loip_k_window_prefill{kind}_scratch_bytes")(chunk, 1, *heads))
        self.scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
        self.pos = [0] * batch

    def _ints(self, v):
        return self.torch.tensor(list(v), dtype=self.torch.int32, device="cuda")

    def _norm(self, x, g):
        torch = self.torch
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + self.m.get("rms_eps", 1e-5))
        return (x * r * g.view(torch.bfloat16).float()).contiguous()

    def _product(self, a, w, x):
        """x += a w^T: the streaming kernel for a few rows, the tensor cores at fp32 precision for more."""
        if a.shape[0] <= 8:
            self.L.loip_k_down(a, w, x)
            return
        bf = self.torch.bfloat16
        hi = a.to(bf)
        planes = self.torch.stack([hi, (a - hi.float()).to(bf)]).view(self.torch.int16)
        self.L.loip_k_gemm_split(planes, w, x)

    def _rows(self, tokens, rows, single):
        """The layers over the rows of one pass.  rows: (request, position) of each token; single: one row per
        request.  Returns the residual stream [rows, hidden]."""
        torch, L, m = self.torch, self.L, self.m
        T, H, F, d, Hq, Hkv = len(rows), m["hidden"], m["ffn"], m["head_dim"], m["n_heads"], m["n_kv_heads"]
        eps = m.get("rms_eps", 1e-5)
        table = torch.from_numpy(self.pool.table).cuda()
        reqs = sorted({r for r, _ in rows})
        positions, row_req = self._ints(p for _, p in rows), self._ints(r for r, _ in rows)
        if single:
            table_rows = table[reqs].contiguous()
            ctx = self._ints(p + 1 for _, p in rows)
        else:
            (r,) = reqs  # a chunk is of one prompt
            table_rows = table[r:r + 1].contiguous()
            starts, first = self._ints([0, T]), self._ints([rows[0][1]])
        x = torch.empty(T, H, device="cuda")
        L.loip_k_embed(self.embed, self._ints(tokens), x)
        q, o = torch.empty(T, self.qd, device="cuda"), torch.empty(T, self.qd, device="cuda")
        for l, w in enumerate(self.layers):
            qkv = torch.zeros(T, self.qd + 2 * self.kvd, device="cuda")
            self._product(self._norm(x, w["g_attn"]), w["wqkv"], qkv)
            self.append(qkv, w["g_q"], w["g_k"], Hq, Hkv, d, eps, m["rope_theta"], positions, row_req, q, self.kv, table,
                        self.pool.max_pages, PAGE, l, self.layer_page_bytes)
            if single:
                self.attend(q, self.kv, table_rows, self.pool.max_pages, ctx, Hq, Hkv, d, PAGE, l,
                            self.layer_page_bytes, self.window, self.sinks, self.max_ctx, self.scratch, o)
            else:
                self.attend_chunk(q, self.kv, table_rows, self.pool.max_pages, starts, first, Hq, Hkv, d, PAGE, l,
                                  self.layer_page_bytes, self.window, self.sinks, self.max_ctx, self.scratch, o)
            self._product(o, w["wo"], x)
            if T <= 8:
                a = torch.empty(T, F, device="cuda")
                L.loip_k_gate_up(x, w["g_mlp"], w["wg"], w["wu"], eps, a)
            else:
                y = self._norm(x, w["g_mlp"])
                gate, up = torch.zeros(T, F, device="cuda"), torch.zeros(T, F, device="cuda")
                self._product(y, w["wg"], gate)
                self._product(y, w["wu"], up)
                a = torch.nn.functional.silu(gate) * up
            self._product(a, w["wd"], x)
        return x

    def _head(self, x):
        """(final hidden states, logits, greedy tokens) of up to 8 rows."""
        torch, L, V = self.torch, self.L, self.m["vocab"]
        B = x.shape[0]
        z, logits = torch.empty_like(x), torch.empty(B, V, device="cuda")
        tokens = torch.empty(B, dtype=torch.int32, device="cuda")
        scratch = torch.empty(L.loip_k_lm_head_scratch_bytes(B, V), dtype=torch.uint8, device="cuda")
        L.loip_k_lm_head(x.contiguous(), self.g_final, self.lm_head, self.m.get("rms_eps", 1e-5), z, logits, tokens,
                         scratch)
        return z, logits, tokens

    def _take(self, tokens, more):
        """The tokens as whole numbers.  Refuses, before anything is enqueued for any of them, tokens that the
        vocabulary or the context has no place for; more: (request, how many of the tokens)."""
        tokens = [int(t) for t in tokens]
        for r, n in more:
            if not 0 <= r < len(self.pos):
                raise ValueError(f"request {r} of {len(self.pos)}")
            if self.pos[r] + n > self.max_ctx:
                raise ValueError(f"request {r} holds {self.pos[r]} tokens: no room for {n} more in a context of "
                                 f"{self.max_ctx}")
        if not tokens or len(tokens) != sum(n for _, n in more):
            raise ValueError(f"{len(tokens)} tokens for {sum(n for _, n in more)} rows")
        if min(tokens) < 0 or max(tokens) >= self.m["vocab"]:
            raise ValueError(f"tokens {min(tokens)} to {max(tokens)} of a vocabulary of {self.m['vocab']}")
        return tokens

    def prefill(self, request: int, prompt):
        """Takes a prompt in chunks; returns (hidden, logits, token) after its last token."""
        prompt = list(prompt)
        prompt = self._take(prompt, [(request, len(prompt))])
        for lo in range(0, len(prompt), self.chunk):
            part = prompt[lo:lo + self.chunk]
            first = self.pos[request]
            self.pool.extend(request, first, first + len(part) - 1)
            x = self._rows(part, [(request, first + i) for i in range(len(part))], single=False)
            self.pos[request] += len(part)
            self.pool.retire(request, self.pos[request], self.window, self.sinks)
        out = self._head(x[-1:])
        code = self.L.loip_k_attention_tc_status()
        if code:
            raise RuntimeError(f"the prompt attention gave up on a wait (code {code}): its rows are not complete")
        return out

    def step(self, tokens):
        """One token of every request; returns (hidden, logits, next tokens)."""
        tokens = self._take(tokens, [(r, 1) for r in range(len(self.pos))])
        rows = []
        for r, p in enumerate(self.pos):
            self.pool.extend(r, p, p)
            rows.append((r, p))
        x = self._rows(tokens, rows, single=True)
        for r in range(len(self.pos)):
            self.pos[r] += 1
            self.pool.retire(r, self.pos[r], self.window, self.sinks)
        return self._head(x)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", default="tiny", choices=sorted(configs.MODELS))
    ap.add_argument("--batch", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--new", type=int, default=200)
    ap.add_argument("--window", type=int, default=256)
    ap.add_argument("--sinks", type=int, default=4)
    ap.add_argument("--chunk", type=int, default=128)
    ap.add_argument("--cache", default="bf16", choices=["bf16", "q8"])
    a = ap.parse_args()
    import torch

    from . import inputs
    m = configs.MODELS[a.model]
    dec = WindowedDecoder(m, a.batch, a.window, a.sinks, a.prompt + a.new, a.chunk, cache=a.cache)
    last = [int(dec.prefill(r, p)[2][0]) for r, p in
            enumerate(inputs.prompts(configs.PROMPT_SEED, a.batch, a.prompt, m["vocab"]))]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(a.new):
        last = dec.step(last)[2].tolist()
    dt = time.perf_counter() - t0
    full = a.batch * -(-(a.prompt + a.new) // PAGE)
    print(f"{a.model}: {a.batch} x ({a.prompt} + {a.new}) tokens behind a window of {a.window} with {a.sinks} sinks: "
          f"{a.new * a.batch / dt:.1f} tokens/s, {dec.pool.most} pages of {dec.pool.page_bytes} bytes held at most "
          f"(without a window: {full})")


if __name__ == "__main__":
    main()
