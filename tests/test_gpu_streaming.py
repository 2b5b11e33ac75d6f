"""The windowed operators together (paper_2512_21835_gb300.streaming): generation with
recycled pages, against the oracle where the window covers everything, and against
itself with an unbounded pool where it does not."""
import numpy as np
import pytest

from gpu_util import argmax_agrees, need_gpu
from paper_2512_21835_gb300 import configs, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.mark.parametrize("model", ["tiny", "tiny-mha", "tiny-qk"])
def test_full_window_matches_the_oracle(torch, orc, model):
    """Prompt in two chunks, then decode steps: final hidden states within 3e-2 of the
    oracle's (the bound of the smoke run: two layers, a cache in bf16), tokens equal."""
    from paper_2512_21835_gb300.streaming import WindowedDecoder
    m = configs.MODELS[model]
    toks = inputs.token_ids(7, 90, m["vocab"])
    dec = WindowedDecoder(m, 1, 1000, 0, 128, chunk=48)
    outs = [dec.prefill(0, toks[:80])] + [dec.step([int(t)]) for t in toks[80:]]
    desc = orc.ModelDesc(**m)
    ref = orc.forward(desc, orc.Weights(desc, configs.WEIGHT_SEED), toks, n_prefill=80, prefill_flags=orc.KV_BF16,
                      decode_flags=orc.KV_BF16, want_logits=True)
    for i, (z, logits, tok) in enumerate(outs):
        assert np.max(np.abs(z.cpu().numpy()[0] - ref["hidden"][79 + i])) <= 3e-2
        assert argmax_agrees(int(tok[0]), logits.cpu().numpy()[0], ref["logits"][79 + i])


@pytest.mark.parametrize("window,sinks", [(100, 4), (64, 0), (130, 70)])
def test_recycled_pages_change_nothing(torch, window, sinks):
    """A pool just large enough for the window gives the bits of one that keeps every page."""
    from paper_2512_21835_gb300.streaming import PAGE, WindowedDecoder
    m, batch, n = configs.MODELS["tiny"], 2, 420
    prompts = inputs.prompts(3, batch, 300, m["vocab"])
    got = []
    for pages in (None, batch * -(-n // PAGE)):
        dec = WindowedDecoder(m, batch, window, sinks, n, chunk=70, n_pages=pages)
        last = [int(dec.prefill(r, p)[2][0]) for r, p in enumerate(prompts)]
        logits = []
        for _ in range(n - 300):
            _, lg, nxt = dec.step(last)
            logits.append(lg)
            last = nxt.tolist()
        got.append(torch.stack(logits).cpu().numpy())
        if pages is None:
            assert dec.pool.most < batch * (-(-n // PAGE))
    assert np.array_equal(*got)


def test_operators_back_to_back(torch):
    """Append, decode, append, ... without a wait in between: the bits of a run that waits after
    every call (each operator may be launched while its predecessor still runs)."""
    from paper_2512_21835_gb300 import loip as L
    Hq, Hkv, d, B, steps, ctx = 8, 2, 128, 6, 40, 300
    lpb = 2 * Hkv * 64 * d * 2
    pages = -(-(ctx + steps) // 64)
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn(steps, B, (Hq + 2 * Hkv) * d, device="cuda", generator=g)
    kv0 = torch.randn(B * pages * lpb // 2, device="cuda", generator=g).bfloat16()
    table = (torch.randperm(B * pages, device="cuda", generator=g) * lpb).view(B, pages)
    scratch = torch.zeros(L.loip_k_window_attention_scratch_bytes(B, Hq, Hkv, d, 200, 4, ctx + steps),
                          dtype=torch.uint8, device="cuda")
    pos = [torch.full((B,), ctx + i, dtype=torch.int32, device="cuda") for i in range(steps)]
    lens = [p + 1 for p in pos]
    got = []
    for wait in (True, False):
        kv, q = kv0.clone(), torch.empty(B, Hq * d, device="cuda")
        out = torch.empty(steps, B, Hq * d, device="cuda")
        torch.cuda.synchronize()
        for i in range(steps):
            L.loip_k_qk_append(qkv[i], None, None, Hq, Hkv, d, 0.0, 1e4, pos[i], None, q, kv, table, pages, 64, 0, lpb)
            if wait:
                torch.cuda.synchronize()
            L.loip_k_window_attention(q, kv, table, pages, lens[i], Hq, Hkv, d, 64, 0, lpb, 200, 4, ctx + steps, scratch,
                                      out[i])
            if wait:
                torch.cuda.synchronize()
        got.append((out.cpu().numpy(), kv.view(torch.int16).cpu().numpy()))
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
