"""Windowed generation over the 8-bit cache (paper_2512_21835_gb300.streaming): the four operators
as they are used together."""
import numpy as np
import pytest

from gpu_util import need_gpu
from paper_2512_21835_gb300 import configs, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.mark.parametrize("model", ["tiny", "tiny-qk"])
@pytest.mark.parametrize("window,sinks", [(100, 4), (130, 70)])
def test_recycled_pages_change_nothing(torch, model, window, sinks):
    """A pool just large enough for the window gives the bits of one that keeps every page, in 33/64 of the
    bf16 cache's memory."""
    from paper_2512_21835_gb300.streaming import PAGE, WindowedDecoder
    m, batch, n = configs.MODELS[model], 2, 420
    prompts = inputs.prompts(3, batch, 300, m["vocab"])
    got = []
    for pages in (None, batch * -(-n // PAGE)):
        dec = WindowedDecoder(m, batch, window, sinks, n, chunk=70, n_pages=pages, cache="q8")
        last = [int(dec.prefill(r, p)[2][0]) for r, p in enumerate(prompts)]
        logits = []
        for _ in range(n - 300):
            _, lg, nxt = dec.step(last)
            logits.append(lg)
            last = nxt.tolist()
        got.append(torch.stack(logits).cpu().numpy())
        if pages is None:
            assert dec.pool.most < batch * (-(-n // PAGE))
            bf16 = WindowedDecoder(m, batch, window, sinks, n, chunk=70)
            assert dec.kv.nbytes * 64 == bf16.kv.nbytes * 33
    assert np.all(np.isfinite(got[0])) and np.array_equal(*got)


def test_a_prefix_moves_to_another_cache(torch):
    """What one decoder has cached of a prompt, read back and appended to another one's cache in one
    chunk, continues as it would have: a row that is read back rounds to itself."""
    from paper_2512_21835_gb300 import loip as L
    from paper_2512_21835_gb300.streaming import PAGE, WindowedDecoder
    m, n, ctx = configs.MODELS["tiny"], 150, 256
    Hq, Hkv, d = m["n_heads"], m["n_kv_heads"], m["head_dim"]
    prompt = inputs.prompts(5, 1, n, m["vocab"])[0]
    a, b = (WindowedDecoder(m, 1, ctx, 0, ctx, chunk=64, cache="q8") for _ in range(2))
    token = int(a.prefill(0, prompt)[2][0])
    b.pool.free = b.pool.free[1:] + b.pool.free[:1]  # other pages than the first one's
    b.pool.extend(0, 0, n - 1)
    b.pos[0] = n
    tables = [torch.from_numpy(x.pool.table).cuda() for x in (a, b)]
    pos, req = torch.arange(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    rows = torch.zeros(n, (Hq + 2 * Hkv) * d, dtype=torch.bfloat16, device="cuda")
    held = torch.empty(n, 2 * Hkv * d, dtype=torch.bfloat16, device="cuda")
    q = torch.empty(n, Hq * d, dtype=torch.bfloat16, device="cuda")
    for l in range(m["n_layers"]):
        L.loip_k_cache_read_q8(a.kv, tables[0], a.pool.max_pages, pos, req, Hkv, d, PAGE, l, a.layer_page_bytes, held)
        rows[:, Hq * d:] = held
        L.loip_k_qk_append_q8(rows, None, None, Hq, Hkv, d, 0.0, 0.0, pos, req, q, b.kv, tables[1], b.pool.max_pages, PAGE,
                              l, b.layer_page_bytes)
    last = [token]
    for _ in range(20):
        (za, la, na), (zb, lb, nb) = a.step(last), b.step(last)
        assert torch.equal(za, zb) and torch.equal(la, lb) and torch.equal(na, nb)
        last = na.tolist()


def test_a_cache_of_another_kind_is_refused(torch):
    from paper_2512_21835_gb300.streaming import WindowedDecoder
    with pytest.raises(ValueError, match="bf16 or q8"):
        WindowedDecoder(configs.MODELS["tiny"], 1, 64, 0, 128, cache="fp8")
