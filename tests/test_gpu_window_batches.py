"""Batches that change from call to call, with one scratch that is sized for the largest,
and batches of one long request among short ones."""
import numpy as np
import pytest

import window_ref as W
from gpu_util import need_gpu
from test_gpu_window import _decode, _decode_cache, _host, _prefill, _prefill_cache, _rows

pytestmark = pytest.mark.gpu

ALL = 1 << 30


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.fixture(scope="module")
def L(torch):
    from paper_2512_21835_gb300 import loip
    return loip


def test_a_draining_batch_keeps_its_scratch(torch, L):
    """Whole waves of blocks, unsplit ones and equal parts, one after the other."""
    Hq, Hkv, d, max_ctx, most = 16, 8, 64, 2000, 60
    scratch = torch.zeros(L.loip_k_window_attention_scratch_bytes(most, Hq, Hkv, d, ALL, 0, max_ctx), dtype=torch.uint8,
                          device="cuda")
    ctx = [2000, 1, 700] + [40 + b for b in range(most - 3)]
    c, _ = _decode_cache(ctx, max_ctx, Hkv, d, ALL, 0, 3)
    qd, q64 = _rows(torch, np.random.default_rng(4).standard_normal((most, Hq * d)).astype(np.float32), "f32")
    want = [W.attend(c, r, n - 1, q64[r].reshape(Hq, d), ALL, 0)[:2] for r, n in enumerate(ctx)]
    for B in (60, 58, 57, 48, 46, 45, 29, 28, 19, 8, 3, 1):
        got = _host(_decode(torch, L, c, qd[:B], ctx[:B], Hq, ALL, 0, max_ctx, scratch=scratch))
        for r in range(B):
            assert np.all(np.abs(got[r].reshape(Hq, d) - want[r][0]) <= want[r][1]), (B, r)


def test_chunks_of_a_prompt_keep_their_scratch(torch, L):
    """Many rows (no split), then the last few (split over blocks)."""
    Hq, Hkv, d, ctx = 8, 8, 64, 900
    c, _ = _prefill_cache([(ctx, 0)], ctx, Hkv, d, ALL, 0, 5)
    qd, q64 = _rows(torch, np.random.default_rng(6).standard_normal((700, Hq * d)).astype(np.float32), "f32")
    scratch = torch.zeros(L.loip_k_window_prefill_scratch_bytes(700, 1, Hq, Hkv, d, ALL, 0, ctx), dtype=torch.uint8,
                          device="cuda")
    for M in (700, 300, 33, 1):
        got = _host(_prefill(torch, L, c, qd[:M], [(M, ctx - M)], Hq, ALL, 0, ctx, scratch=scratch))
        for t in {0, M // 2, M - 1}:
            want, t32, _ = W.attend(c, 0, ctx - M + t, q64[t].reshape(Hq, d), ALL, 0)
            assert np.all(np.abs(got[t].reshape(Hq, d) - want) <= t32), (M, t)


def test_a_long_request_is_split_whatever_the_batch(torch, L):
    """One request of 131072 tokens among short ones takes about as long in any batch: the lengths
    are not known to the host, so no batch may leave a request to a few blocks.  (Left whole in a
    batch of 48 it took 15 times as long as in one of 58.)"""
    Hq, Hkv, d, long, short = 32, 8, 64, 131072, 100
    lpb, pages = 2 * Hkv * W.P * d * 2, long // W.P
    gen = torch.Generator(device="cuda").manual_seed(7)
    kv = torch.randn(pages * lpb // 2, device="cuda", generator=gen).bfloat16()
    q = torch.randn(58, Hq * d, device="cuda", generator=gen)
    table = (torch.randperm(pages, device="cuda", generator=gen) * lpb).repeat(58, 1)  # every request, the same pages
    lens = torch.tensor([long] + [short] * 57, dtype=torch.int32, device="cuda")
    scratch = torch.zeros(L.loip_k_window_attention_scratch_bytes(58, Hq, Hkv, d, long, 0, long), dtype=torch.uint8,
                          device="cuda")
    took, out = {}, {}
    for B in (58, 48, 24, 8):
        o = out[B] = torch.empty(B, Hq * d, device="cuda")
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            L.loip_k_window_attention(q[:B], kv, table[:B], pages, lens[:B], Hq, Hkv, d, W.P, 0, lpb, long, 0, long,
                                      scratch, o)
            b.record()
            torch.cuda.synchronize()
            took[B] = min(took.get(B, 1e9), a.elapsed_time(b))
    for B in (48, 24, 8):
        assert took[B] < 4 * took[58], took
        assert torch.allclose(out[B], out[58][:B], rtol=1e-4, atol=1e-5)
