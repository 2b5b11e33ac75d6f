"""Batches that change from call to call, with one scratch that is sized for the largest."""
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
