"""Both attentions on inputs where every bf16 plane of their operands counts."""
import numpy as np
import pytest

import window_sharp as S
from gpu_util import need_gpu
from test_gpu_window import _decode, _host, _prefill, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.fixture(scope="module")
def L(torch):
    from paper_2512_21835_gb300 import loip
    return loip


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,dtype", [("queries", "f32"), ("weights", "f32"), ("opposed", "f32"), ("opposed", "bf16")])
def test_decode(torch, L, kind, dtype, d):
    R, Hq = 6, 16
    c, q = S.case(kind, R, Hq, 2, d, 7)
    qd, _ = _rows(torch, q.reshape(R, Hq * d), dtype)
    got = _host(_decode(torch, L, c, qd, [2] * R, Hq, 2, 0, 64)).reshape(R, Hq, d)
    assert np.all(np.abs(got - S.exact(kind, q)[..., None]) <= S.bound(kind, q, dtype)[..., None])


# bf16 rows of prompts have one plane of weights by choice
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", S.KINDS)
def test_prefill(torch, L, kind, d):
    R, Hq = 6, 16
    c, q = S.case(kind, R, Hq, 2, d, 8)
    qd, _ = _rows(torch, q.reshape(R, Hq * d), "f32")
    got = _host(_prefill(torch, L, c, qd, [(1, 1)] * R, Hq, 2, 0, 64)).reshape(R, Hq, d)
    assert np.all(np.abs(got - S.exact(kind, q)[..., None]) <= S.bound(kind, q, "f32")[..., None])
