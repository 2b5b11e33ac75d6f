"""Both attentions over the 8-bit cache on inputs where every bf16 plane of their operands counts, at ordinary
sizes and at both ends of the exponents that one product serves."""
import numpy as np
import pytest

import q8_sharp as S8
from gpu_util import need_gpu
from test_gpu_q8 import _decode, _host, _prefill, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.fixture(scope="module")
def L(torch):
    from paper_2512_21835_gb300 import loip
    return loip


def _check(kind, dtype, got, q, Ev, d, dense):
    got = got.reshape(*q.shape)[..., S8.columns(kind, d, dense)]
    err = np.abs(got - S8.exact(kind, q, Ev)[..., None])
    tol = S8.bound(kind, q, dtype, Ev)[..., None]
    assert np.all(err <= tol), float((err / tol).max())


# dense: exponents of 96 to 159, the tile's one-product form; else blocks of zeros, the exact form
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Ek,Ev,dense", [(127, 127, True), (96, 96, True), (159, 159, True), (96, 159, True),
                                         (127, 127, False), (40, 20, False), (200, 230, False)])
@pytest.mark.parametrize("kind,dtype", [("queries", "f32"), ("weights", "f32"), ("opposed", "f32"), ("opposed", "bf16")])
def test_decode(torch, L, kind, dtype, Ek, Ev, dense, d):
    R, Hq = 6, 16
    c, given, q = S8.case(kind, R, R, Hq, 2, d, 7, Ek, Ev, dense)
    qd, _ = _rows(torch, given.reshape(R, Hq * d), dtype)
    _check(kind, dtype, _host(_decode(torch, L, c, qd, [2] * R, Hq, 2, 0, 64)), q, Ev, d, dense)


# a few rows: pages turned into tiles by the row tiles' own loaders
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Ek,Ev", [(127, 127), (71, 71), (191, 191), (191, 71), (40, 127), (127, 230)])
@pytest.mark.parametrize("kind", S8.KINDS)
def test_prefill(torch, L, kind, Ek, Ev, d):
    R, Hq = 6, 16
    c, given, q = S8.case(kind, R, R, Hq, 2, d, 8, Ek, Ev)
    qd, _ = _rows(torch, given.reshape(R, Hq * d), "f32")
    _check(kind, "f32", _host(_prefill(torch, L, c, qd, [(1, 1)] * R, Hq, 2, 0, 64)), q, Ev, d, False)


# many rows that all see the first two positions: images of the pages
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Ek,Ev", [(127, 127), (71, 71), (191, 191), (191, 71), (40, 127), (127, 230)])
@pytest.mark.parametrize("kind", S8.KINDS)
def test_prefill_images(torch, L, kind, Ek, Ev, d):
    M, Hq = 64, 16
    c, given, q = S8.case(kind, 1, M, Hq, 2, d, 9, Ek, Ev)
    qd, _ = _rows(torch, given.reshape(M, Hq * d), "f32")
    _check(kind, "f32", _host(_prefill(torch, L, c, qd, [(M, 1)], Hq, 0, 2, 128)), q, Ev, d, False)
