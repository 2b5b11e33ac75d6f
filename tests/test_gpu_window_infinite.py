"""Infinities that a row does see: the attention operators behind a window answer as the
definition does.  An infinite cached value makes its column infinite (NaN where both signs
meet), an infinite key a score of +inf (the row becomes NaN) or of -inf (a weight of zero)."""
import numpy as np
import pytest

import window_ref as W
from gpu_util import need_gpu
from test_gpu_window import _check_prefill, _decode, _host, _prefill, _prefill_cache, _rows
from window_ref import P, Cache

pytestmark = pytest.mark.gpu

INF, NEG = 0x7F80, 0xFF80
ALL = 1 << 30


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.fixture(scope="module")
def L(torch):
    from paper_2512_21835_gb300 import loip
    return loip


def _spoil(c, r, j, which, column, bits):
    b = c.bits[c.slot(r, j, which)].copy()
    b[:, column] = bits
    c.bits[c.slot(r, j, which)] = b


def _agree(got, want, tol, where):
    assert np.array_equal(np.isnan(got), np.isnan(want)), where
    assert np.array_equal(np.isposinf(got), np.isposinf(want)), where
    assert np.array_equal(np.isneginf(got), np.isneginf(want)), where
    fine = np.isfinite(want)
    assert np.all(np.abs(got[fine] - want[fine]) <= tol[fine]), where


def _values(c, ctx):
    """Column 5 holds +inf, column 9 -inf, column 11 both; position 0 is all there is of the shortest."""
    for r, n in enumerate(ctx):
        _spoil(c, r, 0, 1, 5, INF)
        for j, col, bits in ((3, 9, NEG), (7, 11, INF), (n - 2, 11, NEG)):
            if 0 <= j < n:
                _spoil(c, r, j, 1, col, bits)


# split over blocks, within one block, one position
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_infinite_values(torch, L, d, dtype):
    ctx, Hq, Hkv = (900, 40, 1), 8, 2
    c = Cache(len(ctx), -(-max(ctx) // P), Hkv, d, 5)
    for r, n in enumerate(ctx):
        c.fill_request(r, range(n), 10 + r, scale=0.5)
    _values(c, ctx)
    q = np.random.default_rng(1).standard_normal((len(ctx), Hq * d)).astype(np.float32)
    qd, q64 = _rows(torch, q, dtype)
    got = _host(_decode(torch, L, c, qd, ctx, Hq, ALL, 0, max(ctx)))
    for r, n in enumerate(ctx):
        with np.errstate(invalid="ignore"):
            want, t32, tbf = W.attend(c, r, n - 1, q64[r].reshape(Hq, d), ALL, 0)
        assert np.all(np.isposinf(want[:, 5]))
        _agree(got[r].reshape(Hq, d), want, t32 if dtype == "f32" else tbf, (r, n))


# rows whose tile sees a page in full, rows that see a part of it, a prompt split over blocks
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_infinite_values(torch, L, d, dtype):
    with np.errstate(invalid="ignore"):
        got = _check_prefill(torch, L, [(150, 0), (1, 0), (9, 500)], 4, 2, d, ALL, 0, dtype, 301,
                             edit=lambda c: _values(c, (150, 1, 509)))
    assert np.all(np.isposinf(got[:150, :, 5])) and np.all(np.isneginf(got[3:150, :, 9]))
    assert np.all(np.isposinf(got[150, :, 5])) and np.all(np.isneginf(got[151:, :, 9]))
    assert np.all(np.isposinf(got[7:148, :, 11])) and np.all(np.isnan(got[148:150, :, 11]))


class Without(Cache):
    """A cache that is read as if the positions `gone` were not seen: their weight is zero."""
    gone = ()

    def gather(self, r, js):
        return super().gather(r, [j for j in js if j not in self.gone])


def _signs(rng, rows, Hq, d):
    """Queries whose first element is of either sign, with and without further bf16 planes."""
    q = rng.standard_normal((rows, Hq, d))
    q[..., 0] = np.where(np.arange(Hq) % 2 == 0, 1, -1) * np.where(np.arange(Hq) % 3 == 0, 1.0, np.abs(q[..., 0]) + 0.1)
    return q.reshape(rows, Hq * d).astype(np.float32)


def _check_keys(got, c, rows, Hq, d, dtype, q64, at):
    """rows: (request, position).  Heads with a positive first element have a score of +inf at `at`."""
    c.__class__, c.gone = Without, (at,)
    for i, (r, pos) in enumerate(rows):
        want, t32, tbf = W.attend(c, r, pos, q64[i].reshape(Hq, d), ALL, 0)
        if pos >= at:
            want = np.where(q64[i].reshape(Hq, d)[:, :1] > 0, np.nan, want)
        _agree(got[i].reshape(Hq, d), want, t32 if dtype == "f32" else tbf, (r, pos))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_infinite_keys(torch, L, d, dtype):
    ctx, Hq, Hkv = (900, 40, 8), 8, 2
    c = Cache(len(ctx), -(-max(ctx) // P), Hkv, d, 6)
    for r, n in enumerate(ctx):
        c.fill_request(r, range(n), 20 + r)
        _spoil(c, r, 7, 0, 0, INF)
    qd, q64 = _rows(torch, _signs(np.random.default_rng(2), len(ctx), Hq, d), dtype)
    got = _host(_decode(torch, L, c, qd, ctx, Hq, ALL, 0, max(ctx)))
    _check_keys(got, c, [(r, n - 1) for r, n in enumerate(ctx)], Hq, d, dtype, q64, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_infinite_keys(torch, L, d, dtype):
    runs, Hq, Hkv = [(150, 0), (9, 500)], 4, 2
    c, _ = _prefill_cache(runs, 509, Hkv, d, ALL, 0, 401)
    for r in range(2):
        _spoil(c, r, 7, 0, 0, INF)
    qd, q64 = _rows(torch, _signs(np.random.default_rng(3), 159, Hq, d), dtype)
    got = _host(_prefill(torch, L, c, qd, runs, Hq, ALL, 0, 509))
    _check_keys(got, c, [(r, f + t) for r, (n, f) in enumerate(runs) for t in range(n)], Hq, d, dtype, q64, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefill_infinite_first_key_of_a_row_walked_alone(torch, L, dtype):
    """The first position seen has a score of -inf, in a tile whose rows are computed one by one
    (a value that is not finite, in a page that some of its rows see in part)."""
    runs, Hq, Hkv, d = [(40, 0)], 4, 2, 64
    c, _ = _prefill_cache(runs, 40, Hkv, d, ALL, 0, 501)
    _spoil(c, 0, 0, 0, 0, INF)
    _spoil(c, 0, 30, 1, 5, INF)
    qd, q64 = _rows(torch, _signs(np.random.default_rng(4), 40, Hq, d), dtype)
    got = _host(_prefill(torch, L, c, qd, runs, Hq, ALL, 0, 40))
    _check_keys(got[1:], c, [(0, t) for t in range(1, 40)], Hq, d, dtype, q64[1:], 0)


@pytest.mark.parametrize("walked", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_but_scores_of_minus_infinity(torch, L, dtype, walked):
    """Every position that the row sees has weight zero: the row is zero, as one that sees nothing."""
    Hq, Hkv, d = 4, 2, 64
    c = Cache(1, 1, Hkv, d, 7)
    c.fill_request(0, range(20), 8)
    for j in range(3):
        _spoil(c, 0, j, 0, 0, INF)
    if walked:
        _spoil(c, 0, 10, 1, 5, INF)
    q = -np.abs(np.random.default_rng(5).standard_normal((20, Hq, d))) - 0.1
    q[:, :, 1:] *= 0.1
    qd, _ = _rows(torch, q.reshape(20, Hq * d).astype(np.float32), dtype)
    o = _host(_prefill(torch, L, c, qd, [(20, 0)], Hq, ALL, 0, 20))
    assert np.all(o[:3] == 0) and np.all(np.isfinite(o[3:10])) and np.any(o[3:10] != 0)
    assert np.all(_host(_decode(torch, L, c, qd[:1], [3], Hq, ALL, 0, 20)) == 0)
