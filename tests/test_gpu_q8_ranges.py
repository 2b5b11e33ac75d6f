"""Exponents at the ends of the tensor cores' one-product forms, with nothing visible outside them, so that no
row is computed in another way: prompts 71 to 191 and blocks of zeros, single tokens 96 to 159.  And exponents
outside, through the loaders that turn codes into tiles."""
import numpy as np
import pytest

import window_ref as W
from gpu_util import need_gpu
from q8_ref import Cache8
from test_gpu_q8 import ALL, P, _check_prefill, _decode, _host, _prefill, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.fixture(scope="module")
def L(torch):
    from paper_2512_21835_gb300 import loip
    return loip


def filled(requests, n, Hkv, d, seed, lo, hi, zeros):
    """A cache of n positions a request, codes at random, and the size of each kv head's keys.  Kv head h has keys of
    exponent hi, lo, 127 or lo .. lo + 2 and values of lo, hi, lo .. lo + 4 or hi - 4 .. hi (by h % 4)."""
    rng = np.random.default_rng(seed)
    c = Cache8(requests, -(-n // P), Hkv, d, seed)
    kinds = [((hi, hi), (lo, lo)), ((lo, lo), (hi, hi)), ((127, 127), (lo, lo + 4)), ((lo, lo + 2), (hi - 4, hi))]
    sizes = np.array([2.0 ** (kinds[h % 4][0][0] - 127) for h in range(Hkv)])
    for r in range(requests):
        for which in (0, 1):
            codes, exps = c.slot(r, np.arange(n), which)
            m = rng.integers(0, 128, (n, Hkv, d // 32, 32))
            m[..., 0] = rng.integers(64, 128, m.shape[:-1])  # E is the smallest
            E = np.stack([rng.integers(kinds[h % 4][which][0], kinds[h % 4][which][1] + 1, (n, d // 32))
                          for h in range(Hkv)], 1)
            if zeros:
                none = rng.random(E.shape) < 0.05
                m[none], E[none] = 0, 8
            m = m + 128 * ((rng.random(m.shape) < 0.5) & (m > 0))
            c.bytes[codes], c.bytes[exps] = m.reshape(n, Hkv, d), E
    return c, sizes


def queries(rows, Hq, d, sizes, seed):
    """Scores of a few units: queries as large as the head's keys are small."""
    q = np.random.default_rng(seed).standard_normal((rows, len(sizes), Hq // len(sizes), d))
    return (2 * q / sizes[None, :, None, None]).reshape(rows, Hq * d).astype(np.float32)


def check(got, c, q64, where, Hq, window, sinks, dtype):
    for row, r, pos in where:
        want, t32, tbf = W.attend(c, r, pos, q64[row].reshape(Hq, c.d), window, sinks)
        err, tol = np.abs(got[row].reshape(Hq, c.d) - want), t32 if dtype == "f32" else tbf
        assert np.all(err <= tol), (row, float((err / tol).max()))


# one row tile a block and two, pages through the loaders and through images
SHAPES = {"loaders": (16, 4, [(12, 130)]), "loaders, two tiles": (16, 16, [(300, 0), (129, 70)] + [(30 + i, 40) for i in range(20)]),
          "images": (64, 4, [(150, 30)]), "images, two tiles": (64, 4, [(640, 20)])}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (100, 3)])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_prefill_inside(torch, L, shape, window, sinks, d, dtype):
    Hq, Hkv, runs = SHAPES[shape]
    n = max(rows + first for rows, first in runs)
    c, sizes = filled(len(runs), n, Hkv, d, 301, 71, 191, zeros=True)
    M = sum(rows for rows, _ in runs)
    qd, q64 = _rows(torch, queries(M, Hq, d, sizes, 302), dtype)
    got = _host(_prefill(torch, L, c, qd, runs, Hq, window, sinks, c.max_pages * P))
    starts = np.cumsum([0] + [rows for rows, _ in runs])
    where = [(starts[r] + t, r, first + t) for r, (rows, first) in enumerate(runs) for t in range(0, rows, 17)]
    check(got, c, q64, where, Hq, window, sinks, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (300, 70)])
def test_decode_inside(torch, L, window, sinks, d, dtype):
    ctx, Hq, Hkv = (700, 1, 63, 355), 12, 4
    c, sizes = filled(len(ctx), max(ctx), Hkv, d, 311, 96, 159, zeros=False)
    qd, q64 = _rows(torch, queries(len(ctx), Hq, d, sizes, 312), dtype)
    got = _host(_decode(torch, L, c, qd, ctx, Hq, window, sinks, c.max_pages * P))
    check(got, c, q64, [(r, r, n - 1) for r, n in enumerate(ctx)], Hq, window, sinks, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [254, 255, 40, 200])
@pytest.mark.parametrize("Hq,Hkv,d,runs", [(6, 2, 128, [(70, 70), (33, 110)]),
                                           (16, 16, 64, [(280, 0), (130, 5)] + [(20, 120)] * 18)])
def test_loaders_and_extreme_exponents(torch, L, Hq, Hkv, d, runs, E, dtype):
    """NaN that some rows see, blocks whose exponents the loaders have no form for, and zeros with such exponents."""
    def edit(c):
        for r in range(2):
            for which, j in ((1, 133), (0, 101)):
                c.bytes[c.slot(r, j, which)[1][:, 1]] = E if which else min(E, 120)
        codes, exps = c.slot(2 % c.R, 115, 1)
        c.bytes[codes], c.bytes[exps] = 0, min(E, 253)

    got = _check_prefill(torch, L, runs, Hq, Hkv, d, 100, 1, dtype, 321, edit=edit)
    nan = np.zeros(got.shape, dtype=bool)
    row = 0
    for r, (rows, first) in enumerate(runs):
        for t in range(rows):
            nan[row, :, 32:64] = E >= 254 and r < 2 and first + t >= 133 and first + t < 233
            row += 1
    assert np.array_equal(np.isnan(got), nan)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d,runs", [(16, 4, 64, [(12, 130)]), (64, 4, 128, [(150, 30)]), (64, 4, 64, [(640, 20)]),
                                           (16, 16, 64, [(300, 0)] + [(30, 40)] * 20)])
def test_equal_prompts_give_equal_bits(torch, L, Hq, Hkv, d, runs, dtype):
    n = max(rows + first for rows, first in runs)
    c, sizes = filled(len(runs), n, Hkv, d, 331, 120, 130, zeros=True)
    M = sum(rows for rows, _ in runs)
    qd, _ = _rows(torch, queries(M, Hq, d, sizes, 332), dtype)
    first = _prefill(torch, L, c, qd, runs, Hq, ALL, 0, c.max_pages * P)
    assert bool(torch.isfinite(first).all())
    for _ in range(4):
        assert torch.equal(_prefill(torch, L, c, qd, runs, Hq, ALL, 0, c.max_pages * P), first)


# values of NaN that every row sees: the other columns are computed as without them, bit for bit
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d,runs,window,j", [
    (16, 4, 64, [(12, 130)], ALL, 40), (64, 4, 128, [(150, 130)], ALL, 40), (64, 4, 64, [(640, 130)], ALL, 127),
    (64, 4, 64, [(150, 130)], 500, 0), (64, 4, 128, [(150, 130)], 0, 1)])
def test_a_value_of_nan_that_all_rows_see(torch, L, Hq, Hkv, d, runs, window, j, dtype):
    sinks = 0 if window else 64
    n = max(rows + first for rows, first in runs)
    c, sizes = filled(1, n, Hkv, d, 341, 120, 130, zeros=True)
    M = sum(rows for rows, _ in runs)
    qd, _ = _rows(torch, queries(M, Hq, d, sizes, 342), dtype)
    plain = _host(_prefill(torch, L, c, qd, runs, Hq, window, sinks, c.max_pages * P)).reshape(M, Hkv, -1, d)
    c.bytes[c.slot(0, j, 1)[1][1, 1]] = 255
    got = _host(_prefill(torch, L, c, qd, runs, Hq, window, sinks, c.max_pages * P)).reshape(M, Hkv, -1, d)
    assert np.all(np.isnan(got[:, 1, :, 32:64])) and np.all(np.isfinite(plain))
    got[:, 1, :, 32:64] = plain[:, 1, :, 32:64]
    assert np.array_equal(got, plain)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rows", [(128, 150), (64, 640)])
def test_a_value_of_nan_that_the_first_rows_do_not_see(torch, L, d, rows, dtype):
    """Rows before it are finite; the row tiles behind its page are computed as without it, bit for bit."""
    Hq, Hkv, first, j = 64, 4, 30, 40
    c, sizes = filled(1, rows + first, Hkv, d, 351, 120, 130, zeros=True)
    qd, q64 = _rows(torch, queries(rows, Hq, d, sizes, 352), dtype)
    plain = _host(_prefill(torch, L, c, qd, [(rows, first)], Hq, ALL, 0, c.max_pages * P)).reshape(rows, Hkv, -1, d)
    c.bytes[c.slot(0, j, 1)[1][1, 1]] = 255
    got = _host(_prefill(torch, L, c, qd, [(rows, first)], Hq, ALL, 0, c.max_pages * P)).reshape(rows, Hkv, -1, d)
    nan = np.zeros(got.shape, dtype=bool)
    nan[j - first:, 1, :, 32:64] = True
    assert np.array_equal(np.isnan(got), nan)
    for t in range(j - first):
        want, t32, tbf = W.attend(c, 0, first + t, q64[t].reshape(Hq, d), ALL, 0)
        assert np.all(np.abs(got[t].reshape(Hq, d) - want) <= (t32 if dtype == "f32" else tbf)), t
    behind = P - 1 - first + 16  # two row tiles of eight positions further on
    got[nan] = plain[nan]
    assert np.array_equal(got[behind:], plain[behind:])
    others = [0, 2, 3]
    assert np.array_equal(got[:, others], plain[:, others])
