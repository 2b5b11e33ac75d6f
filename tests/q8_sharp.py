"""The sharp inputs of window_sharp.py over the 8-bit cache, with keys and values of any size: every bf16 plane
of the operands counts, and no two numbers of a block differ in size.

A key has one element that a query meets, a value is the same in all columns.  What the cache holds is exact.  With
`dense` no block is zero: keys have their size wherever queries are zero, and a value of zero has a block's
last column in the size of the other one (which `columns` leaves out)."""
import numpy as np

import window_ref as W
import window_sharp as S
from q8_ref import Cache8

KINDS = S.KINDS


def key_of(kind):
    return 16.0 if kind == "queries" else 1.0


def value_of(kind):
    return 1.0 if kind == "queries" else 256.0


def exponent(size):
    """E of a block whose largest element is this power of two (its magnitude is 64 = 2^6)."""
    return 133 - 6 + int(np.log2(size))


def case(kind, requests, rows, Hq, Hkv, d, seed, Ek, Ev, dense=False):
    """(cache of `requests` requests of one page, q fp32 [rows][Hq][d] as given to the operator, q as window_sharp.py's
    functions know it); keys and values in blocks of exponents Ek and Ev."""
    ks, vs = 2.0 ** (Ek - exponent(key_of(kind))), 2.0 ** (Ev - exponent(value_of(kind)))
    _, q = S.case(kind, 1 if rows is None else rows, Hq, Hkv, d, seed)
    c = Cache8(requests, 2, Hkv, d, seed, fill=0)
    last = np.arange(d) % 32 == 31
    for r in range(requests):
        k, v = np.zeros((2, Hkv, d)), np.zeros((2, Hkv, d))
        for j in range(2):
            k[j, :, j] = key_of(kind) * ks
            if dense:
                k[j, :, 2:] = key_of(kind) * ks
            v[j] = {"queries": (1.0, -1.0), "weights": (0.0, 256.0), "opposed": (256.0, -256.0)}[kind][j] * vs
            if dense and kind == "weights":
                v[j][:, last] = 256.0 * vs
        c.put(r, np.arange(2), k, v)
        got_k, got_v = c.gather(r, np.arange(2))
        assert np.array_equal(got_k, k) and np.array_equal(got_v, v)
        if dense:
            for which, E in ((0, Ek), (1, Ev)):
                assert np.all(c.bytes[c.slot(r, np.arange(2), which)[1]] == E)
    given = (q.astype(np.float64) / ks).astype(np.float32)
    assert np.array_equal(given.astype(np.float64) * ks, q)
    return c, given, q


def columns(kind, d, dense):
    return np.flatnonzero(np.arange(d) % 32 != 31) if dense and kind == "weights" else np.arange(d)


def exact(kind, q, Ev):
    return S.exact(kind, q) * 2.0 ** (Ev - exponent(value_of(kind)))


def bound(kind, q, dtype, Ev):
    return S.bound(kind, q, dtype) * 2.0 ** (Ev - exponent(value_of(kind)))


def definition_agrees(kind, c, given, q, Ev, rows):
    """The exact answers are the plain implementation's."""
    for r in rows:
        want, _, _ = W.attend(c, min(r, c.R - 1), 1, given[r].astype(np.float64), 2, 0)
        cols = columns(kind, c.d, True)
        assert np.allclose(want[:, cols], exact(kind, q, Ev)[r][:, None], rtol=1e-11, atol=0)
