"""Argument checks of the windowed-serving operators, on a machine without a GPU:
every call here is refused, or has no rows, before the library touches CUDA (the
pointers are aligned dummies that nothing may read)."""
import pytest

from paper_2512_21835_gb300 import loip


@pytest.fixture(scope="module")
def L():
    from paper_2512_21835_gb300 import build
    build.build()
    try:
        import torch
        if torch.cuda.is_available():
            pytest.skip("dummy pointers: run only where no CUDA device exists")
    except ImportError:
        pass
    return loip.lib()


A = 1 << 20  # a 16-byte aligned dummy address
CACHE = dict(kv=2 * A, table=3 * A, max_pages=4, page_tokens=64, layer=0, lpb=2 * 2 * 64 * 64 * 2)


def append(L, x=A, dtype=0, stride=512, T=2, Hq=4, Hkv=2, d=64, gq=None, gk=None, eps=1e-6, theta=1e4, pos=4 * A,
           req=None, n_req=2, q=5 * A, **kw):
    c = dict(CACHE, **kw)
    return L.loip_k_qk_append(x, dtype, stride, T, Hq, Hkv, d, gq, gk, eps, theta, pos, req, n_req, q, c["kv"],
                              c["table"], c["max_pages"], c["page_tokens"], c["layer"], c["lpb"], None)


def decode(L, q=A, dtype=0, ctx=4 * A, B=2, Hq=4, Hkv=2, d=64, window=8, sinks=1, max_ctx=256, scratch=6 * A,
           nbytes=None, o=5 * A, **kw):
    c = dict(CACHE, **kw)
    if nbytes is None:
        nbytes = L.loip_k_window_attention_scratch_bytes(B, Hq, Hkv, d, window, sinks, max_ctx)
    return L.loip_k_window_attention(q, dtype, c["kv"], c["table"], c["max_pages"], ctx, B, Hq, Hkv, d,
                                     c["page_tokens"], c["layer"], c["lpb"], window, sinks, max_ctx, scratch, nbytes,
                                     o, None)


def prefill(L, q=A, dtype=0, starts=4 * A, first=None, n=2, M=9, Hq=4, Hkv=2, d=64, window=8, sinks=1, max_ctx=256,
            scratch=6 * A, nbytes=None, o=5 * A, **kw):
    c = dict(CACHE, **kw)
    if nbytes is None:
        nbytes = L.loip_k_window_prefill_scratch_bytes(M, n, Hq, Hkv, d, window, sinks, max_ctx)
    return L.loip_k_window_prefill(q, dtype, c["kv"], c["table"], c["max_pages"], starts, first, n, M, Hq, Hkv, d,
                                   c["page_tokens"], c["layer"], c["lpb"], window, sinks, max_ctx, scratch, nbytes, o,
                                   None)


CACHE_BAD = [dict(dtype=2), dict(dtype=-1), dict(Hq=5), dict(Hkv=0), dict(Hq=0), dict(d=96), dict(d=256), dict(d=0),
             dict(page_tokens=16), dict(page_tokens=0), dict(max_pages=0), dict(layer=-1), dict(kv=None),
             dict(kv=A + 8), dict(table=None), dict(table=A + 4), dict(lpb=24)]
WINDOW_BAD = [dict(q=None), dict(q=A + 8), dict(o=None), dict(o=A + 4), dict(window=-1), dict(sinks=-1),
              dict(max_ctx=0), dict(max_ctx=257), dict(max_ctx=(1 << 30) + 1, max_pages=1 << 25), dict(scratch=None), dict(scratch=A + 8), dict(nbytes=0)]


@pytest.mark.parametrize("bad", CACHE_BAD + [
    dict(T=-1), dict(x=None), dict(x=A + 4), dict(q=None), dict(q=A + 8), dict(stride=511), dict(stride=508),
    dict(stride=514), dict(dtype=1, stride=516), dict(pos=None), dict(pos=A + 2), dict(req=A + 1), dict(n_req=0),
    dict(gq=A), dict(gk=A), dict(gq=A + 2, gk=A), dict(theta=0.5), dict(theta=-1.0), dict(theta=float("nan")),
    dict(theta=float("inf")), dict(eps=-1.0), dict(eps=float("nan"))])
def test_append_refuses(L, bad):
    assert append(L, **bad) == loip.ERR_INVALID
    assert L.loip_last_error(None)


@pytest.mark.parametrize("bad", CACHE_BAD + WINDOW_BAD + [dict(B=-1), dict(ctx=None), dict(ctx=A + 2)])
def test_decode_refuses(L, bad):
    assert decode(L, **bad) == loip.ERR_INVALID
    assert L.loip_last_error(None)


@pytest.mark.parametrize("bad", CACHE_BAD + WINDOW_BAD + [
    dict(M=-1), dict(n=0), dict(n=-1), dict(starts=None), dict(starts=A + 2), dict(first=A + 1)])
def test_prefill_refuses(L, bad):
    assert prefill(L, **bad) == loip.ERR_INVALID
    assert L.loip_last_error(None)


def test_no_rows_launch_nothing(L):
    assert append(L, T=0) == loip.OK
    assert decode(L, B=0) == loip.OK
    assert prefill(L, M=0) == loip.OK
    assert prefill(L, M=0, n=0) == loip.OK


def test_scratch_sizes(L):
    """Sizes grow with the batch and the visible length, and stay the same once the window covers max_ctx."""
    f, g = L.loip_k_window_attention_scratch_bytes, L.loip_k_window_prefill_scratch_bytes
    for a in ((0, 4, 2, 64, 8, 1, 256), (2, 4, 2, 64, 8, 1, 256)):
        assert f(*a) >= 16 and g(a[0], 1, *a[1:]) >= 16
    assert f(1, 32, 8, 128, 1 << 17, 0, 1 << 17) == f(1, 32, 8, 128, 2147483647, 2147483647, 1 << 17)
    for bad in ((-1, 4, 2, 64, 8, 1, 256), (2, 5, 2, 64, 8, 1, 256), (2, 4, 2, 80, 8, 1, 256), (2, 4, 2, 64, -1, 1, 256),
                (2, 4, 2, 64, 8, 1, 0)):
        assert f(*bad) == 0 and g(bad[0], 1, *bad[1:]) == 0
