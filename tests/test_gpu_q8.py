"""The operators of the 8-bit cache on the GPU against a plain 64-bit implementation: append
and reading back, attention of single tokens and of prompts.  What is not written is NaN, and
page-table entries of pages that no row may read point at a page of NaN."""
import numpy as np
import pytest

import q8_ref as Q
import window_ref as W
from gpu_util import dev_bits, dev_f32, need_gpu
from q8_ref import Cache8
from window_ref import P

pytestmark = pytest.mark.gpu

ALL = 1 << 30


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.fixture(scope="module")
def L(torch):
    from paper_2512_21835_gb300 import loip
    return loip


def _rows(torch, a, dtype):
    """fp32 array -> (device tensor of the type, its values in fp64)."""
    if dtype == "f32":
        return dev_f32(a), np.asarray(a, dtype=np.float32).astype(np.float64)
    return dev_bits(W.bf16_bits(a)).view(torch.bfloat16), W.bf16_round(a).astype(np.float64)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _ints(torch, v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def _dev(torch, a):
    return torch.from_numpy(a).cuda()


# ---------------------------------------------------------------------------
# append and reading back
# ---------------------------------------------------------------------------
def _append(torch, L, c, xd, g, Hq, eps, theta, pos, req, q=None):
    """The call on a copy of the cache; returns (q_out, the cache's bytes after it)."""
    kv = _dev(torch, c.bytes)
    if q is None:
        q = torch.full((xd.shape[0], Hq * c.d), float("nan"), dtype=xd.dtype, device="cuda")
    L.loip_k_qk_append_q8(xd, *g, Hq, c.Hkv, c.d, eps, theta, _ints(torch, pos),
                          None if req is None else _ints(torch, req), q, kv, _dev(torch, c.table), c.max_pages, P,
                          c.layer, c.layer_page_bytes)
    return q, kv


# ragged requests out of order, padding rows, rows wider than their heads, a cache of
# several layers; head sizes 64 and 128 with 1 to 8 query heads per kv head
@pytest.mark.parametrize("T", [1, 7, 130])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (7, 7, 64), (12, 4, 128), (64, 8, 128)])
@pytest.mark.parametrize("dtype,norm", [("f32", True), ("f32", False), ("bf16", True), ("bf16", False)])
def test_append_parity(torch, L, T, Hq, Hkv, d, dtype, norm):
    rng = np.random.default_rng(T * 100 + Hq)
    R, pages, theta, eps = 3, 4, 500000.0, 1e-6
    c = Cache8(R, pages, Hkv, d, 5, layers=3, layer=1, gap=256)
    slots = rng.permutation(R * pages * P)[:T]
    req, pos = (slots // (pages * P)).astype(np.int32), (slots % (pages * P)).astype(np.int32)
    if T > 1:  # padding: no position, a position past the table, no such request
        pos[1], pos[-1] = -1, pages * P
        req[T // 2] = (R, -1)[T % 2]
    width = (Hq + 2 * Hkv) * d
    x = (rng.standard_normal((T, width + 16)) * 1.5).astype(np.float32)
    xd, x64 = _rows(torch, x, dtype)
    g = [W.bf16_bits(1 + 0.1 * rng.standard_normal(d)) for _ in range(2)] if norm else [None, None]
    g64 = [None if v is None else W.bits_f64(v) for v in g]
    q, kv = _append(torch, L, c, xd[:, :width], [None if v is None else dev_bits(v) for v in g], Hq, eps, theta, pos, req)
    got_q, got = _host(q).reshape(T, Hq, d), kv.cpu().numpy()
    out = torch.full((T, 2 * Hkv * d), float("nan"), dtype=xd.dtype, device="cuda")
    L.loip_k_cache_read_q8(kv, _dev(torch, c.table), pages, _ints(torch, pos), _ints(torch, req), Hkv, d, P, c.layer,
                           c.layer_page_bytes, out)
    out = _host(out).reshape(T, 2, Hkv, d)
    want = c.bytes.copy()
    for t in range(T):
        if not (0 <= pos[t] < pages * P and 0 <= req[t] < R):
            assert np.all(got_q[t] == 0) and np.all(out[t] == 0)
            continue
        wq, wk, wv, tq, tk = W.append_row(x64[t, :width], int(pos[t]), Hq, Hkv, d, *g64, eps, theta)
        half = 0 if dtype == "f32" else 2.0 ** -8
        assert np.all(np.abs(got_q[t] - wq) <= tq + half * (np.abs(wq) + tq)), t
        (kc, ke), (vc, ve) = c.slot(req[t], pos[t], 0), c.slot(req[t], pos[t], 1)
        # the key before its rounding is off by tk, and with it the block's largest magnitude
        most = (np.abs(wk) + tk).reshape(Hkv, d // 32, 32).max(-1)
        assert np.all(np.abs(Q.decode(got[kc], got[ke]) - wk) <= tk + np.repeat(Q.half_step(most), 32, -1)), t
        assert np.all((got[kc] & 127).reshape(Hkv, -1, 32).max(-1) >= 64)  # the smallest exponent
        codes, exps = Q.encode(wv)
        assert np.array_equal(got[vc], codes) and np.array_equal(got[ve], exps), t
        assert np.array_equal(out[t], np.stack([Q.decode(got[kc], got[ke]), Q.decode(got[vc], got[ve])])), t
        for ix in (kc, ke, vc, ve):
            want[ix] = got[ix]
    assert np.array_equal(got, want)  # nothing else was written


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hkv,d", [(3, 64), (2, 128)])
def test_append_blocks_at_the_borders(torch, L, Hkv, d, dtype):
    """No norm, no rotation: the bytes are the format's.  Rounding borders, zeros, the smallest and
    largest exponents, blocks that are not finite beside ones that are."""
    rng = np.random.default_rng(9)
    kinds = [lambda b: b * 0, lambda b: b * 2.0 ** -125, lambda b: b * 2.0 ** -130, lambda b: b * 2.0 ** -145,
             lambda b: b * 2.0 ** 118, lambda b: np.where(b == b.max(), 127.5 * 2.0 ** 120, b),
             lambda b: np.where(b == b.max(), 127.0 * 2.0 ** 120, b), lambda b: np.where(b == b.max(), np.inf, b),
             lambda b: np.where(b == b.max(), -np.inf, b), lambda b: np.where(b == b.max(), np.nan, b),
             lambda b: np.rint(b * 50) + 0.5, lambda b: np.where(b == b.max(), 127.5, np.rint(b * 30) / 2),
             lambda b: np.where(b == b.max(), 127.0, np.rint(b * 30) / 2), lambda b: np.where(b == b.max(), 255 * 2.0 ** 7, b),
             lambda b: b]
    T = 90
    x = rng.standard_normal((T, 3 * Hkv * d)).astype(np.float64)
    b = x.reshape(T, -1, 32)
    for i in range(b.shape[0]):
        for j in range(b.shape[1]):
            b[i, j] = kinds[rng.integers(len(kinds))](b[i, j])
    with np.errstate(over="ignore"):
        x32 = x.astype(np.float32)
    if dtype == "f32":
        xd, x64 = dev_f32(x32), x32.astype(np.float64)
    else:
        xd = _dev(torch, x32).to(torch.bfloat16)
        x64 = _host(xd)
    c = Cache8(1, 2, Hkv, d, 6)
    _, kv = _append(torch, L, c, xd, (None, None), Hkv, 0.0, 0.0, range(T), [0] * T)
    got = kv.cpu().numpy()
    out = torch.empty(T, 2 * Hkv * d, dtype=xd.dtype, device="cuda")
    L.loip_k_cache_read_q8(kv, _dev(torch, c.table), 2, _ints(torch, range(T)), _ints(torch, [0] * T), Hkv, d, P, 0,
                           c.layer_page_bytes, out)
    out = _host(out).reshape(T, 2, Hkv, d)
    for t in range(T):
        for which in (0, 1):
            codes, exps = Q.encode(x64[t].reshape(3, Hkv, d)[1 + which])
            ic, ie = c.slot(0, t, which)
            assert np.array_equal(got[ie], exps), t
            assert np.array_equal(got[ic], codes), t
            assert np.array_equal(out[t, which], Q.decode(codes, exps), equal_nan=True), t


def test_append_identity_rows_and_no_rows(torch, L):
    """row_req None: row t is request t; zero rows launch nothing; rows are read back in any order, one of them twice."""
    Hq, Hkv, d, R = 4, 4, 64, 5
    c = Cache8(R, 1, Hkv, d, 1)
    x = np.random.default_rng(4).standard_normal((R, 3 * Hq * d)).astype(np.float32)
    args = ((None, None), Hq, 0.0, 0.0)
    q, kv = _append(torch, L, c, dev_f32(x)[:0], *args, [], None)
    assert np.array_equal(kv.cpu().numpy(), c.bytes)
    q, kv = _append(torch, L, c, dev_f32(x), *args, range(R), None)
    assert np.array_equal(q.cpu().numpy(), x[:, :Hq * d])
    want = Q.decode(*Q.encode(x[:, Hq * d:]))
    tab = _dev(torch, c.table)

    def read(pos, req):
        out = torch.full((len(pos), 2 * Hkv * d), 7.0, device="cuda")
        L.loip_k_cache_read_q8(kv, tab, 1, _ints(torch, pos), None if req is None else _ints(torch, req), Hkv, d, P, 0,
                               c.layer_page_bytes, out)
        return _host(out)

    assert read([], []).shape == (0, 2 * Hkv * d)
    assert np.array_equal(read(range(R), None), want)
    order = [3, 0, 3, 4, 1]
    assert np.array_equal(read(order, order), want[order])
    assert np.all(np.isnan(read([1], [0])))  # not written


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hkv,d,T", [(40, 64, 5003), (40, 128, 2501)])
def test_read_of_many_rows(torch, L, Hkv, d, T, dtype):
    """Enough rows that a thread takes four: any order, padding among them, the last group not full."""
    c = Cache8(1, 10, Hkv, d, 13, layers=2, layer=1)
    c.fill_request(0, range(600), 14)  # the last 40 positions are not written
    pos = np.random.default_rng(15).integers(0, 640, T).astype(np.int32)
    pos[[3, T - 2]] = -1, 640
    out = torch.full((T, 2 * Hkv * d), 7.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    L.loip_k_cache_read_q8(_dev(torch, c.bytes), _dev(torch, c.table), 10, _ints(torch, pos), _ints(torch, [0] * T), Hkv,
                           d, P, c.layer, c.layer_page_bytes, out)
    k, v = c.gather(0, np.arange(640))
    want = np.concatenate([k, v], 1).reshape(640, -1)[pos.clip(0, 639)]
    want[[3, T - 2]] = 0
    assert np.array_equal(_host(out), want, equal_nan=True)


# ---------------------------------------------------------------------------
# attention of single tokens
# ---------------------------------------------------------------------------
def _decode(torch, L, c, q, ctx, Hq, window, sinks, max_ctx, kv=None, scratch=None, stream=None):
    need = L.loip_k_window_attention_q8_scratch_bytes(len(ctx), Hq, c.Hkv, c.d, window, sinks, max_ctx)
    if scratch is None:
        scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, float("nan"))
    L.loip_k_window_attention_q8(q, _dev(torch, c.bytes) if kv is None else kv, _dev(torch, c.table), c.max_pages,
                                 _ints(torch, ctx), Hq, c.Hkv, c.d, P, c.layer, c.layer_page_bytes, window, sinks,
                                 max_ctx, scratch, o, stream)
    return o


def _decode_cache(ctx, max_ctx, Hkv, d, window, sinks, seed, **kw):
    """Only what a query sees is written; table entries of other pages lead to a page of NaN."""
    c = Cache8(len(ctx), -(-max_ctx // P), Hkv, d, seed, **kw)
    lean = np.random.default_rng(seed + 1).standard_normal((Hkv, d))
    for r, n in enumerate(ctx):
        js = W.seen_positions([n - 1], window, sinks)
        c.fill_request(r, js, seed + 2 + r, lean={j: lean for j in range(min(sinks, max_ctx))})
        for pg in set(range(c.max_pages)) - {j // P for j in js}:
            c.table[r, pg] = c.nobody
    return c, lean


def _check_decode(torch, L, ctx, Hq, Hkv, d, window, sinks, dtype, seed, max_ctx=None, **kw):
    max_ctx = max_ctx or max(max(ctx), 1)
    c, lean = _decode_cache(ctx, max_ctx, Hkv, d, window, sinks, seed, **kw)
    G = Hq // Hkv
    q = np.random.default_rng(seed + 99).standard_normal((len(ctx), Hkv, G, d)) + 0.5 * lean[None, :, None]
    qd, q64 = _rows(torch, q.reshape(len(ctx), Hq * d).astype(np.float32), dtype)
    got = _host(_decode(torch, L, c, qd, ctx, Hq, window, sinks, max_ctx))
    for r, n in enumerate(ctx):
        want, t32, tbf = W.attend(c, r, n - 1, q64[r].reshape(Hq, d), window, sinks)
        err = np.abs(got[r].reshape(Hq, d) - want)
        assert np.all(err <= (t32 if dtype == "f32" else tbf)), (r, n, float(err.max()))


# contexts of zero and one token, on and around granule and page boundaries
CTX = (0, 1, 2, 15, 16, 17, 63, 64, 65, 129, 200, 321)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (0, 0), (0, 5), (16, 4), (63, 1), (64, 64), (65, 3), (100, 70),
                                          (1000, 0), (2147483647, 2147483647)])
def test_decode_windows(torch, L, window, sinks, dtype):
    _check_decode(torch, L, CTX, 8, 2, 64, window, sinks, dtype, 7)
    _check_decode(torch, L, CTX, 4, 1, 128, window, sinks, dtype, 8, layers=2, layer=1, gap=64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (4, 4, 128), (6, 2, 128), (20, 4, 64), (14, 2, 64), (8, 1, 128),
                                      (32, 8, 128), (64, 8, 128), (9, 1, 64), (16, 1, 128), (40, 2, 64)])
def test_decode_heads(torch, L, Hq, Hkv, d, dtype):
    _check_decode(torch, L, (70, 1, 0, 130), Hq, Hkv, d, 100, 4, dtype, 11)
    _check_decode(torch, L, (257,), Hq, Hkv, d, ALL, 0, dtype, 12)


# one long request among short ones: the length is split, the parts are joined
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("ctx,window,sinks", [((5000,), ALL, 0), ((5000, 3, 0, 2049), 2000, 9),
                                              ((1, 4097, 1025), 4096, 1)])
def test_decode_long(torch, L, ctx, window, sinks, Hq, Hkv, d, dtype):
    _check_decode(torch, L, ctx, Hq, Hkv, d, window, sinks, dtype, 21, max_ctx=8000)


def test_decode_large_scores(torch, L):
    """Scores of several hundred: the running maximum carries the softmax."""
    ctx, Hq, Hkv, d = (300, 77), 4, 2, 64
    c, _ = _decode_cache(ctx, 320, Hkv, d, ALL, 0, 31)
    q = (60 * np.random.default_rng(1).standard_normal((2, Hq * d))).astype(np.float32)
    qd, q64 = _rows(torch, q, "f32")
    got = _host(_decode(torch, L, c, qd, ctx, Hq, ALL, 0, 320))
    for r, n in enumerate(ctx):
        want, t32, _ = W.attend(c, r, n - 1, q64[r].reshape(Hq, d), ALL, 0)
        assert np.all(np.abs(got[r].reshape(Hq, d) - want) <= t32)


# blocks of every size beside one another, the smallest and the largest exponents among them: the
# bound of attend() is relative to the sums of magnitudes, so a block read with another's exponent shows
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["decode", "prefill"])
def test_blocks_of_every_size(torch, L, d, kind):
    n, Hq, Hkv = 150, 4, 2
    c = Cache8(1, 3, Hkv, d, 33)
    rng = np.random.default_rng(34)
    k = rng.standard_normal((n, Hkv, d // 32, 32)) * 2.0 ** rng.integers(-6, 1, (n, Hkv, d // 32, 1))
    v = rng.standard_normal((n, Hkv, d // 32, 32)) * 2.0 ** rng.integers(-100, 100, (n, Hkv, d // 32, 1))
    k[:, :, 0] *= 2.0 ** -110
    v[5], v[6], v[7] = 2.0 ** -125, 127 * 2.0 ** 120, 0.0
    v[6, 0, 1:] = 1.0
    c.put(0, np.arange(n), k.reshape(n, Hkv, d), v.reshape(n, Hkv, d))
    q = rng.standard_normal((1, Hq, d))
    q[:, :, :32] *= 2.0 ** 108
    qd, q64 = _rows(torch, q.reshape(1, Hq * d).astype(np.float32), "f32")
    o = (_decode(torch, L, c, qd, (n,), Hq, ALL, 0, 192) if kind == "decode"
         else _prefill(torch, L, c, qd, [(1, n - 1)], Hq, ALL, 0, 192))
    want, t32, _ = W.attend(c, 0, n - 1, q64[0].reshape(Hq, d), ALL, 0)
    assert np.all(np.abs(_host(o).reshape(Hq, d) - want) <= t32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,E", [(64, -60), (128, -60), (128, 60), (128, -120), (64, 110)])
def test_decode_meets_extreme_blocks_late(torch, L, d, E, dtype):
    """Ordinary blocks first, then values of 2^E (and keys of 2^-60) among them: what was summed before counts on."""
    n, Hq, Hkv = 700, 6, 2
    c = Cache8(2, 11, Hkv, d, 37)
    rng = np.random.default_rng(38)
    for r in range(2):
        k, v = rng.standard_normal((2, n, Hkv, d))
        v[400::37, :, 32:] *= 2.0 ** E
        k[433::64, :, :32] *= 2.0 ** -60
        c.put(r, np.arange(n), k, v)
    q = rng.standard_normal((2, Hq * d)).astype(np.float32)
    qd, q64 = _rows(torch, q, dtype)
    got = _host(_decode(torch, L, c, qd, (n, 399), Hq, ALL, 0, 704))
    for r, ctx in enumerate((n, 399)):
        want, t32, tbf = W.attend(c, r, ctx - 1, q64[r].reshape(Hq, d), ALL, 0)
        assert np.all(np.abs(got[r].reshape(Hq, d) - want) <= (t32 if dtype == "f32" else tbf)), r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["decode", "prefill"])
def test_blocks_of_nan_that_a_row_sees(torch, L, d, dtype, kind):
    """A key's block spoils its kv head's rows, a value's block its own 32 elements; unseen ones nothing."""
    n, Hq, Hkv, window = 200, 6, 3, 90
    c, _ = _decode_cache((n,), 256, Hkv, d, window, 0, 35)
    key, val = c.slot(0, 150, 0)[1], c.slot(0, 177, 1)[1]
    c.bytes[key[1, d // 32 - 1]] = 254
    c.bytes[val[2, 1]] = 255
    q = np.random.default_rng(36).standard_normal((1, Hq * d)).astype(np.float32)
    qd, q64 = _rows(torch, q, dtype)
    o = (_decode(torch, L, c, qd, (n,), Hq, window, 0, 256) if kind == "decode"
         else _prefill(torch, L, c, qd, [(1, n - 1)], Hq, window, 0, 256))
    got = _host(o).reshape(Hkv, Hq // Hkv, d)
    want, t32, tbf = W.attend(c, 0, n - 1, q64[0].reshape(Hq, d), window, 0)
    nan = np.zeros((Hkv, Hq // Hkv, d), dtype=bool)
    nan[1], nan[2, :, 32:64] = True, True
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(np.isnan(want), nan.reshape(Hq, d))
    err = np.abs(got.reshape(Hq, d) - want)[~nan.reshape(Hq, d)]
    assert np.all(err <= (t32 if dtype == "f32" else tbf)[~nan.reshape(Hq, d)])


def test_decode_same_scratch_other_shapes(torch, L):
    """One scratch, zeroed once, serves calls of other shapes; equal calls give equal bits."""
    shapes = [((900, 5, 400), 8, 2, 64, ALL, 0), ((1500,), 4, 1, 64, 1000, 4), ((2, 64), 16, 2, 128, 64, 1),
              ((1900, 640), 8, 2, 128, ALL, 0)]
    need = max(L.loip_k_window_attention_q8_scratch_bytes(len(s[0]), *s[1:], 2048) for s in shapes)
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    first = {}
    for i in (0, 1, 2, 3, 0, 2, 1, 3, 0):
        ctx, Hq, Hkv, d, window, sinks = shapes[i]
        c, _ = _decode_cache(ctx, 2048, Hkv, d, window, sinks, 41 + i)
        q = dev_f32(np.random.default_rng(i).standard_normal((len(ctx), Hq * d)))
        o = _decode(torch, L, c, q, ctx, Hq, window, sinks, 2048, scratch=scratch).cpu().numpy()
        assert np.all(np.isfinite(o))
        assert np.array_equal(o, first.setdefault(i, o))


def test_a_draining_batch_keeps_its_scratch(torch, L):
    """Whole waves of blocks, unsplit ones and equal parts, one after the other."""
    Hq, Hkv, d, max_ctx, most = 16, 8, 64, 2000, 60
    scratch = torch.zeros(L.loip_k_window_attention_q8_scratch_bytes(most, Hq, Hkv, d, ALL, 0, max_ctx),
                          dtype=torch.uint8, device="cuda")
    ctx = [2000, 1, 700] + [40 + b for b in range(most - 3)]
    c, _ = _decode_cache(ctx, max_ctx, Hkv, d, ALL, 0, 3)
    qd, q64 = _rows(torch, np.random.default_rng(4).standard_normal((most, Hq * d)).astype(np.float32), "f32")
    want = [W.attend(c, r, n - 1, q64[r].reshape(Hq, d), ALL, 0)[:2] for r, n in enumerate(ctx)]
    for B in (60, 58, 57, 48, 46, 45, 29, 28, 19, 8, 3, 1):
        got = _host(_decode(torch, L, c, qd[:B], ctx[:B], Hq, ALL, 0, max_ctx, scratch=scratch))
        for r in range(B):
            assert np.all(np.abs(got[r].reshape(Hq, d) - want[r][0]) <= want[r][1]), (B, r)


# ---------------------------------------------------------------------------
# attention of prompts
# ---------------------------------------------------------------------------
def _prefill_cache(runs, max_ctx, Hkv, d, window, sinks, seed):
    """runs: (rows, first position) of each prompt; only what some row sees is written."""
    c = Cache8(len(runs), -(-max_ctx // P), Hkv, d, seed)
    lean = np.random.default_rng(seed + 1).standard_normal((Hkv, d))
    for r, (rows, first) in enumerate(runs):
        js = W.seen_positions(range(first, first + rows), window, sinks)
        c.fill_request(r, js, seed + 2 + r, lean={j: lean for j in range(min(sinks, max_ctx))})
        for pg in set(range(c.max_pages)) - {j // P for j in js}:
            c.table[r, pg] = c.nobody
    return c, lean


def _prefill(torch, L, c, q, runs, Hq, window, sinks, max_ctx, scratch=None, kv=None):
    starts = np.concatenate([[0], np.cumsum([r for r, _ in runs])])
    M = int(starts[-1])
    need = L.loip_k_window_prefill_q8_scratch_bytes(M, len(runs), Hq, c.Hkv, c.d, window, sinks, max_ctx)
    if scratch is None:
        scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, float("nan"))
    L.loip_k_window_prefill_q8(q, _dev(torch, c.bytes) if kv is None else kv, _dev(torch, c.table), c.max_pages,
                               _ints(torch, starts),
                               _ints(torch, [f for _, f in runs]) if any(f for _, f in runs) else None, Hq, c.Hkv, c.d,
                               P, c.layer, c.layer_page_bytes, window, sinks, max_ctx, scratch, o)
    return o


def _check_prefill(torch, L, runs, Hq, Hkv, d, window, sinks, dtype, seed, max_ctx=None, edit=None):
    max_ctx = max_ctx or max(max(f + r for r, f in runs), 1)
    c, lean = _prefill_cache(runs, max_ctx, Hkv, d, window, sinks, seed)
    if edit:
        edit(c)
    M, G = sum(r for r, _ in runs), Hq // Hkv
    q = np.random.default_rng(seed + 99).standard_normal((M, Hkv, G, d)) + 0.5 * lean[None, :, None]
    qd, q64 = _rows(torch, q.reshape(M, Hq * d).astype(np.float32), dtype)
    got = _host(_prefill(torch, L, c, qd, runs, Hq, window, sinks, max_ctx)).reshape(M, Hq, d)
    row = 0
    for r, (rows, first) in enumerate(runs):
        for t in range(rows):
            want, t32, tbf = W.attend(c, r, first + t, q64[row].reshape(Hq, d), window, sinks)
            tol = t32 if dtype == "f32" else tbf
            assert np.array_equal(np.isnan(got[row]), np.isnan(want)), (r, t)
            fine = np.isfinite(want)
            err = np.abs(got[row] - want)[fine]
            assert np.all(err <= tol[fine]), (r, t, float(err.max()))
            row += 1
    return got


RUNS = [(1, 0), (40, 0), (65, 30), (0, 0), (17, 100), (3, 63), (130, 0)]  # a prompt without rows among them


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (0, 0), (0, 5), (16, 4), (64, 64), (65, 3), (100, 70), (ALL, 0),
                                          (2147483647, 2147483647)])
def test_prefill_windows(torch, L, window, sinks, dtype):
    _check_prefill(torch, L, RUNS, 4, 2, 64, window, sinks, dtype, 71)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (2, 2, 128), (6, 2, 128), (5, 1, 64), (7, 1, 128), (8, 1, 128),
                                      (16, 2, 64), (9, 1, 64), (16, 1, 128)])
def test_prefill_heads(torch, L, Hq, Hkv, d, dtype):
    _check_prefill(torch, L, [(70, 3), (33, 0)], Hq, Hkv, d, 50, 4, dtype, 81)


# long enough for several key tiles per row, whole prompts and chunks of them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("runs,window,sinks", [([(300, 0)], ALL, 0), ([(90, 700)], ALL, 0),
                                               ([(90, 700), (200, 411)], 256, 66), ([(260, 513)], 300, 0)])
def test_prefill_long(torch, L, runs, window, sinks, dtype):
    _check_prefill(torch, L, runs, 4, 2, 128, window, sinks, dtype, 91, max_ctx=1000)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_values_that_later_rows_alone_see(torch, L, dtype, d):
    """A value's block of NaN spoils the rows that see it and no other."""
    def edit(c):
        c.bytes[c.slot(0, 20, 1)[1][:, 1]] = 255
        c.bytes[c.slot(0, 90, 1)[1][:, 0]] = 254

    got = _check_prefill(torch, L, [(150, 0)], 4, 2, d, 40, 0, dtype, 101, edit=edit)
    nan = np.zeros(got.shape, dtype=bool)
    nan[20:60, :, 32:64], nan[90:130, :, :32] = True, True
    assert np.array_equal(np.isnan(got), nan)


def test_prefill_keys_that_later_rows_alone_see(torch, L):
    """A key's block of NaN that later rows alone see leaves the earlier rows alone."""
    def edit(c):
        c.bytes[c.slot(0, 37, 0)[1][:, 0]] = 255

    got = _check_prefill(torch, L, [(64, 0)], 4, 2, 64, ALL, 0, "f32", 111, edit=edit)
    assert np.all(np.isfinite(got[:37])) and np.all(np.isnan(got[37:]))


def test_prefill_negative_first_position(torch, L):
    """Rows before position 0 see nothing."""
    got = _check_prefill(torch, L, [(40, -10)], 2, 2, 64, 20, 1, "f32", 121)
    assert np.all(got[:10] == 0)


def test_prefill_many_prompts(torch, L):
    """More prompts than a warp has lanes, single rows among them."""
    runs = [(1 + (i % 3 == 0) * (i % 7), (i * 5) % 60) for i in range(100)]
    _check_prefill(torch, L, runs, 2, 1, 64, 30, 2, "bf16", 131)


# enough row tiles that a block takes two of them (bf16): the second one empty, partly
# filled, full, or with key tiles of its own behind the first one's window
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (40, 3), (150, 70), (0, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefill_many_tiles(torch, L, d, window, sinks, dtype):
    runs = [(300, 0), (129, 70), (128, 500), (0, 9)] + [(1 + i, 30 * i) for i in range(18)]
    _check_prefill(torch, L, runs, 16, 16, d, window, sinks, dtype, 161)


def test_prefill_two_tiles_and_values_that_later_rows_alone_see(torch, L):
    def edit(c):
        c.bytes[c.slot(0, 133, 1)[1][:, 1]] = 255

    runs = [(280, 0)] + [(2, 5)] * 20
    got = _check_prefill(torch, L, runs, 16, 16, 64, 100, 1, "bf16", 171, edit=edit)
    nan = np.zeros(got.shape, dtype=bool)
    nan[133:233, :, 32:] = True
    assert np.array_equal(np.isnan(got), nan)


# enough row tiles per page that images of the pages are made first
IMAGE_RUNS = [(400, 70), (330, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(64, 4, 64), (64, 4, 128)])
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (100, 70), (65, 3)])
def test_prefill_many_tiles_of_a_page(torch, L, Hq, Hkv, d, window, sinks, dtype):
    _check_prefill(torch, L, IMAGE_RUNS, Hq, Hkv, d, window, sinks, dtype, 191, max_ctx=600)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [254, 255, 40, 200])
def test_prefill_many_tiles_of_a_page_and_extreme_exponents(torch, L, E, dtype):
    """NaN that some rows see, and blocks whose exponents images (and loaders) have no form for."""
    def edit(c):
        for which, j in ((1, 133), (0, 260)):
            c.bytes[c.slot(0, j, which)[1][:, 1]] = E if which else min(E, 120)

    got = _check_prefill(torch, L, IMAGE_RUNS[:1] + [(2, 5)], 64, 4, 64, 100, 1, dtype, 201, edit=edit)
    nan = np.zeros(got.shape, dtype=bool)
    if E >= 254:
        nan[133 - 70:233 - 70, :, 32:] = True
    assert np.array_equal(np.isnan(got), nan)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("runs", [[(150, 30)], [(520, 30)]])
def test_prefill_exponents_at_the_borders(torch, L, runs, dtype):
    """Blocks on both sides of the exponents that one product serves, in keys and in values, zeros too."""
    Hkv, d, n = 4, 128, 600
    c = Cache8(1, 10, Hkv, d, 211)
    rng = np.random.default_rng(212)
    k = rng.standard_normal((n, Hkv, d // 32, 32)) * 2.0 ** rng.integers(-70, 1, (n, Hkv, d // 32, 1))
    v = rng.standard_normal((n, Hkv, d // 32, 32)) * 2.0 ** rng.choice([-70, -58, -57, -56, 0, 1, 57, 60], (n, Hkv, d // 32, 1))
    v[::7, :, 1] = 0
    c.put(0, np.arange(n), k.reshape(n, Hkv, d), v.reshape(n, Hkv, d))
    (rows, first), = runs
    q = rng.standard_normal((rows, 64, d)).astype(np.float32)
    qd, q64 = _rows(torch, q.reshape(rows, -1), dtype)
    got = _host(_prefill(torch, L, c, qd, runs, 64, ALL, 2, 600)).reshape(rows, 64, d)
    for t in range(0, rows, 13):
        want, t32, tbf = W.attend(c, 0, first + t, q64[t].reshape(64, d), ALL, 2)
        assert np.all(np.abs(got[t] - want) <= (t32 if dtype == "f32" else tbf)), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_of_captured_calls_change(torch, L, dtype):
    """Two captured calls on one scratch, one of them with images, replayed in turn while the prompts' rows and
    positions change on the device; rows that no prompt has keep what they hold."""
    Hq, Hkv, d, M, ctx = 64, 4, 64, 500, 640
    c = Cache8(3, ctx // P, Hkv, d, 221)
    for r in range(3):
        c.fill_request(r, range(ctx), 222 + r)
    kv, table = _dev(torch, c.bytes), _dev(torch, c.table)
    qd, q64 = _rows(torch, np.random.default_rng(223).standard_normal((M, Hq * d)).astype(np.float32), dtype)
    starts, first = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    need = max(L.loip_k_window_prefill_q8_scratch_bytes(m, 3, Hq, Hkv, d, 200, 3, ctx) for m in (M, 20))
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    graphs = []
    for m in (M, 20):
        o = torch.zeros(m, Hq * d, dtype=qd.dtype, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.loip_k_window_prefill_q8(qd[:m], kv, table, c.max_pages, starts, first, Hq, Hkv, d, P, 0, c.layer_page_bytes,
                                       200, 3, ctx, scratch, o)
        graphs.append((m, g, o))
    for i, (m, rows, at) in enumerate([(M, (300, 200, 0), (0, 440, 9)), (20, (7, 0, 12), (600, 3, 50)),
                                       (M, (1, 2, 390), (639, 0, 250)), (20, (20, 0, 0), (0, 0, 0)),
                                       (M, (0, 0, 480), (5, 5, 160))]):
        starts.copy_(torch.tensor([0, *np.cumsum(rows)]))
        first.copy_(torch.tensor(at))
        _, g, o = graphs[m != M]
        o.fill_(7.0)
        g.replay()
        got = _host(o).reshape(m, Hq, d)
        assert np.all(got[sum(rows):] == 7.0), i
        row = 0
        for r, (n, lo) in enumerate(zip(rows, at)):
            for t in range(0, n, 11):
                want, t32, tbf = W.attend(c, r, lo + t, q64[row + t].reshape(Hq, d), 200, 3)
                assert np.all(np.abs(got[row + t] - want) <= (t32 if dtype == "f32" else tbf)), (i, r, t)
            row += n


def test_prefill_rows_behind_the_last_prompt(torch, L):
    """Rows past row_starts[-1] keep what they hold."""
    c, _ = _prefill_cache([(20, 0)], 64, 2, 64, ALL, 0, 181)
    q = dev_f32(np.random.default_rng(7).standard_normal((33, 4 * 64)))
    scratch = torch.zeros(L.loip_k_window_prefill_q8_scratch_bytes(33, 1, 4, 2, 64, ALL, 0, 64), dtype=torch.uint8,
                          device="cuda")
    o = torch.full_like(q, 7.0)
    L.loip_k_window_prefill_q8(q, _dev(torch, c.bytes), _dev(torch, c.table), 1, _ints(torch, [0, 20]), None, 4, 2, 64,
                               P, 0, c.layer_page_bytes, ALL, 0, 64, scratch, o)
    o = _host(o)
    assert np.all(o[20:] == 7.0) and np.all(np.isfinite(o)) and not np.any(np.all(o[:20] == 7.0, -1))


def test_chunks_of_a_prompt_keep_their_scratch(torch, L):
    """Many rows (no split), then the last few (split over blocks)."""
    Hq, Hkv, d, ctx = 8, 8, 64, 900
    c, _ = _prefill_cache([(ctx, 0)], ctx, Hkv, d, ALL, 0, 5)
    qd, q64 = _rows(torch, np.random.default_rng(6).standard_normal((700, Hq * d)).astype(np.float32), "f32")
    scratch = torch.zeros(L.loip_k_window_prefill_q8_scratch_bytes(700, 1, Hq, Hkv, d, ALL, 0, ctx), dtype=torch.uint8,
                          device="cuda")
    for M in (700, 300, 33, 1):
        got = _host(_prefill(torch, L, c, qd[:M], [(M, ctx - M)], Hq, ALL, 0, ctx, scratch=scratch))
        for t in {0, M // 2, M - 1}:
            want, t32, _ = W.attend(c, 0, ctx - M + t, q64[t].reshape(Hq, d), ALL, 0)
            assert np.all(np.abs(got[t].reshape(Hq, d) - want) <= t32), (M, t)


def test_prefill_equals_decode(torch, L):
    """A prompt of one row is a decode step: both agree to the sum of their bounds."""
    ctx, Hq, Hkv, d = (500, 1, 77), 8, 2, 128
    c, _ = _decode_cache(ctx, 512, Hkv, d, 200, 4, 141)
    q = dev_f32(np.random.default_rng(6).standard_normal((3, Hq * d)))
    a = _host(_decode(torch, L, c, q, ctx, Hq, 200, 4, 512))
    b = _host(_prefill(torch, L, c, q, [(1, n - 1) for n in ctx], Hq, 200, 4, 512))
    for r, n in enumerate(ctx):
        _, t32, _ = W.attend(c, r, n - 1, _host(q)[r].reshape(Hq, d), 200, 4)
        assert np.all(np.abs(a[r] - b[r]).reshape(Hq, d) <= 2 * t32)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
def test_one_scratch_for_every_attention(torch, L):
    """Single tokens and prompts, over this cache and the bf16 one, in turn on one scratch."""
    import test_gpu_window as B
    Hq, Hkv, d, n, window, sinks = 8, 2, 64, 1500, 1200, 3
    c8, _ = _decode_cache((n,), 1536, Hkv, d, window, sinks, 151)
    cb, _ = B._decode_cache((n,), 1536, Hkv, d, window, sinks, 151)
    args = (Hq, Hkv, d, window, sinks, 1536)
    need = max(L.loip_k_window_attention_q8_scratch_bytes(1, *args), L.loip_k_window_prefill_q8_scratch_bytes(1, 1, *args),
               L.loip_k_window_attention_scratch_bytes(1, *args), L.loip_k_window_prefill_scratch_bytes(1, 1, *args))
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    q = dev_f32(np.random.default_rng(8).standard_normal((1, Hq * d)))
    calls = [lambda s: _decode(torch, L, c8, q, (n,), Hq, window, sinks, 1536, scratch=s),
             lambda s: _prefill(torch, L, c8, q, [(1, n - 1)], Hq, window, sinks, 1536, scratch=s),
             lambda s: B._decode(torch, L, cb, q, (n,), Hq, window, sinks, 1536, scratch=s),
             lambda s: B._prefill(torch, L, cb, q, [(1, n - 1)], Hq, window, sinks, 1536, scratch=s)]
    alone = [f(None).cpu().numpy() for f in calls]
    for i in (0, 1, 2, 3, 1, 0, 3, 2, 0):
        assert np.array_equal(calls[i](scratch).cpu().numpy(), alone[i]), i


def test_offsets_past_32_bits(torch, L):
    """Pages that lie more than 4 GiB into the cache, for all four operators."""
    Hq, Hkv, d, n = 4, 2, 64, 100
    c = Cache8(1, 2, Hkv, d, 61)
    c.fill_request(0, range(n - 1), 62)
    base = 5 << 30
    kv = torch.zeros(base + c.bytes.nbytes, dtype=torch.uint8, device="cuda")
    kv[base:] = _dev(torch, c.bytes)
    table = _dev(torch, c.table) + base
    rng = np.random.default_rng(63)
    x = rng.standard_normal((1, (Hq + 2 * Hkv) * d)).astype(np.float32)
    q = torch.empty(1, Hq * d, device="cuda")
    L.loip_k_qk_append_q8(dev_f32(x), None, None, Hq, Hkv, d, 0.0, 0.0, _ints(torch, [n - 1]), None, q, kv, table, 2, P,
                          0, c.layer_page_bytes)
    kvx = x[0, Hq * d:].reshape(2, Hkv, d)
    c.put(0, n - 1, kvx[0], kvx[1])
    out = torch.empty(1, 2 * Hkv * d, device="cuda")
    L.loip_k_cache_read_q8(kv, table, 2, _ints(torch, [n - 1]), None, Hkv, d, P, 0, c.layer_page_bytes, out)
    assert np.array_equal(_host(out).reshape(2, Hkv, d), Q.decode(*Q.encode(kvx)))
    want, t32, _ = W.attend(c, 0, n - 1, x[0, :Hq * d].astype(np.float64).reshape(Hq, d), 90, 2)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    scratch = torch.zeros(max(L.loip_k_window_attention_q8_scratch_bytes(1, Hq, Hkv, d, 90, 2, 128),
                              L.loip_k_window_prefill_q8_scratch_bytes(1, 1, Hq, Hkv, d, 90, 2, 128)),
                          dtype=torch.uint8, device="cuda")
    L.loip_k_window_attention_q8(q, kv, table, 2, _ints(torch, [n]), Hq, Hkv, d, P, 0, c.layer_page_bytes, 90, 2, 128,
                                 scratch, o)
    L.loip_k_window_prefill_q8(q, kv, table, 2, _ints(torch, [0, 1]), _ints(torch, [n - 1]), Hq, Hkv, d, P, 0,
                               c.layer_page_bytes, 90, 2, 128, scratch, o2)
    for got in (o, o2):
        assert np.all(np.abs(_host(got).reshape(Hq, d) - want) <= t32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_run_of_all_four(torch, L, dtype):
    """A prompt in two chunks, then single tokens, without a wait in between, and once more from a
    captured graph on another stream: what is read back is the appended rows rounded once, and the
    attention that of the rows read back."""
    Hq, Hkv, d, chunks, steps, window, sinks, theta = 8, 2, 128, (70, 45), 5, 80, 3, 1e4
    n = sum(chunks) + steps
    pages = -(-n // P)
    tdt = torch.float32 if dtype == "f32" else torch.bfloat16
    x, x64 = _rows(torch, np.random.default_rng(11).standard_normal((n, (Hq + 2 * Hkv) * d)).astype(np.float32), dtype)
    c = Cache8(1, pages, Hkv, d, 12)
    kv, table = _dev(torch, c.bytes), _dev(torch, c.table)
    q, o = (torch.zeros(n, Hq * d, dtype=tdt, device="cuda") for _ in range(2))
    out = torch.zeros(n, 2 * Hkv * d, device="cuda")
    pos, req = _ints(torch, range(n)), torch.zeros(n, dtype=torch.int32, device="cuda")
    args = (Hq, Hkv, d, window, sinks, n)
    scratch = torch.zeros(max(L.loip_k_window_attention_q8_scratch_bytes(1, *args),
                              L.loip_k_window_prefill_q8_scratch_bytes(max(chunks), 1, *args)), dtype=torch.uint8,
                          device="cuda")
    runs = [(0, chunks[0]), (chunks[0], sum(chunks))] + [(i, i + 1) for i in range(sum(chunks), n)]
    starts = [_ints(torch, [0, hi - lo]) for lo, hi in runs]
    firsts, lens = [_ints(torch, [lo]) for lo, _ in runs], [_ints(torch, [hi]) for _, hi in runs]
    lpb = c.layer_page_bytes

    def run():
        for i, (lo, hi) in enumerate(runs):
            L.loip_k_qk_append_q8(x[lo:hi], None, None, Hq, Hkv, d, 0.0, theta, pos[lo:hi], req[lo:hi], q[lo:hi], kv,
                                  table, pages, P, 0, lpb)
            if hi - lo > 1:
                L.loip_k_window_prefill_q8(q[lo:hi], kv, table, pages, starts[i], firsts[i], Hq, Hkv, d, P, 0, lpb,
                                           window, sinks, n, scratch, o[lo:hi])
            else:
                L.loip_k_window_attention_q8(q[lo:hi], kv, table, pages, lens[i], Hq, Hkv, d, P, 0, lpb, window, sinks,
                                             n, scratch, o[lo:hi])
        L.loip_k_cache_read_q8(kv, table, pages, pos, req, Hkv, d, P, 0, lpb, out)

    run()
    first = [t.float().cpu().numpy() for t in (q, o, out)]
    held = first[2].astype(np.float64).reshape(n, 2, Hkv, d)
    for t in range(n):
        wq, wk, wv, tq, tk = W.append_row(x64[t], t, Hq, Hkv, d, None, None, 0.0, theta)
        most = (np.abs(wk) + tk).reshape(Hkv, d // 32, 32).max(-1)
        assert np.all(np.abs(held[t, 0] - wk) <= tk + np.repeat(Q.half_step(most), 32, -1)), t
        assert np.array_equal(held[t, 1], Q.decode(*Q.encode(wv))), t
        c.put(0, t, held[t, 0], held[t, 1])  # (a held row rounds to itself)
    assert np.array_equal(c.gather(0, range(n))[0], held[:, 0])
    for t in range(n):
        want, t32, tbf = W.attend(c, 0, t, first[0][t].astype(np.float64).reshape(Hq, d), window, sinks)
        assert np.all(np.abs(first[1][t].reshape(Hq, d) - want) <= (t32 if dtype == "f32" else tbf)), t
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(2):
        for t in (q, o, out):
            t.zero_()
        kv.fill_(255)
        graph.replay()
        for t, want in zip((q, o, out), first):
            assert np.array_equal(t.float().cpu().numpy(), want)
