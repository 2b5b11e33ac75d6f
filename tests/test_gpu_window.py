"""The windowed-serving operators on the GPU against a plain 64-bit implementation:
append with norm and rotation, attention of single tokens and of prompts behind a
sliding window with sinks.  Unwritten cache elements are NaN, and page-table
entries of pages that no row may read point at a page of NaN."""
import numpy as np
import pytest

import window_ref as W
from gpu_util import dev_bits, dev_f32, need_gpu
from window_ref import P, U, Cache

pytestmark = pytest.mark.gpu


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


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
# ragged requests out of order, padding rows, rows wider than their heads, a cache of
# several layers; head sizes 64 and 128 with 1 to 8 query heads per kv head
@pytest.mark.parametrize("T", [1, 7, 130])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (7, 7, 64), (12, 4, 128), (64, 8, 128)])
@pytest.mark.parametrize("dtype,norm", [("f32", True), ("f32", False), ("bf16", True), ("bf16", False)])
def test_append_parity(torch, L, T, Hq, Hkv, d, dtype, norm):
    rng = np.random.default_rng(T * 100 + Hq)
    R, pages, theta, eps = 3, 4, 500000.0, 1e-6
    c = Cache(R, pages, Hkv, d, 5, layers=3, layer=1, gap=256)
    slots = rng.permutation(R * pages * P)[:T]
    req, pos = (slots // (pages * P)).astype(np.int32), (slots % (pages * P)).astype(np.int32)
    if T > 1:  # padding: no position, a position past the table, no such request
        pos[1], pos[-1] = -1, pages * P
        req[T // 2] = (R, -1)[T % 2]
    width = (Hq + 2 * Hkv) * d
    x = (rng.standard_normal((T, width + 16)) * 1.5).astype(np.float32)
    xd, x64 = _rows(torch, x, dtype)
    g = [1 + 0.1 * rng.standard_normal(d) for _ in range(2)] if norm else [None, None]
    gb = [None if v is None else W.bf16_bits(v) for v in g]
    g64 = [None if v is None else W.bits_f64(v) for v in gb]
    kv, q = dev_bits(c.bits), torch.full((T, Hq * d), float("nan"), dtype=xd.dtype, device="cuda")
    L.loip_k_qk_append(xd[:, :width], *[None if v is None else dev_bits(v) for v in gb], Hq, Hkv, d, eps, theta,
                       _ints(torch, pos), _ints(torch, req), q, kv, torch.from_numpy(c.table).cuda(), pages, P,
                       c.layer, c.layer_page_bytes)
    got_q, got = _host(q).reshape(T, Hq, d), kv.cpu().numpy().view(np.uint16)
    want = c.bits.copy()
    for t in range(T):
        if not (0 <= pos[t] < pages * P and 0 <= req[t] < R):
            assert np.all(got_q[t] == 0)
            continue
        wq, wk, wv, tq, tk = W.append_row(x64[t, :width], int(pos[t]), Hq, Hkv, d, *g64, eps, theta)
        half = 0 if dtype == "f32" else 2.0 ** -8
        assert np.all(np.abs(got_q[t] - wq) <= tq + half * (np.abs(wq) + tq)), t
        ik, iv = c.slot(req[t], pos[t], 0), c.slot(req[t], pos[t], 1)
        assert np.all(np.abs(W.bits_f64(got[ik]) - wk) <= tk + 2.0 ** -8 * (np.abs(wk) + tk)), t
        assert np.array_equal(got[iv], W.bf16_bits(wv.astype(np.float32)))
        want[ik], want[iv] = got[ik], got[iv]
    assert np.array_equal(got, want)  # nothing else was written


# positions far out, where an fp32 angle has no digits left, and no rotation at all
@pytest.mark.parametrize("theta", [500000.0, 10000.0, 1.0, 0.0])
def test_append_far_positions(torch, L, theta):
    Hq, Hkv, d, pages = 2, 1, 128, 1 << 20
    pos = np.array([0, 1, 63, 64, 131071, 1 << 20, (1 << 26) - 1], dtype=np.int32)
    T = len(pos)
    x = np.random.default_rng(3).standard_normal((T, (Hq + 2 * Hkv) * d)).astype(np.float32)
    table = torch.zeros(1, pages, dtype=torch.int64, device="cuda")  # one page stands for all: only q is looked at
    kv = torch.zeros(2 * Hkv * P * d, dtype=torch.int16, device="cuda")
    q = torch.empty(T, Hq * d, device="cuda")
    L.loip_k_qk_append(dev_f32(x), None, None, Hq, Hkv, d, 0.0, theta, _ints(torch, pos),
                       torch.zeros(T, dtype=torch.int32, device="cuda"), q, kv, table, pages, P, 0, 2 * Hkv * P * d * 2)
    for t in range(T):
        wq, _, _, tq, _ = W.append_row(x[t].astype(np.float64), int(pos[t]), Hq, Hkv, d, None, None, 0.0, theta)
        assert np.all(np.abs(_host(q)[t].reshape(Hq, d) - wq) <= tq), (t, theta)


def test_append_identity_rows_and_no_rows(torch, L):
    """row_req None: row t is request t; zero rows launch nothing."""
    Hq, Hkv, d, R = 4, 4, 64, 5
    c = Cache(R, 1, Hkv, d, 1)
    x = np.random.default_rng(4).standard_normal((R, 3 * Hq * d)).astype(np.float32)
    kv, table = dev_bits(c.bits), torch.from_numpy(c.table).cuda()
    q = torch.empty(R, Hq * d, device="cuda")
    args = (None, None, Hq, Hkv, d, 0.0, 0.0)
    L.loip_k_qk_append(dev_f32(x)[:0], *args, _ints(torch, []), None, q[:0], kv, table, 1, P, 0, c.layer_page_bytes)
    assert np.array_equal(kv.cpu().numpy().view(np.uint16), c.bits)
    L.loip_k_qk_append(dev_f32(x), *args, _ints(torch, range(R)), None, q, kv, table, 1, P, 0, c.layer_page_bytes)
    assert np.array_equal(q.cpu().numpy(), x[:, :Hq * d])
    got = kv.cpu().numpy().view(np.uint16)
    for r in range(R):
        assert np.array_equal(got[c.slot(r, r, 1)].ravel(), W.bf16_bits(x[r, 2 * Hq * d:]))


# ---------------------------------------------------------------------------
# attention of single tokens
# ---------------------------------------------------------------------------
def _decode(torch, L, c, q, ctx, Hq, window, sinks, max_ctx, kv=None, scratch=None, stream=None):
    need = L.loip_k_window_attention_scratch_bytes(len(ctx), Hq, c.Hkv, c.d, window, sinks, max_ctx)
    if scratch is None:
        scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, float("nan"))
    L.loip_k_window_attention(q, dev_bits(c.bits) if kv is None else kv, torch.from_numpy(c.table).cuda(),
                              c.max_pages, _ints(torch, ctx), Hq, c.Hkv, c.d, P, c.layer, c.layer_page_bytes, window,
                              sinks, max_ctx, scratch, o, stream)
    return o


def _decode_cache(ctx, max_ctx, Hkv, d, window, sinks, seed, **kw):
    """Only what a query sees is written; table entries of other pages lead to a page of NaN."""
    c = Cache(len(ctx), -(-max_ctx // P), Hkv, d, seed, **kw)
    lean = np.random.default_rng(seed + 1).standard_normal((Hkv, d))
    for r, n in enumerate(ctx):
        js = W.seen_positions([n - 1], window, sinks)
        c.fill_request(r, js, seed + 2 + r, lean={j: lean for j in range(min(sinks, max_ctx))})
        for pg in set(range(c.max_pages)) - {j // P for j in js}:
            c.table[r, pg] = c.nobody
    return c, lean


def _check_decode(torch, L, ctx, Hq, Hkv, d, window, sinks, dtype, seed, max_ctx=None):
    max_ctx = max_ctx or max(max(ctx), 1)
    c, lean = _decode_cache(ctx, max_ctx, Hkv, d, window, sinks, seed)
    G = Hq // Hkv
    q = np.random.default_rng(seed + 99).standard_normal((len(ctx), Hkv, G, d)) + 0.5 * lean[None, :, None]
    qd, q64 = _rows(torch, q.reshape(len(ctx), Hq * d).astype(np.float32), dtype)
    got = _host(_decode(torch, L, c, qd, ctx, Hq, window, sinks, max_ctx))
    for r, n in enumerate(ctx):
        want, t32, tbf = W.attend(c, r, n - 1, q64[r].reshape(Hq, d), window, sinks)
        err = np.abs(got[r].reshape(Hq, d) - want)
        assert np.all(err <= (t32 if dtype == "f32" else tbf)), (r, n, float(err.max()))


# contexts of zero and one token, on and around page boundaries
CTX = (0, 1, 2, 15, 16, 17, 63, 64, 65, 129, 200, 321)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (0, 0), (0, 5), (16, 4), (63, 1), (64, 64), (65, 3), (100, 70),
                                          (1000, 0), (2147483647, 2147483647)])
def test_decode_windows(torch, L, window, sinks, dtype):
    _check_decode(torch, L, CTX, 8, 2, 64, window, sinks, dtype, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (4, 4, 128), (6, 2, 128), (20, 4, 64), (14, 2, 64), (8, 1, 128),
                                      (32, 8, 128), (64, 8, 128), (9, 1, 64), (16, 1, 128), (40, 2, 64)])
def test_decode_heads(torch, L, Hq, Hkv, d, dtype):
    _check_decode(torch, L, (70, 1, 0, 130), Hq, Hkv, d, 100, 4, dtype, 11)
    _check_decode(torch, L, (257,), Hq, Hkv, d, 1 << 30, 0, dtype, 12)


# one long request among short ones: the length is split, the parts are joined
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ctx,window,sinks", [((5000,), 1 << 30, 0), ((5000, 3, 0, 2049), 2000, 9),
                                              ((1, 4097, 1025), 4096, 1)])
def test_decode_long(torch, L, ctx, window, sinks, dtype):
    _check_decode(torch, L, ctx, 4, 2, 64, window, sinks, dtype, 21, max_ctx=8000)


def test_decode_large_scores(torch, L):
    """Scores of several hundred: the running maximum carries the softmax."""
    ctx, Hq, Hkv, d = (300, 77), 4, 2, 64
    c, _ = _decode_cache(ctx, 320, Hkv, d, 1 << 30, 0, 31)
    q = (60 * np.random.default_rng(1).standard_normal((2, Hq * d))).astype(np.float32)
    qd, q64 = _rows(torch, q, "f32")
    got = _host(_decode(torch, L, c, qd, ctx, Hq, 1 << 30, 0, 320))
    for r, n in enumerate(ctx):
        want, t32, _ = W.attend(c, r, n - 1, q64[r].reshape(Hq, d), 1 << 30, 0)
        assert np.all(np.abs(got[r].reshape(Hq, d) - want) <= t32)


def test_decode_same_scratch_other_shapes(torch, L):
    """One scratch, zeroed once, serves calls of other shapes; equal calls give equal bits."""
    shapes = [((900, 5, 400), 8, 2, 64, 1 << 30, 0), ((1500,), 4, 1, 64, 1000, 4), ((2, 64), 16, 2, 128, 64, 1)]
    need = max(L.loip_k_window_attention_scratch_bytes(len(s[0]), *s[1:], 2048) for s in shapes)
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    first = {}
    for i in (0, 1, 2, 0, 2, 1, 0):
        ctx, Hq, Hkv, d, window, sinks = shapes[i]
        c, _ = _decode_cache(ctx, 2048, Hkv, d, window, sinks, 41 + i)
        q = dev_f32(np.random.default_rng(i).standard_normal((len(ctx), Hq * d)))
        o = _decode(torch, L, c, q, ctx, Hq, window, sinks, 2048, scratch=scratch).cpu().numpy()
        assert np.all(np.isfinite(o))
        assert np.array_equal(o, first.setdefault(i, o))


def test_decode_on_another_stream_and_in_a_graph(torch, L):
    ctx, Hq, Hkv, d = (700, 33), 8, 2, 64
    c, _ = _decode_cache(ctx, 704, Hkv, d, 512, 4, 51)
    q = dev_f32(np.random.default_rng(5).standard_normal((2, Hq * d)))
    want = _decode(torch, L, c, q, ctx, Hq, 512, 4, 704).cpu().numpy()
    kv, table, lens = dev_bits(c.bits), torch.from_numpy(c.table).cuda(), _ints(torch, ctx)
    scratch = torch.zeros(L.loip_k_window_attention_scratch_bytes(2, Hq, Hkv, d, 512, 4, 704), dtype=torch.uint8,
                          device="cuda")
    o = torch.zeros_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def call():
        L.loip_k_window_attention(q, kv, table, c.max_pages, lens, Hq, Hkv, d, P, 0, c.layer_page_bytes, 512, 4, 704,
                                  scratch, o)

    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert np.array_equal(o.cpu().numpy(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        o.zero_()
        graph.replay()
        assert np.array_equal(o.cpu().numpy(), want)


def test_offsets_past_32_bits(torch, L):
    """Pages that lie more than 4 GiB into the cache, for all three operators."""
    Hq, Hkv, d, n = 4, 2, 64, 100
    c = Cache(1, 2, Hkv, d, 61)
    c.fill_request(0, range(n - 1), 62)
    base = 5 << 30
    kv = torch.zeros((base + c.bits.nbytes) // 2, dtype=torch.int16, device="cuda")
    kv[base // 2:] = dev_bits(c.bits)
    table = torch.from_numpy(c.table).cuda() + base
    rng = np.random.default_rng(63)
    x = rng.standard_normal((1, (Hq + 2 * Hkv) * d)).astype(np.float32)
    q = torch.empty(1, Hq * d, device="cuda")
    L.loip_k_qk_append(dev_f32(x), None, None, Hq, Hkv, d, 0.0, 0.0, _ints(torch, [n - 1]), None, q, kv, table, 2, P,
                       0, c.layer_page_bytes)
    c.put(0, n - 1, W.bf16_bits(x[0, Hq * d:(Hq + Hkv) * d].reshape(Hkv, d)),
          W.bf16_bits(x[0, (Hq + Hkv) * d:].reshape(Hkv, d)))
    want, t32, _ = W.attend(c, 0, n - 1, x[0, :Hq * d].astype(np.float64).reshape(Hq, d), 90, 2)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    scratch = torch.zeros(max(L.loip_k_window_attention_scratch_bytes(1, Hq, Hkv, d, 90, 2, 128),
                              L.loip_k_window_prefill_scratch_bytes(1, 1, Hq, Hkv, d, 90, 2, 128)),
                          dtype=torch.uint8, device="cuda")
    L.loip_k_window_attention(q, kv, table, 2, _ints(torch, [n]), Hq, Hkv, d, P, 0, c.layer_page_bytes, 90, 2, 128,
                              scratch, o)
    L.loip_k_window_prefill(q, kv, table, 2, _ints(torch, [0, 1]), _ints(torch, [n - 1]), Hq, Hkv, d, P, 0,
                            c.layer_page_bytes, 90, 2, 128, scratch, o2)
    for got in (o, o2):
        assert np.all(np.abs(_host(got).reshape(Hq, d) - want) <= t32)


# ---------------------------------------------------------------------------
# attention of prompts
# ---------------------------------------------------------------------------
def _prefill_cache(runs, max_ctx, Hkv, d, window, sinks, seed):
    """runs: (rows, first position) of each prompt; only what some row sees is written."""
    c = Cache(len(runs), -(-max_ctx // P), Hkv, d, seed)
    lean = np.random.default_rng(seed + 1).standard_normal((Hkv, d))
    for r, (rows, first) in enumerate(runs):
        js = W.seen_positions(range(first, first + rows), window, sinks)
        c.fill_request(r, js, seed + 2 + r, lean={j: lean for j in range(min(sinks, max_ctx))})
        for pg in set(range(c.max_pages)) - {j // P for j in js}:
            c.table[r, pg] = c.nobody
    return c, lean


def _prefill(torch, L, c, q, runs, Hq, window, sinks, max_ctx, scratch=None):
    starts = np.concatenate([[0], np.cumsum([r for r, _ in runs])])
    M = int(starts[-1])
    need = L.loip_k_window_prefill_scratch_bytes(M, len(runs), Hq, c.Hkv, c.d, window, sinks, max_ctx)
    if scratch is None:
        scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, float("nan"))
    L.loip_k_window_prefill(q, dev_bits(c.bits), torch.from_numpy(c.table).cuda(), c.max_pages, _ints(torch, starts),
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
@pytest.mark.parametrize("window,sinks", [(1, 0), (0, 0), (0, 5), (16, 4), (64, 64), (65, 3), (100, 70), (1 << 30, 0),
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
@pytest.mark.parametrize("runs,window,sinks", [([(300, 0)], 1 << 30, 0), ([(90, 700)], 1 << 30, 0),
                                               ([(90, 700), (200, 411)], 256, 66), ([(260, 513)], 300, 0)])
def test_prefill_long(torch, L, runs, window, sinks, dtype):
    _check_prefill(torch, L, runs, 4, 2, 128, window, sinks, dtype, 91, max_ctx=1000)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefill_values_that_later_rows_alone_see(torch, L, dtype):
    """A NaN and an infinity in cached values spoil the rows that see them and no other."""
    bad = {20: np.nan, 90: np.inf}

    def edit(c):
        for j, v in bad.items():
            bits = c.bits[c.slot(0, j, 1)].copy()
            bits[:, 5] = 0x7FC0 if np.isnan(v) else 0x7F80
            c.bits[c.slot(0, j, 1)] = bits

    with np.errstate(invalid="ignore"):
        got = _check_prefill(torch, L, [(150, 0)], 4, 2, 64, 40, 0, dtype, 101, edit=edit)
    assert np.all(np.isfinite(got[:20])) and np.all(np.isnan(got[20:60, :, 5]))
    assert np.all(np.isposinf(got[90:130, :, 5])) and np.all(np.isfinite(got[130:]))
    assert np.all(np.isfinite(np.delete(got, 5, axis=-1)))


def test_prefill_keys_that_no_row_sees(torch, L):
    """A key of NaN that later rows alone see leaves the earlier rows alone."""
    def edit(c):
        bits = c.bits[c.slot(0, 37, 0)].copy()
        bits[:, 0] = 0x7FC0
        c.bits[c.slot(0, 37, 0)] = bits

    with np.errstate(invalid="ignore"):
        got = _check_prefill(torch, L, [(64, 0)], 4, 2, 64, 1 << 30, 0, "f32", 111, edit=edit)
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
@pytest.mark.parametrize("window,sinks", [(1 << 30, 0), (40, 3), (150, 70), (0, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefill_many_tiles(torch, L, d, window, sinks, dtype):
    runs = [(300, 0), (129, 70), (128, 500), (0, 9)] + [(1 + i, 30 * i) for i in range(18)]
    _check_prefill(torch, L, runs, 16, 16, d, window, sinks, dtype, 161)


def test_prefill_two_tiles_and_values_that_later_rows_alone_see(torch, L):
    def edit(c):
        bits = c.bits[c.slot(0, 133, 1)].copy()
        bits[:, 7] = 0xFF80  # minus infinity
        c.bits[c.slot(0, 133, 1)] = bits

    runs = [(280, 0)] + [(2, 5)] * 20
    got = _check_prefill(torch, L, runs, 16, 16, 64, 100, 1, "bf16", 171, edit=edit)
    assert np.all(np.isfinite(got[:133])) and np.all(np.isneginf(got[133:233, :, 7])) and np.all(np.isfinite(got[233:]))


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


def test_one_scratch_for_both_attentions(torch, L):
    """Prompts whose row tiles are split leave the scratch usable for single tokens, and the reverse."""
    ctx, Hq, Hkv, d = (900, 640), 8, 2, 64
    c, _ = _decode_cache(ctx, 1024, Hkv, d, 1 << 30, 0, 181)
    q = dev_f32(np.random.default_rng(8).standard_normal((2, Hq * d)))
    runs = [(1, n - 1) for n in ctx]
    need = max(L.loip_k_window_attention_scratch_bytes(2, Hq, Hkv, d, 1 << 30, 0, 1024),
               L.loip_k_window_prefill_scratch_bytes(2, 2, Hq, Hkv, d, 1 << 30, 0, 1024))
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    a0 = b0 = None
    for _ in range(4):
        a = _decode(torch, L, c, q, ctx, Hq, 1 << 30, 0, 1024, scratch=scratch).cpu().numpy()
        b = _prefill(torch, L, c, q, runs, Hq, 1 << 30, 0, 1024, scratch=scratch).cpu().numpy()
        a0, b0 = (a, b) if a0 is None else (a0, b0)
        assert np.array_equal(a, a0) and np.array_equal(b, b0) and np.all(np.isfinite(a)) and np.all(np.isfinite(b))


def test_prefill_same_scratch_and_graph(torch, L):
    runs, Hq, Hkv, d = [(20, 600), (7, 3)], 4, 2, 64
    c, _ = _prefill_cache(runs, 640, Hkv, d, 1 << 30, 0, 151)
    q = dev_f32(np.random.default_rng(7).standard_normal((27, Hq * d)))
    need = L.loip_k_window_prefill_scratch_bytes(27, 2, Hq, Hkv, d, 1 << 30, 0, 640)
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    want = _prefill(torch, L, c, q, runs, Hq, 1 << 30, 0, 640, scratch=scratch).cpu().numpy()
    kv, table = dev_bits(c.bits), torch.from_numpy(c.table).cuda()
    starts, first, o = _ints(torch, [0, 20, 27]), _ints(torch, [600, 3]), torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.loip_k_window_prefill(q, kv, table, c.max_pages, starts, first, Hq, Hkv, d, P, 0, c.layer_page_bytes,
                                1 << 30, 0, 640, scratch, o)
    for _ in range(3):
        o.zero_()
        graph.replay()
        assert np.array_equal(o.cpu().numpy(), want)


# ---------------------------------------------------------------------------
# refusals (the CPU tests hold the complete list)
# ---------------------------------------------------------------------------
def test_refusals_of_the_binding(torch, L):
    Hq, Hkv, d = 4, 2, 64
    c = Cache(1, 1, Hkv, d, 1)
    kv, table = dev_bits(c.bits), torch.from_numpy(c.table).cuda()
    q = torch.zeros(1, Hq * d, device="cuda")
    scratch = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")

    def decode(q=q, o=None, scratch=scratch, window=4):
        L.loip_k_window_attention(q, kv, table, 1, _ints(torch, [1]), Hq, Hkv, d, P, 0, c.layer_page_bytes, window, 0,
                                  64, scratch, torch.empty_like(q) if o is None else o)

    decode()
    for bad in (dict(q=q.double()), dict(q=q.half()), dict(o=q.bfloat16()), dict(o=q[:, :64]), dict(window=-1),
                dict(scratch=scratch[:0]), dict(scratch=scratch[1:])):
        with pytest.raises(L.LoipError) as e:
            decode(**bad)
        assert e.value.code == L.ERR_INVALID
    for call in (lambda: L.loip_k_window_attention(q, kv, table, 1, _ints(torch, []), Hq, Hkv, d, P, 0,
                                                   c.layer_page_bytes, 4, 0, 64, scratch, torch.empty_like(q)),
                 lambda: L.loip_k_window_prefill(q, kv, table, 2, _ints(torch, [0, 1]), None, Hq, Hkv, d, P, 0,
                                                 c.layer_page_bytes, 4, 0, 64, scratch, torch.empty_like(q)),
                 lambda: L.loip_k_qk_append(torch.zeros(1, 8 * d, device="cuda"), None, None, Hq, Hkv, d, 0.0, 0.0,
                                            _ints(torch, [0]), _ints(torch, []), q, kv, table, 1, P, 0,
                                            c.layer_page_bytes)):
        with pytest.raises(L.LoipError):  # arrays shorter than the rows
            call()
    with pytest.raises(L.LoipError, match="both gains"):
        L.loip_k_qk_append(torch.zeros(1, 8 * d, device="cuda"), dev_bits(np.zeros(d, np.uint16)), None, Hq, Hkv, d,
                           0.0, 0.0, _ints(torch, [0]), None, q, kv, table, 1, P, 0, c.layer_page_bytes)
