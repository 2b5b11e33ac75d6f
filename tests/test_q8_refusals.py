"""Argument checks of the 8-bit cache's operators, on a machine without a GPU: of the library
(every call is refused, or has no rows, before CUDA is touched) and of the binding."""
import pytest

from paper_2512_21835_gb300 import loip

torch = pytest.importorskip("torch")

A = 1 << 20  # a 16-byte aligned dummy address
LPB = 2 * 132 * 64


@pytest.fixture(scope="module")
def L():
    from paper_2512_21835_gb300 import build
    build.build()
    if torch.cuda.is_available():
        pytest.skip("dummy pointers: run only where no CUDA device exists")
    return loip.lib()


CACHE = dict(kv=2 * A, table=3 * A, max_pages=4, page_tokens=64, layer=0, lpb=LPB)


def append(L, x=A, dtype=0, stride=512, T=2, Hq=4, Hkv=2, d=64, gq=None, gk=None, eps=1e-6, theta=1e4, pos=4 * A,
           req=None, n_req=2, q=5 * A, **kw):
    c = dict(CACHE, **kw)
    return L.loip_k_qk_append_q8(x, dtype, stride, T, Hq, Hkv, d, gq, gk, eps, theta, pos, req, n_req, q, c["kv"],
                                 c["table"], c["max_pages"], c["page_tokens"], c["layer"], c["lpb"], None)


def read(L, o=A, dtype=0, T=2, Hkv=2, d=64, pos=4 * A, req=None, n_req=2, **kw):
    c = dict(CACHE, **kw)
    return L.loip_k_cache_read_q8(c["kv"], c["table"], c["max_pages"], pos, req, n_req, T, Hkv, d, c["page_tokens"],
                                  c["layer"], c["lpb"], o, dtype, None)


def decode(L, q=A, dtype=0, ctx=4 * A, B=2, Hq=4, Hkv=2, d=64, window=8, sinks=1, max_ctx=256, scratch=6 * A,
           nbytes=None, o=5 * A, **kw):
    c = dict(CACHE, **kw)
    if nbytes is None:
        nbytes = L.loip_k_window_attention_q8_scratch_bytes(B, Hq, Hkv, d, window, sinks, max_ctx)
    return L.loip_k_window_attention_q8(q, dtype, c["kv"], c["table"], c["max_pages"], ctx, B, Hq, Hkv, d,
                                        c["page_tokens"], c["layer"], c["lpb"], window, sinks, max_ctx, scratch, nbytes,
                                        o, None)


def prefill(L, q=A, dtype=0, starts=4 * A, first=None, n=2, M=9, Hq=4, Hkv=2, d=64, window=8, sinks=1, max_ctx=256,
            scratch=6 * A, nbytes=None, o=5 * A, **kw):
    c = dict(CACHE, **kw)
    if nbytes is None:
        nbytes = L.loip_k_window_prefill_q8_scratch_bytes(M, n, Hq, Hkv, d, window, sinks, max_ctx)
    return L.loip_k_window_prefill_q8(q, dtype, c["kv"], c["table"], c["max_pages"], starts, first, n, M, Hq, Hkv, d,
                                      c["page_tokens"], c["layer"], c["lpb"], window, sinks, max_ctx, scratch, nbytes,
                                      o, None)


CACHE_BAD = [dict(dtype=2), dict(dtype=-1), dict(Hkv=0), dict(Hkv=1 << 16, lpb=1 << 40), dict(d=96), dict(d=256),
             dict(d=0), dict(page_tokens=16), dict(page_tokens=0), dict(max_pages=0), dict(layer=-1), dict(kv=None),
             dict(kv=A + 8), dict(table=None), dict(table=A + 4), dict(lpb=LPB + 8), dict(lpb=LPB - 16), dict(lpb=0)]
HEADS_BAD = [dict(Hq=5), dict(Hq=0)]
WINDOW_BAD = [dict(q=None), dict(q=A + 8), dict(o=None), dict(o=A + 4), dict(window=-1), dict(sinks=-1),
              dict(max_ctx=0), dict(max_ctx=257), dict(max_ctx=(1 << 30) + 1, max_pages=1 << 25), dict(scratch=None),
              dict(scratch=A + 8), dict(nbytes=0)]
ROWS_BAD = [dict(T=-1), dict(pos=None), dict(pos=A + 2), dict(req=A + 1), dict(n_req=0)]


@pytest.mark.parametrize("call,bad", [(append, b) for b in CACHE_BAD + HEADS_BAD + ROWS_BAD + [
    dict(x=None), dict(x=A + 4), dict(q=None), dict(q=A + 8), dict(stride=511), dict(stride=508), dict(stride=514),
    dict(dtype=1, stride=516), dict(gq=A), dict(gk=A), dict(gq=A + 2, gk=A), dict(theta=0.5), dict(theta=-1.0),
    dict(theta=float("nan")), dict(theta=float("inf")), dict(eps=-1.0), dict(eps=float("nan"))]]
    + [(read, b) for b in CACHE_BAD + ROWS_BAD + [dict(o=None), dict(o=A + 8), dict(o=A + 16)]]
    + [(decode, b) for b in CACHE_BAD + HEADS_BAD + WINDOW_BAD + [dict(B=-1), dict(ctx=None), dict(ctx=A + 2)]]
    + [(prefill, b) for b in CACHE_BAD + HEADS_BAD + WINDOW_BAD + [
        dict(M=-1), dict(n=0), dict(n=-1), dict(starts=None), dict(starts=A + 2), dict(first=A + 1)]])
def test_library_refuses(L, call, bad):
    assert call(L, **bad) == loip.ERR_INVALID
    assert L.loip_last_error(None)


def test_no_rows_launch_nothing(L):
    assert append(L, T=0) == loip.OK
    assert read(L, T=0) == loip.OK
    assert decode(L, B=0) == loip.OK
    assert prefill(L, M=0) == loip.OK
    assert prefill(L, M=0, n=0) == loip.OK


def test_scratch_sizes(L):
    f, g = L.loip_k_window_attention_q8_scratch_bytes, L.loip_k_window_prefill_q8_scratch_bytes
    for a in ((0, 4, 2, 64, 8, 1, 256), (2, 4, 2, 64, 8, 1, 256)):
        assert f(*a) >= 16 and g(a[0], 1, *a[1:]) >= 16
    for bad in ((-1, 4, 2, 64, 8, 1, 256), (2, 5, 2, 64, 8, 1, 256), (2, 4, 2, 80, 8, 1, 256), (2, 4, 2, 64, -1, 1, 256),
                (2, 4, 2, 64, 8, 1, 0)):
        assert f(*bad) == 0 and g(bad[0], 1, *bad[1:]) == 0
    import random
    rng = random.Random(1)

    def draw():
        return [int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 4)), rng.choice([0, int(2 ** rng.uniform(0, 30))]),
                rng.choice([0, 1, 4, 100]), int(2 ** rng.uniform(0, 24))]

    for _ in range(3000):  # no size falls as another grows
        heads, a = rng.choice([(4, 4, 64), (32, 8, 128), (64, 8, 128), (40, 40, 128), (20, 4, 64), (9, 1, 64)]), draw()
        b = [max(x, y) for x, y in zip(a, draw())]
        assert f(a[0], *heads, *a[2:]) <= f(b[0], *heads, *b[2:]), (heads, a, b)
        assert g(a[0], a[1], *heads, *a[2:]) <= g(b[0], b[1], *heads, *b[2:]), (heads, a, b)


def test_scratch_sizes_of_the_largest_arguments(L):
    f, g = L.loip_k_window_attention_q8_scratch_bytes, L.loip_k_window_prefill_q8_scratch_bytes
    most = (1 << 31) - 1
    for heads in ((65536 - 3 * 8192 * 2, 8192, 128), (8, 1, 128), (64, 64, 64)):
        for ctx in (1, 1 << 30):
            assert f(1, *heads, most, most, ctx) <= f(most, *heads, most, most, ctx) < 1 << 30
            small, large = g(1, 1, *heads, most, most, ctx), g(1 << 30, 1 << 20, *heads, most, most, ctx)
            assert 16 <= small <= large < 3 << 30


# ---------------------------------------------------------------------------
# the binding (the library is a stand-in that records its calls, the tensors say that they are on a GPU)
# ---------------------------------------------------------------------------
HQ, HKV, D, B, PAGES = 4, 2, 64, 3, 5


class OnGpu(torch.Tensor):
    is_cuda = True
    device_index = 0

    def get_device(self):
        return self.device_index


class OnAnotherGpu(OnGpu):
    device_index = 1


def dev(x, kind=OnGpu):
    return x.as_subclass(kind)


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(loip, "lib", lambda: lib)
    loip._torch()
    monkeypatch.setattr(loip, "_of_torch", [loip._of_torch[0], lambda: 0, *loip._of_torch[2:]])  # device 0 is current
    return lib


def i32(n):
    return dev(torch.zeros(n, dtype=torch.int32))


def common():
    return dict(kv_base=dev(torch.zeros(1024, dtype=torch.uint8)),
                page_offsets=dev(torch.zeros(B, PAGES, dtype=torch.int64)), max_pages=PAGES, Hkv=HKV, d=D, page_tokens=64,
                layer=0, layer_page_bytes=LPB, stream=0)


def rows(n=B, heads=HQ, **kw):
    return dev(torch.zeros(n, heads * D, **kw))


def b_append(**bad):
    return loip.loip_k_qk_append_q8(**{**common(), **dict(
        Hq=HQ, qkv=rows(heads=HQ + 2 * HKV), g_q=None, g_k=None, eps=0.0, theta=0.0, positions=i32(B), row_req=i32(B),
        q_out=rows()), **bad})


def b_read(**bad):
    return loip.loip_k_cache_read_q8(**{**common(), **dict(positions=i32(B), row_req=i32(B), out=rows(heads=2 * HKV)),
                                        **bad})


def b_attention(**bad):
    return loip.loip_k_window_attention_q8(**{**common(), **dict(
        Hq=HQ, q=rows(), ctx_lens=i32(B), window=8, sinks=0, max_ctx=300,
        scratch=dev(torch.zeros(4096, dtype=torch.uint8)), o=rows()), **bad})


def b_prefill(**bad):
    return loip.loip_k_window_prefill_q8(**{**common(), **dict(
        Hq=HQ, q=rows(7), row_starts=i32(B + 1), first_pos=i32(B), window=8, sinks=0, max_ctx=300,
        scratch=dev(torch.zeros(4096, dtype=torch.uint8)), o=rows(7)), **bad})


OPS = [b_append, b_read, b_attention, b_prefill]


@pytest.mark.parametrize("op,good", [
    (b_append, {}), (b_append, dict(row_req=None)), (b_append, dict(kv_base=1 << 20)), (b_read, {}),
    (b_read, dict(row_req=None, out=rows(heads=2 * HKV, dtype=torch.bfloat16))), (b_attention, {}), (b_prefill, {}),
    (b_prefill, dict(first_pos=None))])
def test_what_is_in_order_reaches_the_library(library, op, good):
    op(**good)
    ((name, args),) = library.calls
    assert name == {b_append: "loip_k_qk_append_q8", b_read: "loip_k_cache_read_q8",
                    b_attention: "loip_k_window_attention_q8", b_prefill: "loip_k_window_prefill_q8"}[op]
    assert len(args) == len(loip._SIGS[name][1])


@pytest.mark.parametrize("op", OPS)
def test_tensors_of_another_device(library, op):
    name = {b_append: "qkv", b_read: "out", b_attention: "q", b_prefill: "q"}[op]
    heads = {b_append: HQ + 2 * HKV, b_read: 2 * HKV}.get(op, HQ)
    with pytest.raises(loip.LoipError, match="device 1"):
        op(**{name: dev(torch.zeros(7 if op is b_prefill else B, heads * D), OnAnotherGpu)})
    assert not library.calls


@pytest.mark.parametrize("op", OPS)
def test_a_cache_in_host_memory(library, op):
    class Pinned(torch.Tensor):
        def is_pinned(self):
            return True

    with pytest.raises(loip.LoipError, match="device memory"):
        op(kv_base=torch.zeros(1024, dtype=torch.uint8).as_subclass(Pinned))
    assert not library.calls


@pytest.mark.parametrize("op,bad", [
    (b_read, dict(out=torch.zeros(B, 2 * HKV * D))), (b_read, dict(out=rows(heads=HKV))),
    (b_read, dict(out=dev(torch.zeros(B, 4 * HKV * D))[:, ::2])), (b_read, dict(out=rows(heads=2 * HKV, dtype=torch.float16))),
    (b_read, dict(positions=i32(B - 1))), (b_read, dict(positions=dev(torch.zeros(B, dtype=torch.int64)))),
    (b_read, dict(row_req=i32(B - 1))), (b_read, dict(page_offsets=dev(torch.zeros(B, PAGES, dtype=torch.int32)))),
    (b_read, dict(kv_base=torch.zeros(1024))), (b_append, dict(q_out=rows(dtype=torch.bfloat16))),
    (b_append, dict(positions=i32(B - 1))), (b_append, dict(kv_base=dev(torch.zeros(2048))[::2])),
    (b_attention, dict(ctx_lens=i32(B - 1))), (b_attention, dict(o=rows(B - 1))),
    (b_attention, dict(scratch=torch.zeros(4096, dtype=torch.uint8))), (b_prefill, dict(first_pos=i32(B - 1))),
    (b_prefill, dict(row_starts=dev(torch.zeros(B + 1, dtype=torch.int64))))])
def test_buffers_that_do_not_fit(library, op, bad):
    with pytest.raises(loip.LoipError) as e:
        op(**bad)
    assert e.value.code == loip.ERR_INVALID and not library.calls


def test_arguments_are_those_of_the_bf16_calls():
    for name in ("loip_k_qk_append", "loip_k_window_attention", "loip_k_window_attention_scratch_bytes",
                 "loip_k_window_prefill", "loip_k_window_prefill_scratch_bytes"):
        other = name.replace("_scratch_bytes", "") + "_q8" + ("_scratch_bytes" if name.endswith("_scratch_bytes") else "")
        assert loip._SIGS[name] == loip._SIGS[other]
    assert loip.loip_k_cache_q8_layer_bytes(8, 128) == 8 * 132 * 128


def test_entries_without_ctypes(L):
    """The extension module's functions take what the ctypes ones take, and no other number of arguments."""
    import ctypes as C

    from paper_2512_21835_gb300 import _calls
    names = [n for n in dir(_calls) if n.startswith("loip_k_")]
    assert len(names) == 7
    for name in names:
        sig = loip._SIGS[name][1]
        assert getattr(L, name) is getattr(_calls, name)
        zero = [0.0 if t is C.c_float else None if t is C.c_void_p else 0 for t in sig]
        assert getattr(L, name)(*zero) == loip.ERR_INVALID and L.loip_last_error(None)
        assert getattr(L, name)(*[C.c_void_p() if t is C.c_void_p else z for t, z in zip(sig, zero)]) == loip.ERR_INVALID
        for wrong in (zero[1:], zero + [0]):
            with pytest.raises(TypeError, match=f"takes {len(sig)} arguments"):
                getattr(L, name)(*wrong)
        for i, t in enumerate(sig):
            for bad, error in (("x", (TypeError, AttributeError)), (1 << 70, OverflowError)):
                if t is C.c_float and bad != "x":
                    continue
                with pytest.raises(error):
                    getattr(L, name)(*zero[:i], bad, *zero[i + 1:])
