"""What the binding of the windowed operators lets through to the library (host only: the
library is a stand-in that records its calls, the tensors say that they are on a GPU)."""
import pytest

from paper_2512_21835_gb300 import loip

torch = pytest.importorskip("torch")

HQ, HKV, D, B, PAGES = 4, 2, 64, 3, 5


class OnGpu(torch.Tensor):
    is_cuda = True


def dev(x):
    return x.as_subclass(OnGpu)


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(loip, "lib", lambda: lib)
    return lib


def i32(n):
    return dev(torch.zeros(n, dtype=torch.int32))


def table(rows=B, pages=PAGES):
    return dev(torch.zeros(rows, pages, dtype=torch.int64))


def common():
    return dict(kv_base=dev(torch.zeros(1024, dtype=torch.bfloat16)), page_offsets=table(), max_pages=PAGES, Hq=HQ,
                Hkv=HKV, d=D, page_tokens=64, layer=0, layer_page_bytes=65536, stream=0)


def rows(n=B, heads=HQ):
    return dev(torch.zeros(n, heads * D))


def append(**bad):
    return loip.loip_k_qk_append(**{**common(), **dict(
        qkv=rows(heads=HQ + 2 * HKV), g_q=dev(torch.zeros(D, dtype=torch.bfloat16)),
        g_k=dev(torch.zeros(D, dtype=torch.int16)), eps=0.0, theta=0.0, positions=i32(B), row_req=i32(B), q_out=rows()),
        **bad})


def attention(**bad):
    return loip.loip_k_window_attention(**{**common(), **dict(
        q=rows(), ctx_lens=i32(B), window=8, sinks=0, max_ctx=300, scratch=dev(torch.zeros(4096, dtype=torch.uint8)),
        o=rows()), **bad})


def prefill(**bad):
    return loip.loip_k_window_prefill(**{**common(), **dict(
        q=rows(7), row_starts=i32(B + 1), first_pos=i32(B), window=8, sinks=0, max_ctx=300,
        scratch=dev(torch.zeros(4096, dtype=torch.uint8)), o=rows(7)), **bad})


OPS = {"append": append, "attention": attention, "prefill": prefill}


@pytest.mark.parametrize("op,good", [
    ("append", {}), ("append", dict(g_q=None, g_k=None, row_req=None)), ("append", dict(kv_base=1 << 20)),
    ("append", dict(positions=i32(B + 4))), ("append", dict(g_q=4096, g_k=8192)),
    ("attention", {}), ("attention", dict(page_offsets=dev(torch.zeros(B * PAGES, dtype=torch.int64)))),
    ("attention", dict(page_offsets=table(B + 2))), ("attention", dict(q=rows(1), o=rows(1), page_offsets=table(1, 9))),
    ("prefill", {}), ("prefill", dict(first_pos=None))])
def test_what_is_in_order_reaches_the_library(library, op, good):
    OPS[op](**good)
    assert len(library.calls) == 1


INTS = {"append": ("positions", "row_req"), "attention": ("ctx_lens",), "prefill": ("row_starts", "first_pos")}
LENGTH = {"row_starts": B + 1}


@pytest.mark.parametrize("op,name", [(o, n) for o, names in INTS.items() for n in names])
def test_index_arrays(library, op, name):
    n = LENGTH.get(name, B)
    for bad in (dev(torch.zeros(n, dtype=torch.int64)), dev(torch.zeros(n)), dev(torch.zeros(2 * n, dtype=torch.int32))[::2],
                torch.zeros(n, dtype=torch.int32)):
        with pytest.raises(loip.LoipError, match=name) as e:
            OPS[op](**{name: bad})
        assert e.value.code == loip.ERR_INVALID
    if name != "row_starts":  # (its length says how many prompts there are)
        with pytest.raises(loip.LoipError, match=name):
            OPS[op](**{name: i32(n - 1)})
    assert not library.calls


@pytest.mark.parametrize("op", sorted(OPS))
@pytest.mark.parametrize("bad", [
    dev(torch.zeros(B, 2 * PAGES, dtype=torch.int32)),           # as many bytes, half as wide
    dev(torch.zeros(B, PAGES)), table(pages=PAGES + 3),          # rows wider than max_pages
    table(pages=PAGES + 3)[:, :PAGES], table(PAGES, B).t(),      # strided views
    table(pages=PAGES - 1), torch.zeros(B, PAGES, dtype=torch.int64)])
def test_page_tables(library, op, bad):
    with pytest.raises(loip.LoipError, match="page table"):
        OPS[op](page_offsets=bad)
    assert not library.calls


@pytest.mark.parametrize("bad", [dev(torch.zeros(D)), dev(torch.zeros(D, dtype=torch.float16)),
                                 dev(torch.zeros(D - 8, dtype=torch.bfloat16)),
                                 dev(torch.zeros(2 * D, dtype=torch.bfloat16))[::2], torch.zeros(D, dtype=torch.bfloat16)])
def test_gains(library, bad):
    for name in ("g_q", "g_k"):
        with pytest.raises(loip.LoipError, match="gain"):
            append(**{name: bad})
    assert not library.calls


@pytest.mark.parametrize("op,bad", [
    ("append", dict(q_out=torch.zeros(B, HQ * D))), ("append", dict(qkv=torch.zeros(B, (HQ + 2 * HKV) * D))),
    ("append", dict(kv_base=torch.zeros(1024))), ("attention", dict(kv_base=dev(torch.zeros(2048))[::2])),
    ("attention", dict(q=torch.zeros(B, HQ * D))), ("attention", dict(o=torch.zeros(B, HQ * D))),
    ("attention", dict(scratch=torch.zeros(4096, dtype=torch.uint8))),
    ("prefill", dict(scratch=dev(torch.zeros(8192, dtype=torch.uint8))[::2])),
    ("prefill", dict(kv_base=torch.zeros(1024).numpy()))])
def test_buffers_that_the_device_cannot_use(library, op, bad):
    with pytest.raises(loip.LoipError) as e:
        OPS[op](**bad)
    assert e.value.code == loip.ERR_INVALID and not library.calls
