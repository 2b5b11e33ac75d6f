"""Tensors of another device than the call's are refused by the 8-bit cache's operators before anything
reaches the library (host only: see test_q8_refusals.py for the stand-ins)."""
import pytest

from test_q8_refusals import (B, D, HKV, HQ, PAGES, OnAnotherGpu, b_append, b_attention, b_prefill, b_read, dev,
                              library, loip, torch)  # noqa: F401 (library is a fixture)


def away(*shape, dtype=torch.float32):
    return dev(torch.zeros(*shape, dtype=dtype), OnAnotherGpu)


I32, U8, BF16 = torch.int32, torch.uint8, torch.bfloat16
EVERY = dict(kv_base=away(1024, dtype=U8), page_offsets=away(B, PAGES, dtype=torch.int64))
OTHERS = {b_append: dict(EVERY, positions=away(B, dtype=I32), row_req=away(B, dtype=I32), q_out=away(B, HQ * D),
                         g_q=away(D, dtype=BF16)),
          b_read: dict(EVERY, positions=away(B, dtype=I32), row_req=away(B, dtype=I32)),
          b_attention: dict(EVERY, ctx_lens=away(B, dtype=I32), scratch=away(4096, dtype=U8), o=away(B, HQ * D)),
          b_prefill: dict(EVERY, row_starts=away(B + 1, dtype=I32), first_pos=away(B, dtype=I32),
                          scratch=away(4096, dtype=U8), o=away(7, HQ * D))}


@pytest.mark.parametrize("op,name", [(op, name) for op, names in OTHERS.items() for name in names])
def test_every_tensor_is_of_the_current_device(library, op, name):  # noqa: F811
    more = dict(g_k=dev(torch.zeros(D, dtype=BF16))) if name == "g_q" else {}
    with pytest.raises(loip.LoipError, match="device 1") as e:
        op(**{name: OTHERS[op][name]}, **more)
    assert e.value.code == loip.ERR_INVALID and not library.calls


class Foreign:
    """An array of another library on the GPU: no tensor, whatever else it has."""
    dtype, shape, device, is_cuda = "int32", (B,), "cuda:1", True


@pytest.mark.parametrize("op,name", [(op, name) for op, names in OTHERS.items() for name in names
                                     if name in ("positions", "row_req", "ctx_lens", "first_pos", "page_offsets")])
def test_what_is_no_tensor_is_refused_by_its_own_check(library, op, name):  # noqa: F811
    with pytest.raises(loip.LoipError) as e:
        op(**{name: Foreign()})
    assert e.value.code == loip.ERR_INVALID and not library.calls
