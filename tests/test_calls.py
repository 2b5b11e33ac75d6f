"""What the extension module of the windowed-serving entries does with arguments that do not convert, and what the
binding makes of it (host only)."""
import ctypes as C

import numpy as np
import pytest

from paper_2512_21835_gb300 import loip

NAMES = [n + s for s in ("", "_q8") for n in ("loip_k_qk_append", "loip_k_window_attention", "loip_k_window_prefill")]
NAMES.append("loip_k_cache_read_q8")


@pytest.fixture(scope="module")
def calls():
    from paper_2512_21835_gb300 import build
    build.build()
    loip.lib()
    return pytest.importorskip("paper_2512_21835_gb300._calls")


def zeros(name):
    return [0.0 if t is C.c_float else None if t is C.c_void_p else 0 for t in loip._SIGS[name][1]]


@pytest.mark.parametrize("number", [np.int64, np.uint64, np.int32, bool])
@pytest.mark.parametrize("name", NAMES)
def test_whole_numbers_of_other_types(calls, name, number):
    """Numbers that are not Python's own (a size that numpy has worked out), as ctypes takes them."""
    args = [0.0 if t is C.c_float else None if t is C.c_void_p else number(0) for t in loip._SIGS[name][1]]
    assert getattr(calls, name)(*args) == loip.ERR_INVALID


class Number:
    """A whole number and a float that say when they are looked at."""

    def __init__(self, seen, error=None):
        self.seen, self.error = seen, error

    def __index__(self):
        self.seen.append(self)
        if self.error:
            raise self.error
        return 0

    def __float__(self):
        return float(self.__index__())


@pytest.mark.parametrize("name", NAMES)
def test_nothing_is_converted_behind_an_error(calls, name):
    sig = loip._SIGS[name][1]
    numbers = [i for i, t in enumerate(sig) if t is not C.c_void_p]
    for first in numbers:
        seen, args = [], zeros(name)
        for i in numbers:
            args[i] = Number(seen, ZeroDivisionError(f"argument {i}") if i >= first else None)
        with pytest.raises(ZeroDivisionError, match=f"argument {first}$"):
            getattr(calls, name)(*args)
        assert len(seen) == numbers.index(first) + 1


class Overflowing:
    """A library whose entries find a number that does not fit."""

    def __getattr__(self, name):
        def entry(*a):
            raise OverflowError("an argument does not fit into 32 bits")
        return entry


def test_numbers_past_their_type_are_refusals(monkeypatch):
    """The binding's error is that of every other refusal."""
    import test_q8_refusals as R
    import test_window_binding as W
    loip._torch()
    monkeypatch.setattr(loip, "_of_torch", [loip._of_torch[0], lambda: 0, *loip._of_torch[2:]])  # device 0 is current
    monkeypatch.setattr(loip, "lib", lambda: Overflowing())
    for call in (W.append, W.attention, W.prefill, R.b_append, R.b_read, R.b_attention, R.b_prefill):
        with pytest.raises(loip.LoipError, match="32 bits") as e:
            call()
        assert e.value.code == loip.ERR_INVALID


@pytest.mark.parametrize("number", [1 << 31, -(1 << 31) - 1, 1 << 32, 1 << 70])
@pytest.mark.parametrize("name", NAMES)
def test_numbers_past_their_type(calls, name, number):
    """Not cut off to another number, which the library may accept."""
    sig = loip._SIGS[name][1]
    for i, t in enumerate(sig):
        if t is C.c_int32 or (t is C.c_uint64 and number < 0):
            with pytest.raises(OverflowError):
                getattr(calls, name)(*zeros(name)[:i], number, *zeros(name)[i + 1:])


def pointers(name):
    return [i for i, t in enumerate(loip._SIGS[name][1]) if t is C.c_void_p]


@pytest.mark.parametrize("name", NAMES)
def test_addresses_of_every_kind(calls, name):
    """What ctypes takes as an address: arrays, pointers and references are theirs; the number in an int object is none."""
    number, array = C.c_int(64), (C.c_int * 4)()
    for i in pointers(name):
        for good in (C.c_void_p(64), C.c_void_p(), array, C.pointer(number), C.byref(number), True):
            args = zeros(name)
            args[i] = good
            assert getattr(calls, name)(*args) == loip.ERR_INVALID
        for bad in (number, C.c_uint64(64), C.c_float(1), 1.0, np.float64(1), np.int64(64), "x", b"x", object()):
            args = zeros(name)
            args[i] = bad
            with pytest.raises((TypeError, C.ArgumentError)):
                getattr(calls, name)(*args)


def test_an_address_is_the_objects_own(calls):
    """The check of alignment sees the address that ctypes would pass."""
    raw = C.create_string_buffer(64)
    at = C.addressof(raw)
    at16, odd = at + -at % 16, at + -at % 16 + 4
    name = "loip_k_cache_read_q8"  # kv_base and page_offsets come first; the shape is right, T is 0
    def read(kv, table=16):
        return getattr(calls, name)(kv, table, 1, None, None, 1, 0, 1, 64, 64, 0, 132 * 64, None, 0, None)
    for make in (C.c_void_p, lambda a: (C.c_int * 4).from_address(a), lambda a: C.pointer(C.c_int.from_address(a)),
                 lambda a: C.byref(C.c_int.from_address(a)), int):
        assert read(make(at16)) == loip.OK
        assert read(make(odd)) == loip.ERR_INVALID
        assert read(make(at16), make(odd)) == loip.ERR_INVALID
