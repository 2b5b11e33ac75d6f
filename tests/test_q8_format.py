"""The 8-bit cache's format, as the tests' reference has it: what a block stands for."""
import numpy as np
import pytest

import q8_ref as Q


def blocks(*rows):
    x = np.zeros((len(rows), 32))
    for i, r in enumerate(rows):
        x[i, :len(r)] = r
    return x


def test_every_value_is_a_bf16_number_off_by_half_a_step():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((400, 64)) * 2.0 ** rng.integers(-120, 120, (400, 1))).astype(np.float32)
    c, e = Q.encode(x)
    y = Q.decode(c, e)
    assert np.all(y.astype(np.float32).view(np.uint32) & 0xffff == 0)
    step = np.repeat(2.0 ** (e.astype(np.float64) - 133), 32, -1)
    assert np.all(np.abs(y - x) <= step / 2)
    m = (c & 127).reshape(400, 2, 32).max(-1)
    assert np.all((m >= 64) | (e == 8)) and m.max() == 127
    again = Q.encode(y)
    assert np.array_equal(again[0], c & np.where(c == 128, 0, 255).astype(np.uint8)) and np.array_equal(again[1], e)


@pytest.mark.parametrize("most,E,m", [
    (127.0, 133, 127), (127.5, 134, 64), (127.49, 133, 127), (128.0, 134, 64), (64.0, 133, 64), (63.75, 133, 64),
    (0.0, 8, 0), (2.0 ** -125, 8, 1), (2.0 ** -126, 8, 0), (2.0 ** -119, 8, 64), (127 * 2.0 ** -125, 8, 127),
    (127.5 * 2.0 ** -125, 9, 64), (127 * 2.0 ** 120, 253, 127)])
def test_exponents(most, E, m):
    c, e = Q.encode(blocks([most], [-most, most / 2]))
    if most == 63.75:  # 127.5 quarters: the next exponent has it as 64
        E, m = 133, 64
    assert e.tolist() == [[E], [E]]
    assert c[0, 0] == m and (c[1, 0] & 127) == m


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan, 127.5 * 2.0 ** 120, -3e38])
def test_blocks_that_are_not_held(bad):
    c, e = Q.encode(np.concatenate([blocks([1.0, bad]), blocks([1.0])], -1))
    assert e.tolist() == [[255, 127]] and not c[0, :32].any()
    y = Q.decode(c, e)
    assert np.all(np.isnan(y[0, :32])) and y[0, 32] == 1.0


def test_slots_of_a_layer_fill_it_once():
    for Hkv, d in ((2, 64), (1, 128), (3, 128)):
        cache = Q.Cache8(1, 2, Hkv, d, 3, layers=2, layer=1)
        seen = np.zeros(len(cache.bytes), dtype=int)
        for j in range(128):
            for which in (0, 1):
                for ix in cache.slot(0, j, which):
                    np.add.at(seen, ix, 1)
        page = 2 * cache.layer_page_bytes
        want = np.zeros(len(cache.bytes), dtype=int)
        for at in cache.table[0]:
            want[at + page // 2:at + page] = 1
        assert np.array_equal(seen, want)
