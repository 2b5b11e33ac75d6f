"""Sizes of the windowed attentions' scratch: a scratch for the largest call of a program
serves every smaller one (host only)."""
import random

import pytest

from paper_2512_21835_gb300 import loip


@pytest.fixture(scope="module")
def sizes():
    from paper_2512_21835_gb300 import build
    build.build()
    return loip.loip_k_window_attention_scratch_bytes, loip.loip_k_window_prefill_scratch_bytes


HEADS = [(4, 4, 64), (32, 8, 128), (64, 8, 128), (40, 40, 128), (20, 4, 64), (9, 1, 64)]
VISIBLE = [(1 << 30, 0), (4096, 64), (1024, 4), (0, 5), (1, 0)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", VISIBLE)
def test_a_draining_batch(sizes, heads, window, sinks):
    """A batch that drains from 200 requests, at contexts short and long."""
    for max_ctx in (64, 300, 4352, 131072):
        need = [sizes[0](B, *heads, window, sinks, max_ctx) for B in range(201)]
        assert need == sorted(need), max_ctx


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", VISIBLE)
def test_the_last_chunk_of_a_prompt(sizes, heads, window, sinks):
    """A chunk of fewer rows than the others."""
    for n in (1, 3):
        for max_ctx in (64, 300, 4352, 131072):
            need = [sizes[1](M, n, *heads, window, sinks, max_ctx) for M in [*range(300), 512, 1000, 2048, 8192]]
            assert need == sorted(need), (n, max_ctx)


def test_no_size_falls_as_another_grows(sizes):
    rng = random.Random(1)

    def draw():
        return [int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 4)), rng.choice([0, int(2 ** rng.uniform(0, 30))]),
                rng.choice([0, 1, 4, 100]), int(2 ** rng.uniform(0, 24))]

    for _ in range(4000):
        heads, a = rng.choice(HEADS), draw()
        b = [max(x, y) for x, y in zip(a, draw())]
        for (M, n, *rest), (M2, n2, *rest2) in ((a, b),):
            assert sizes[0](M, *heads, *rest) <= sizes[0](M2, *heads, *rest2), (heads, a, b)
            assert sizes[1](M, n, *heads, *rest) <= sizes[1](M2, n2, *heads, *rest2), (heads, a, b)


def test_a_scratch_is_small(sizes):
    """What the parts of one wave take, for calls within the card's reach."""
    assert sizes[0](8, 64, 8, 128, 1024, 4, 4352) <= 4 << 20
    assert sizes[0](64, 64, 8, 128, 4096, 64, 32768) <= 8 << 20
    assert sizes[1](8192, 1, 32, 8, 128, 4096, 4, 16384) <= 16 << 20
