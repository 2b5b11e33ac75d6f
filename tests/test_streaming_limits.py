"""What windowed generation refuses (host only: the passes over the layers are stand-ins)."""
from types import SimpleNamespace

import pytest

from paper_2512_21835_gb300.streaming import PAGE, PagePool, WindowedDecoder, pages_of_a_request


class Decoder(WindowedDecoder):
    """Bookkeeping alone: a pass records its rows."""

    def __init__(self, batch, max_ctx, chunk=256, window=100, sinks=4, vocab=50):
        self.m = dict(vocab=vocab)
        self.window, self.sinks, self.max_ctx, self.chunk = window, sinks, max_ctx, chunk
        self.pool = PagePool(1000, batch, max_ctx, 4096)
        self.pos, self.passes = [0] * batch, []
        self.L = SimpleNamespace(loip_k_attention_tc_status=lambda: 0)

    def _rows(self, tokens, rows, single):
        self.passes.append((list(tokens), rows))
        return [None] * len(rows)

    def _head(self, x):
        return x


@pytest.mark.parametrize("max_ctx", [1000, 1024, 65, 1])
def test_no_position_reaches_the_end_of_the_context(max_ctx):
    """The last page may have room past max_ctx; positions there would be appended and never read."""
    d = Decoder(2, max_ctx)
    d.prefill(0, [1] * max_ctx)
    with pytest.raises(ValueError):
        d.prefill(0, [1])
    if max_ctx > 1:
        d.prefill(1, [1] * (max_ctx - 1))
        with pytest.raises(ValueError):
            d.prefill(1, [1, 1])
    n = len(d.passes)
    with pytest.raises(ValueError):
        d.step([1, 1])
    assert len(d.passes) == n and d.pos == [max_ctx, max(max_ctx - 1, 0)]
    assert max(p for _, rows in d.passes for _, p in rows) == max_ctx - 1


def test_a_prompt_too_long_takes_no_pass():
    d = Decoder(1, 1000, chunk=64)
    with pytest.raises(ValueError):
        d.prefill(0, [1] * 1001)
    assert not d.passes and d.pos == [0] and not d.pool.held[0]


def test_the_pool_refuses_positions_past_the_context():
    pool = PagePool(100, 1, 1000, 4096)
    pool.extend(0, 0, 999)
    with pytest.raises(ValueError):
        pool.extend(0, 1000, 1000)
    assert len(pool.held[0]) == -(-1000 // PAGE)


@pytest.mark.parametrize("tokens", [[], [1], [1, 1, 1], [1, 50], [-1, 1]])
def test_steps_take_a_token_of_the_vocabulary_for_each_request(tokens):
    """More tokens than rows, or a token outside the table, would be read and written out of range."""
    d = Decoder(2, 1000)
    d.prefill(0, [1, 2])
    n = len(d.passes)
    with pytest.raises(ValueError):
        d.step(tokens)
    assert len(d.passes) == n and d.pos == [2, 0]
    d.step([0, 49])
    assert d.pos == [3, 1]


@pytest.mark.parametrize("request_, prompt", [(0, []), (0, [50]), (0, [3, -1]), (2, [1]), (-1, [1])])
def test_prompts_are_of_the_vocabulary_and_of_a_request(request_, prompt):
    d = Decoder(2, 1000)
    with pytest.raises(ValueError):
        d.prefill(request_, prompt)
    assert not d.passes and d.pos == [0, 0]


@pytest.mark.parametrize("window,sinks,max_ctx,chunk", [(1 << 20, 0, 1000, 256), (1 << 30, 1 << 30, 128, 64), (100, 4, 420, 70),
                                                        (64, 0, 3000, 1), (130, 70, 5000, 256), (1, 0, 64, 1), (0, 0, 65, 32)])
def test_pages_of_a_request(window, sinks, max_ctx, chunk):
    """Enough for a whole context taken in chunks, then token by token; never more than the context has."""
    n = pages_of_a_request(window, sinks, max_ctx, chunk)
    assert 1 <= n <= -(-max_ctx // PAGE)
    for prompt in {0, max_ctx // 3, max_ctx}:
        d = Decoder(1, max_ctx, chunk, window, sinks)
        d.pool = PagePool(n, 1, max_ctx, 4096)
        if prompt:
            d.prefill(0, [1] * prompt)
        for _ in range(max_ctx - prompt):
            d.step([1])
        assert d.pool.most <= n


@pytest.mark.parametrize("code", [6, -1])
def test_a_prompt_whose_attention_gave_up_is_an_error(code):
    d = Decoder(1, 1000)
    d.L.loip_k_attention_tc_status = lambda: code
    with pytest.raises(RuntimeError, match="gave up"):
        d.prefill(0, [1] * 40)
