"""Page bookkeeping of windowed generation (host only): which pages a request holds,
and that no page a later query sees is ever given back."""
import random

import pytest

from paper_2512_21835_gb300.streaming import PAGE, PagePool
from window_ref import seen_positions


@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 0), (65, 1), (100, 70), (256, 4), (10 ** 6, 0)])
def test_held_pages_cover_what_is_seen(window, sinks):
    rng = random.Random(window)
    pool = PagePool(100, 2, 3000, 4096)
    pos = [0, 0]
    while max(pos) < 2500:
        r, n = rng.randrange(2), rng.choice([1, 1, 1, 7, 64, 130])
        pool.extend(r, pos[r], pos[r] + n - 1)
        rows = range(pos[r], pos[r] + n)
        need = {j // PAGE for j in seen_positions(rows, window, sinks)}
        assert need <= set(pool.held[r])
        assert all(pool.table[r, i] == p * pool.page_bytes for i, p in pool.held[r].items())
        pos[r] += n
        pool.retire(r, pos[r], window, sinks)
        later = {j // PAGE for j in seen_positions(range(pos[r], pos[r] + 1), window, sinks) if j < pos[r]}
        assert later <= set(pool.held[r])
        pages = [p for h in pool.held for p in h.values()] + pool.free
        assert sorted(pages) == list(range(100))  # none lost, none held twice


def test_a_window_bounds_the_pool():
    pool = PagePool(6, 1, 100000, 4096)  # sinks 1 page, window 256: at most 5 pages, and one in the making
    for p in range(5000):
        pool.extend(0, p, p)
        pool.retire(0, p + 1, 256, 4)
    assert pool.most <= 6
    with pytest.raises(MemoryError):
        PagePool(2, 1, 1000, 4096).extend(0, 0, 3 * PAGE)
