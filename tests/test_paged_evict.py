"""The bookkeeping around evictions in runner.PagedCache on the CPU: the library's calls are replaced by ones that note what they were given."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import PagedCache
from tests.test_paged_cache import HKV, MOST, PAGE, PAGES, Calls, D, held, step

W = 30


@pytest.fixture
def calls(monkeypatch):
    c = Calls(monkeypatch)
    c.weights, c.evictions = [], []
    monkeypatch.setattr(B, "l2a_cache_weights", lambda p, cache, q, start, pos, lse, most, decay, old, new: c.weights.append((lse.shape, most, decay, old is new)))

    def evict(p, cache, rows, keep, most, old, new):
        if c.refuse == "evict":
            raise ValueError("evict")
        c.evictions.append((rows.tolist(), keep.tolist(), most, cache.tensors[4].clone().numpy()))
    monkeypatch.setattr(B, "l2a_cache_evict", evict)
    return c


def make(sequences=2, flags=0, decay=0.5):
    return PagedCache(B.make_params(sequences, 1, 4, HKV, D, W, flags=flags), PAGES, PAGE, MOST, device="cpu", decay=decay)


def test_weights_follow_every_step(calls):
    cache = make()
    step(cache, [5, 0])
    step(cache, [1, 40])
    assert calls.weights == [((4, 5), 5, 0.5, True), ((4, 41), 40, 0.5, True)]
    step(make(decay=None), [5, 0])
    assert len(calls.weights) == 2


@pytest.mark.parametrize("lengths,limit,rows,keep", [
    ([96, 10], 64, [64, 0], [32, 0]),      # 96 - 30 rows may go: four pages; 32 behind them leave room for two
    ([96, 96], [96, 50], [0, 64], [0, 16]),
    ([95, 33], 0, [64, 0], [0, 0]),        # as far as it goes
    ([80, 81], 79, [48, 48], [32, 32]),
    ([29, 30], 5, [0, 0], [0, 0])])        # all in the window
def test_which_rows_go(calls, lengths, limit, rows, keep):
    cache = make()
    step(cache, lengths)
    tables, free = cache.table.copy(), list(cache.free)
    gone = cache.evict(limit)
    assert gone.tolist() == [r - k for r, k in zip(rows, keep)]
    if any(gone):
        assert calls.evictions[0][:3] == (rows, keep, max(rows)) and np.array_equal(calls.evictions[0][3], tables)
    else:
        assert not calls.evictions
    for b in range(2):
        kept = [x for i, x in enumerate(tables[b].tolist()) if not keep[b] // PAGE <= i < rows[b] // PAGE]
        assert cache.table[b].tolist() == kept + [-1] * (MOST - len(kept))
    assert cache.length.tolist() == [n - g for n, g in zip(lengths, gone)] and len(cache.free) == len(free) + sum(gone) // PAGE
    held(cache)
    assert np.array_equal(cache.cache.tensors[4].numpy(), cache.table)  # on the GPU, too
    # positions go on, and what was freed is handed out again
    more = [2 if cache.length[0] + 2 <= MOST * PAGE else 0, 1]  # (a table may be full)
    assert cache.positions(more).tolist() == [[lengths[0], lengths[0] + 1][:more[0]] + [lengths[1]]]
    step(cache, more)
    held(cache)
    cache.end(0)
    assert cache.positions([1, 0]).tolist() == [[0]]


def test_a_sequence_longer_than_its_table(calls):
    """Positions beyond the rows that the table holds, in a cache that stays within its bound."""
    cache = make(1)
    for i in range(300):
        assert cache.positions([1]).tolist() == [[i]]
        step(cache, [1])
        cache.evict(64)
        held(cache)
    assert int(cache.length[0]) <= 64 and int(cache.length[0] + cache.evicted[0]) == 300


def test_what_is_refused_changes_nothing(calls):
    cache = make()
    step(cache, [96, 90])
    before, evicted = held(cache), cache.evicted.copy()
    calls.refuse = "evict"
    for call in (lambda: cache.evict(40), lambda: cache.evict(-1), lambda: cache.evict([1, 2, 3]), lambda: cache.evict(40, recent=W - 1), lambda: cache.evict(40, recent=-1),
                 lambda: cache.positions([1]), lambda: cache.positions([1, -1]), lambda: cache.positions([0.5, 0])):
        with pytest.raises(ValueError):
            call()
        after = held(cache)
        assert after[0] == before[0] and np.array_equal(after[1], before[1]) and after[2] == before[2] and np.array_equal(cache.evicted, evicted)
    with pytest.raises(ValueError, match="no attention weights"):
        make(decay=None).evict(40)
    for decay in (-0.5, float("nan"), float("inf")):
        with pytest.raises(ValueError, match="fade"):
            make(decay=decay)


def test_without_windows_all_rows_may_go(calls):
    cache = make(flags=B.L2A_FLAG_SKIP_LOCAL)
    step(cache, [96, 40])
    assert cache.evict(0, recent=0).tolist() == [96, 32]
    assert cache.length.tolist() == [0, 8]
    held(cache)
