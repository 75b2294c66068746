"""The bookkeeping of runner.PagedCache on the CPU: the library's calls are replaced by ones that note what they were given, or refuse it."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import PagedCache

D, HKV, PAGE, PAGES, MOST = 128, 2, 16, 12, 6


class Calls:
    """Stands for the library: notes (call, T, seq_start, pos, pages in the table), and refuses the call named in `refuse`."""

    def __init__(self, monkeypatch):
        self.seen, self.refuse = [], None

        def alloc_cache(p, pages, page_size, max_pages, fp8, device):
            c = B.l2a_cache(page_size=page_size, pages=pages, max_pages=max_pages)
            c.tensors = (None, None, None, None, torch.full((p.B, max_pages), -1, dtype=torch.int32))
            return c

        def call(name):
            def f(p, c, *args, **kw):
                if name == self.refuse:
                    raise ValueError(name)
                start, pos = (args[2], args[3]) if name == "write" else (args[1], args[2]) if name == "extend" else (args[0], args[1])
                self.seen.append((name, p.T, start.tolist(), pos.tolist(), c.tensors[4].clone().numpy()))
            return f
        monkeypatch.setattr(B, "alloc_cache", alloc_cache)
        monkeypatch.setattr(B, "l2a_cache_write", call("write"))
        monkeypatch.setattr(B, "l2a_attn_extend", call("extend"))
        monkeypatch.setattr(B, "l2a_cache_read", call("read"))


@pytest.fixture
def calls(monkeypatch):
    return Calls(monkeypatch)


def make(sequences=2):
    return PagedCache(B.make_params(sequences, 1, 4, HKV, D, 30), PAGES, PAGE, MOST, device="cpu")


def step(cache, new):
    n = int(np.sum(np.asarray(new)))
    kv = torch.zeros(n, HKV, D, dtype=torch.bfloat16)
    return cache.extend(new, torch.zeros(n, 4, D, dtype=torch.bfloat16), kv, kv, torch.zeros(1, n, dtype=torch.uint8))


def held(cache):
    """What the bookkeeping says, after a look at whether it agrees with itself."""
    used = -(-cache.length // PAGE)
    for b, n in enumerate(used):
        assert (cache.table[b, :n] >= 0).all() and (cache.table[b, n:] == -1).all()
    assert sorted(list(cache.free) + cache.table[cache.table >= 0].tolist()) == list(range(PAGES))
    return cache.length.tolist(), cache.table.copy(), list(cache.free)


@pytest.mark.parametrize("refused", ["write", "extend"])
def test_a_refused_step_leaves_everything_as_it_was(calls, refused):
    cache = make()
    step(cache, [20, 3])
    before = held(cache)
    calls.refuse = refused
    with pytest.raises(ValueError, match=refused):
        step(cache, [40, 14])  # pages would have been handed out
    after = held(cache)
    assert after[0] == before[0] == [20, 3] and np.array_equal(after[1], before[1]) and after[2] == before[2]
    calls.refuse, calls.seen = None, []
    step(cache, [2, 1])
    assert [x[:4] for x in calls.seen] == [(name, 3, [0, 2, 3], [20, 3]) for name in ("write", "extend")]
    assert held(cache)[0] == [22, 4]


def test_a_step_without_room_leaves_everything_as_it_was(calls):
    cache = make()
    step(cache, [20, 3])
    before = held(cache)
    for new in ([80, 0], [70, 94], [-1, 2]):
        with pytest.raises(ValueError, match="no room"):
            step(cache, new)
        after = held(cache)
        assert after[0] == before[0] and np.array_equal(after[1], before[1]) and after[2] == before[2]


def test_steps_pages_and_ends(calls):
    cache = make()
    step(cache, [20, 0])
    step(cache, [1, 33])
    assert held(cache)[0] == [21, 33] and len(cache.free) == PAGES - 5
    assert [x[1:4] for x in calls.seen[::2]] == [(20, [0, 20, 20], [0, 0]), (34, [0, 1, 34], [20, 0])]
    assert np.array_equal(calls.seen[-1][4], cache.table)
    cache.end(0)
    assert held(cache)[0] == [0, 33] and len(cache.free) == PAGES - 3
    step(cache, [6 * PAGE, 2])
    assert held(cache)[0] == [96, 35]


@pytest.mark.parametrize("new", [[2], [1, 1, 1], 2, [[1, 1]], []])
def test_a_number_of_tokens_for_every_sequence(calls, new):
    """(a list of one entry would stand for all of them)"""
    cache = make()
    step(cache, [20, 3])
    before = held(cache)
    with pytest.raises(ValueError, match="each of the 2 sequences"):
        cache.begin_step(new)
    after = held(cache)
    assert after[0] == before[0] and np.array_equal(after[1], before[1]) and len(calls.seen) == 2


def test_a_step_without_new_tokens(calls):
    """(the library refuses a call of no tokens)"""
    cache = make()
    for _ in range(2):
        before = held(cache)
        assert step(cache, [0, 0]).shape == (0, 4, D)
        after = held(cache)
        assert after[0] == before[0] and np.array_equal(after[1], before[1])
        step(cache, [5, 0])
    assert [x[1] for x in calls.seen] == [5, 5, 5, 5]
    before = held(cache)
    for rows in ((1, 0, 0), (0, 1, 0), (0, 0, 1)):
        q, k, v = (torch.zeros(n, h, D, dtype=torch.bfloat16) for n, h in zip(rows, (4, HKV, HKV)))
        with pytest.raises(ValueError, match="no new tokens"):
            cache.extend([0, 0], q, k, v, None)
    assert held(cache)[0] == before[0]


@pytest.mark.parametrize("new", [[2 ** 31 - 1, 0], [2 ** 31 - 16, 2 ** 31 - 16], [2 ** 40, 0], [2 ** 63 - 1, 1], [-2 ** 31, 2 ** 31 - 1]])
def test_lengths_that_pass_32_bits(calls, new):
    cache = make()
    step(cache, [20, 3])
    before = held(cache)
    with pytest.raises(ValueError, match="no room"):
        cache.begin_step(new)
    after = held(cache)
    assert after[0] == before[0] and np.array_equal(after[1], before[1]) and after[2] == before[2]


def test_lengths_that_are_no_whole_numbers(calls):
    cache = make()
    for new in ([1.5, 1], [float("nan"), 1], [float("inf"), 1], ["a", 1], [None, 1]):
        with pytest.raises(ValueError, match="whole numbers"):
            cache.begin_step(new)
    for new in ([1, 2], [1.0, 2.0], (1, 2), np.array([1, 2], np.uint8), torch.tensor([1, 2])):
        step(cache, new)
    assert held(cache)[0] == [5, 10]


def test_sequences_that_there_are_none_of(calls):
    cache = make()
    step(cache, [20, 3])
    before = held(cache)
    for b in (-3, 2, 100):
        with pytest.raises(IndexError):
            cache.read(b)
        with pytest.raises(IndexError):
            cache.end(b)
    assert held(cache)[0] == before[0] and len(calls.seen) == 2
    for b in (1, -1):  # (the last sequence's length came with no sequence's rows)
        k, v = cache.read(b)
        assert k.shape == v.shape == (3, HKV, D) and calls.seen[-1][:4] == ("read", 3, [0, 0, 3], [0, 0])
    cache.end(-1)
    assert held(cache)[0] == [20, 0]


def test_the_params_given_stay_as_they_are(calls):
    p = B.make_params(2, 77, 4, HKV, D, 30, flags=B.L2A_FLAG_DENSE)
    caches = [PagedCache(p, PAGES, PAGE, MOST, device="cpu") for _ in range(2)]
    for cache in caches:  # (layers of one model)
        step(cache, [20, 3])
        cache.read(0)
    assert p.T == 77 and [x[1] for x in calls.seen] == [23, 23, 20] * 2
    assert all(c.p.flags == B.L2A_FLAG_DENSE and c.p.W == 30 for c in caches)


def test_steps_cannot_be_captured(calls, monkeypatch):
    """Indices come from the host's memory: a graph would repeat the step it was captured in."""
    cache = make()
    step(cache, [20, 3])
    before = held(cache)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for call in (lambda: cache.begin_step([1, 1]), lambda: step(cache, [1, 1]), lambda: cache.read(0)):
        with pytest.raises(RuntimeError, match="captured"):
            call()
    after = held(cache)
    assert after[0] == before[0] and np.array_equal(after[1], before[1]) and len(calls.seen) == 2
