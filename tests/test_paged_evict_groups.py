"""PagedCache.evict in several calls, and what it leaves of the cache's params: on the CPU with calls that note what they were given, and on the GPU in one call and in several."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd import runner
from paper_2603_17484_amd.runner import PagedCache
from tests.test_long_abi import lib  # noqa: F401
from tests.test_paged_abi import cache as some_cache, ref
from tests.test_paged_cache import D, Calls, step


@pytest.fixture
def calls(monkeypatch):
    c = Calls(monkeypatch)
    c.evictions = []
    monkeypatch.setattr(B, "l2a_cache_weights", lambda *args: None)

    def make_cache(k, v, table, ks=None, vs=None):
        x = B.l2a_cache()
        x.tensors = (k, v, ks, vs, table)
        return x

    def evict(p, cache, rows, keep, most, old, new):
        assert len(rows) == len(keep) == p.B == len(cache.tensors[4])
        c.evictions.append((rows.tolist(), keep.tolist(), most, cache.tensors[4].tolist()))
        if c.refuse == len(c.evictions):
            raise MemoryError("evict")
    monkeypatch.setattr(B, "make_cache", make_cache)
    monkeypatch.setattr(B, "l2a_cache_evict", evict)
    return c


def make(lengths=(96, 33, 10, 80)):
    """Pages of 16 tokens; W = 0: all rows but those of a last part of a page may go."""
    cache = PagedCache(B.make_params(len(lengths), 1, 4, 2, D, 0), 24, 16, 6, device="cpu", decay=0.5)
    step(cache, lengths)
    return cache


def state(cache):
    return cache.length.tolist(), cache.evicted.tolist(), cache.table.tolist(), sorted(cache.free)


def test_a_large_eviction_goes_in_several_calls(calls, monkeypatch):
    whole = make()
    whole.evict([16, 16, 0, 40])
    assert len(calls.evictions) == 1
    calls.evictions.clear()
    monkeypatch.setattr(runner, "EVICT_ROWS", 2 * 2 * 90)  # two sequences of up to 90 rows, or one longer one
    cache = make()
    tables = cache.table.copy()
    assert cache.evict([16, 16, 0, 40]).tolist() == [80, 32, 0, 48]
    assert calls.evictions == [([96], [16], 96, tables[[0]].tolist()), ([80, 32], [32, 0], 80, tables[[3, 1]].tolist())]
    assert state(cache) == state(whole) and cache.cache.tensors[4].tolist() == cache.table.tolist()


def test_a_call_without_memory_leaves_its_sequences_as_they_were(calls, monkeypatch):
    monkeypatch.setattr(runner, "EVICT_ROWS", 2 * 90)
    cache, calls.refuse = make(), 2
    with pytest.raises(MemoryError):
        cache.evict([16, 16, 0, 40])
    assert cache.length.tolist() == [16, 33, 10, 80] and cache.evicted.tolist() == [80, 0, 0, 0]  # the longest is done
    assert cache.cache.tensors[4].tolist() == cache.table.tolist()
    assert sorted(cache.free + cache.table[cache.table >= 0].tolist()) == list(range(24))


def test_lengths_that_were_taken_before_stay(calls):
    cache = make()
    length, evicted = cache.length, cache.evicted
    cache.evict([16, 16, 0, 40])
    assert length.tolist() == [96, 33, 10, 80] and evicted.tolist() == [0] * 4 and cache.length.tolist() == [16, 1, 10, 32]


def test_params_of_the_step_stay(calls):
    cache = make()
    cache.begin_step([0, 7, 5, 0])
    cache.evict([16, 16, 0, 40])
    assert cache.p.T == 12 and cache.p.B == 4


@pytest.mark.parametrize("Hkv,rows", [(8, [114688] + [64] * 63), (8, [28672] * 256), (1, [2 ** 20] * 3), (4, [8192] * 300), (16, [8193] * 100), (8, [16] * 4000)])
def test_the_workspace_stays_small(lib, Hkv, rows):  # noqa: F811
    """What the calls of an eviction need at a time: 2^22 rows of 4 or about 17 bytes, those rounded up to 8192 a KV head (at most twice as many); or one
    sequence's."""
    cache = PagedCache.__new__(PagedCache)
    cache.p = B.make_params(len(rows), 1, Hkv, Hkv, D, 0)
    groups = cache._evict_groups(np.array(rows))
    assert sorted(int(b) for g in groups for b in g) == list(range(len(rows)))
    for g in groups:
        p = B.make_params(len(g), 1, Hkv, Hkv, D, 0)
        most = max(rows[b] for b in g)
        need = lib.l2a_evict_workspace_bytes(ref(p), ref(some_cache(pages=1 << 20, page_size=1024, max_pages=1 << 14)), most)
        assert 0 < need <= max(2 * 18 << 22, 2 * 18 * Hkv * most), (len(g), need)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8,lengths", [(False, [400, 30, 555, 200, 64]), (True, [9000, 300, 8200, 100, 40])])
def test_in_one_call_and_in_several(fp8, lengths, monkeypatch):
    """Bit for bit: each KV head of a sequence is selected from by itself."""
    results = []
    for limit in (1 << 22, 2 * 600):
        monkeypatch.setattr(runner, "EVICT_ROWS", limit)
        g = torch.Generator(device="cuda").manual_seed(3)
        n = sum(lengths)
        cache = PagedCache(B.make_params(5, 1, 8, 2, 128, 20), 700, 32, 300, fp8=fp8, decay=0.9)
        q, k, v = (torch.randn(n, h, 128, generator=g, device="cuda").bfloat16() for h in (8, 2, 2))
        cache.extend(lengths, q, k, v, torch.ones(1, n, dtype=torch.uint8, device="cuda"))
        gone = cache.evict([100, 10, 333, 200, 50])
        assert gone.tolist() == [x - y for x, y in zip(lengths, cache.length.tolist())] and gone[0] > 0 and gone[3] == 0
        results.append((cache.length.tolist(), [t for b in range(5) for t in cache.read(b)],
                        [torch.cat([cache.weight[i] for i in cache.table[b] if i >= 0], 1)[:, :int(cache.length[b])] for b in range(5) if cache.length[b]]))
    a, b = results
    assert a[0] == b[0] and all(torch.equal(x, y) for x, y in zip(a[1], b[1])) and all(torch.equal(x, y) for x, y in zip(a[2], b[2]))
