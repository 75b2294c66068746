"""Eviction from a paged KV cache against a sort: which rows stay, where they go, and that nothing else changes, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator
from tests.fp4_helpers import make_step, whole_cache
from tests.paged_helpers import up

pytestmark = pytest.mark.gpu


def reference(w, keep):
    """-> which row each of rows 0 .. keep - 1 was before, by the definition."""
    n = len(w)
    order = sorted(range(n), key=lambda j: (-np.inf if np.isnan(w[j]) else w[j], -j), reverse=True)
    # (NaN is less than everything, -inf too)
    order = [j for j in order if not np.isnan(w[j])] + [j for j in range(n) if np.isnan(w[j])]
    stays = set(order[:keep])
    behind = iter(sorted(j for j in stays if j >= keep))
    return [j if j in stays else next(behind) for j in range(keep)]


def check(s, rows, keep, weights, in_place=True, kept_wanted=True, max_rows=None):
    """weights(rng, shape): of all rows of the pool."""
    alloc = GuardedAllocator()
    p, c, _, _ = whole_cache(s, alloc)
    rng = np.random.default_rng(1)
    w = weights(rng, (s.pages, s.Hkv, s.page)).astype(np.float32)
    max_rows = max(max(rows), 1) if max_rows is None else max_rows
    weight_in = alloc(w.shape).copy_(up(w))
    weight = weight_in if in_place else alloc(w.shape).fill_(-77.0)
    kept = alloc((s.B, s.Hkv, max_rows), torch.int32).fill_(-9) if kept_wanted else None
    before = [t.view(torch.uint8).cpu().numpy().reshape(s.pages, s.Hkv, s.page, -1) for t in c.tensors[:4] if t is not None]
    want = [x.copy() for x in before]
    want_w, want_kept = (w.copy() if in_place else np.full_like(w, -77.0)), np.full((s.B, s.Hkv, max_rows), -9)
    for b in range(s.B):
        n = min(max(rows[b], 0), max_rows)
        m = min(max(keep[b], 0), n)
        for hk in range(s.Hkv):
            source = reference([w[s.place(b, j)[0], hk, s.place(b, j)[1]] for j in range(n)], m)
            want_kept[b, hk, :m] = source
            for j, src in enumerate(source):
                (tp, ta), (fp, fa) = s.place(b, j), s.place(b, src)
                for x, y in zip(want, before):
                    x[tp, hk, ta] = y[fp, hk, fa]
                want_w[tp, hk, ta] = w[fp, hk, fa]
    ws = B.alloc_evict_workspace(p, c, max_rows, alloc).fill_(255)
    B.l2a_cache_evict(p, c, up(np.array(rows, np.int32)), up(np.array(keep, np.int32)), max_rows, weight_in, weight, kept, ws)
    torch.cuda.synchronize()
    alloc.check()
    if kept is not None:
        assert np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(weight.cpu().numpy().view(np.uint32), want_w.view(np.uint32))
    for t, x in zip((t for t in c.tensors[:4] if t is not None), want):
        assert np.array_equal(t.view(torch.uint8).cpu().numpy().reshape(x.shape), x)
    if not in_place:
        assert np.array_equal(weight_in.cpu().numpy().view(np.uint32), w.view(np.uint32))


def spread(rng, shape):
    return np.exp(3 * rng.standard_normal(shape)) * (rng.random(shape) < 0.9)


CASES = {  # bits, lengths, Hkv, page, rows, keep
    "one row": (16, [1], 1, 16, [1], [1]),
    "one row goes": (16, [1], 1, 16, [1], [0]),
    "one of two": (8, [2], 3, 16, [2], [1]),
    "half": (16, [64], 2, 16, [48], [16]),
    "e4m3": (8, [100, 7, 333], 4, 16, [96, 0, 320], [32, 0, 300]),
    "e2m1": (4, [100, 77, 333], 4, 32, [96, 64, 320], [0, 64, 1]),
    "all stay, all go, more than there are": (16, [90, 90, 90], 2, 64, [64, 64, 64], [64, 0, 1000]),
    "odd": (4, [1000, 17], 2, 16, [999, 17], [333, 16]),
    "a round of the selection and one more": (8, [1025, 1024, 1023], 1, 256, [1025, 1024, 1023], [512, 511, 1022]),
    "long": (16, [9000], 2, 64, [8960], [4032]),
    "longer": (4, [40000, 3], 1, 128, [39936, 2], [20096, 1]),
    "more heads than CUs": (16, [40 + i % 7 for i in range(40)], 8, 16, [32 + i % 9 for i in range(40)], [16 + i % 13 for i in range(40)]),
    "more heads than CUs, e4m3": (8, [400 + 16 * (i % 5) for i in range(33)], 8, 16, [400 - i for i in range(33)], [180 + 5 * i for i in range(33)]),
    "more heads than CUs, e2m1": (4, [2100, 3, 16] + [30] * 30, 8, 16, [2099, 3, 16] + [30] * 30, [1000, 1, 16] + [i for i in range(30)]),
    "twice as many": (4, [5 + 3 * i for i in range(66)], 8, 16, [4 + 3 * i for i in range(66)], [2 + i for i in range(66)]),
    "twice as many, long": (8, [2048, 2047, 1] + [20] * 61, 8, 64, [2048, 2046, 1] + [19] * 61, [1024, 2000, 0] + [i % 20 for i in range(61)]),
    "many": (8, [33 + 5 * i for i in range(60)], 2, 16, [32 + 5 * i for i in range(60)], [16 + i for i in range(60)]),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(name, in_place):
    bits, lengths, Hkv, page, rows, keep = CASES[name]
    s = make_step(bits, [0] * len(lengths), lengths, Hkv, Hkv, 4, page, seed=len(name), tail=1)
    check(s, rows, keep, spread, in_place, kept_wanted=in_place)


VALUES = {
    "equal": lambda rng, shape: np.full(shape, 0.25),
    "few values": lambda rng, shape: rng.integers(0, 3, shape) / 2.0,
    "zeros of both signs": lambda rng, shape: np.where(rng.random(shape) < 0.5, -0.0, 0.0),
    "signs": lambda rng, shape: rng.standard_normal(shape),
    "near one another": lambda rng, shape: 1.0 + rng.integers(0, 300, shape) * 2.0 ** -23,
    "subnormal": lambda rng, shape: rng.integers(0, 2000, shape) * 2.0 ** -149,
    "infinities and NaN": lambda rng, shape: rng.choice([np.inf, -np.inf, np.nan, -np.nan, 0.0, 1.0, -1.0], shape),
    "NaN": lambda rng, shape: np.full(shape, np.nan),
    "ascending": lambda rng, shape: np.arange(np.prod(shape)).reshape(shape),
}


@pytest.mark.parametrize("name", VALUES)
@pytest.mark.parametrize("rows,keep", [(100, 37), (2100, 1050), (2100, 5)])
def test_weights_of_all_kinds(name, rows, keep):
    check(make_step(8, [0], [rows], 2, 2, 4, 64, seed=2, tail=1), [rows], [keep], VALUES[name])


@pytest.mark.parametrize("name", VALUES)
@pytest.mark.parametrize("sequences", [33, 65])  # times 8 KV heads
def test_weights_of_all_kinds_where_a_workgroup_does_it_all(name, sequences):
    rows = [1500] + [40 + i % 50 for i in range(sequences - 1)]
    check(make_step(4, [0] * sequences, rows, 8, 8, 4, 16, seed=3, tail=1), rows, [700] + [i % 60 for i in range(sequences - 1)], VALUES[name], in_place=sequences == 65)


@pytest.mark.parametrize("page", [16, 1024])
def test_as_many_rows_as_a_workgroup_takes(page):
    lengths = [8192, 8191] + [5] * 126
    check(make_step(8, [0] * 128, lengths, 2, 2, 4, page, seed=4, tail=1, more_pages=0), lengths, [4096, 8000] + [3] * 126, spread, in_place=False)


@pytest.mark.parametrize("rows,keep,kinds", [(600001, 299999, 10 ** 9), (600001, 599990, 50), (530000, 17, 10 ** 9), (8193, 4000, 10 ** 9), (16385, 9000, 1)])
def test_long_caches(rows, keep, kinds):
    """More rows than a workgroup takes, and more than 64 times that many; ties across their shares."""
    rng = np.random.default_rng(rows + keep)
    page, Hkv = 128, 2
    pages = -(-rows // page)
    p = B.make_params(1, 1, Hkv, Hkv, 128, 4)
    c = B.alloc_cache(p, pages, page, pages, fp4=True)
    table = rng.permutation(pages).astype(np.int32)
    c.tensors[4].copy_(up(table[None]))
    for t in c.tensors[:4]:
        t.copy_(torch.randint(0, 256, t.shape, dtype=torch.uint8, device="cuda"))
    w = np.exp(rng.standard_normal((Hkv, rows)) * 4).astype(np.float32) if kinds > rows else rng.integers(0, kinds, (Hkv, rows)).astype(np.float32)
    place = table[np.arange(rows) // page].astype(np.int64), np.arange(rows) % page
    pool = np.zeros((pages, Hkv, page), np.float32)
    for h in range(Hkv):
        pool[place[0], h, place[1]] = w[h]
    weight, kept = up(pool), torch.full((1, Hkv, rows), -9, dtype=torch.int32, device="cuda")
    before = [t.cpu().numpy() for t in c.tensors[:4]]
    B.l2a_cache_evict(p, c, up(np.array([rows], np.int32)), up(np.array([keep], np.int32)), rows, weight, weight, kept)
    got, got_kept = weight.cpu().numpy(), kept.cpu().numpy()[0]
    for h in range(Hkv):
        stays = np.zeros(rows, bool)
        stays[np.argsort(-w[h], kind="stable")[:keep]] = True
        source = np.arange(keep)
        source[~stays[:keep]] = keep + np.nonzero(stays[keep:])[0]
        assert np.array_equal(got_kept[h, :keep], source) and (got_kept[h, keep:] == -9).all()
        assert np.array_equal(got[place[0][:keep], h, place[1][:keep]], w[h][source])
        assert np.array_equal(got[place[0][keep:], h, place[1][keep:]], w[h][keep:])
        for t, x in zip(c.tensors[:4], before):
            y = x.copy()
            y[place[0][:keep], h, place[1][:keep]] = x[place[0][source], h, place[1][source]]
            assert np.array_equal(t.cpu().numpy()[:, h], y[:, h])


def test_sizes_out_of_range_are_clamped():
    s = make_step(16, [0, 0, 0], [40, 40, 40], 2, 2, 4, 16, seed=3, tail=1)
    check(s, [-5, 30, 2 ** 31 - 1], [7, -3, 16], spread, max_rows=40)


def test_pages_outside_the_pool_are_not_followed():
    s = make_step(4, [0, 0], [64, 64], 2, 2, 4, 16, seed=4, tail=1)
    alloc = GuardedAllocator()
    p, c, _, _ = whole_cache(s, alloc)
    weight = alloc((s.pages, s.Hkv, s.page)).copy_(up(spread(np.random.default_rng(2), (s.pages, s.Hkv, s.page)).astype(np.float32)))
    used = s.table[:, :4].copy()
    s.table[0, 1], s.table[0, 3] = -1, 2 ** 31 - 1
    c.tensors[4].copy_(up(s.table))
    before = [t.clone() for t in c.tensors[:4]] + [weight.clone()]
    B.l2a_cache_evict(p, c, up(np.array([64, 0], np.int32)), up(np.array([32, 0], np.int32)), 64, weight, weight)
    torch.cuda.synchronize()
    alloc.check()
    others = [i for i in range(s.pages) if i != used[0, 0]]  # rows 0..15 are the only ones that can have changed
    for t, x in zip((*c.tensors[:4], weight), before):
        assert torch.equal(t[others], x[others])


def test_calls_without_rows_change_nothing():
    s = make_step(8, [0, 0], [64, 10], 2, 2, 4, 16, seed=5, tail=1)
    check(s, [0, 0], [0, 5], spread, max_rows=1)
