"""Every form of the eviction's kernels with every type of elements, and with tables that name pages outside the pool, bit for bit against a sort."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator
from tests.fp4_helpers import make_step, whole_cache
from tests.paged_helpers import up
from tests.test_gpu_cache_evict import check, reference, spread

pytestmark = pytest.mark.gpu

FORMS = {  # lengths, Hkv: the moves by a kernel of their own; by who selects, of 1024 threads and of 256; several workgroups a KV head
    "moves apart": ([600, 77, 2100], 2),
    "a workgroup does it all": ([2500, 300] + [40 + i % 30 for i in range(31)], 8),
    "one of 256 threads": ([2048, 300] + [40 + i % 30 for i in range(63)], 8),
    "many workgroups a KV head": ([9000, 100, 17000], 1),
}


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("form", FORMS)
def test_elements_of_all_types(form, bits):
    lengths, Hkv = FORMS[form]
    s = make_step(bits, [0] * len(lengths), lengths, Hkv, Hkv, 4, 16, seed=bits, tail=1)
    check(s, lengths, [n * (3 + b % 4) // 8 for b, n in enumerate(lengths)], spread, in_place=bits != 8)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("form", FORMS)
def test_pages_outside_the_pool(form, bits):
    """Moves from and to their rows are left out, all others are made.  (What such a row weighs is the weight in the nearest page there is.)"""
    lengths, Hkv = FORMS[form]
    s = make_step(bits, [0] * len(lengths), lengths, Hkv, Hkv, 4, 16, seed=bits, tail=1)
    alloc = GuardedAllocator()
    p, c, _, _ = whole_cache(s, alloc)
    rng = np.random.default_rng(7)
    w = spread(rng, (s.pages, s.Hkv, s.page)).astype(np.float32)
    table = s.table.copy()
    for b, n in enumerate(lengths):  # a page before and one behind the rows that stay
        pages = -(-n // 16)
        table[b, pages // 8], table[b, pages - 1] = (-1, s.pages) if b % 2 else (2 ** 31 - 1, -2 ** 31)
    c.tensors[4].copy_(up(table))
    keep = [n // 2 for n in lengths]
    weight_in, weight = alloc(w.shape).copy_(up(w)), alloc(w.shape).fill_(-77.0)
    kept = alloc((s.B, s.Hkv, max(lengths)), torch.int32).fill_(-9)
    before = [t.view(torch.uint8).cpu().numpy().reshape(s.pages, s.Hkv, s.page, -1) for t in c.tensors[:4] if t is not None]
    want, want_w, want_kept = [x.copy() for x in before], np.full_like(w, -77.0), np.full(tuple(kept.shape), -9)

    def place(b, j):
        page = int(table[b, j // 16])
        return 0 <= page < s.pages, min(max(page, 0), s.pages - 1), j % 16
    left_out = made = 0
    for b, n in enumerate(lengths):
        for hk in range(Hkv):
            source = reference([w[place(b, j)[1], hk, place(b, j)[2]] for j in range(n)], keep[b])
            want_kept[b, hk, :keep[b]] = source
            for j, src in enumerate(source):
                (to_real, tp, ta), (from_real, fp, fa) = place(b, j), place(b, src)
                if not to_real or not from_real:
                    left_out += src != j
                    # a weight that stays in its place is copied, one that leaves is copied too before another takes the place
                    if to_real:
                        want_w[tp, hk, ta] = w[tp, hk, ta]
                    continue
                made += src != j
                for x, y in zip(want, before):
                    x[tp, hk, ta] = y[fp, hk, fa]
                want_w[tp, hk, ta] = w[fp, hk, fa]
    assert left_out > 0 and made > 0
    B.l2a_cache_evict(p, c, up(np.array(lengths, np.int32)), up(np.array(keep, np.int32)), max(lengths), weight_in, weight, kept, B.alloc_evict_workspace(p, c, max(lengths), alloc).fill_(255))
    torch.cuda.synchronize()
    alloc.check()
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    for t, x in zip((t for t in c.tensors[:4] if t is not None), want):
        assert np.array_equal(t.view(torch.uint8).cpu().numpy().reshape(x.shape), x)
    assert np.array_equal(weight.cpu().numpy().view(np.uint32), want_w.view(np.uint32))
