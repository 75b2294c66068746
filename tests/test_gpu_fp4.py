"""A paged KV cache in 4 bits against plain 64-bit forms: rows written (bits) and read back, and the attention of new tokens over it."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator, to_host
from tests import paged_helpers
from tests.fp4_helpers import E2M1, Step4, cache_on_gpu, dequantise4, quantise4
from tests.paged_helpers import D, SENTINEL, up

pytestmark = pytest.mark.gpu


@pytest.fixture
def check(monkeypatch):
    """paged_helpers' whole comparison, whose tolerances are those of any bf16 cache values, on a cache in 4 bits."""
    monkeypatch.setattr(paged_helpers, "cache_on_gpu", cache_on_gpu)
    return paged_helpers.check_extend


ROWS = [  # new, cached, KV heads, page, tokens before the first and behind the last sequence
    ([1], [0], 1, 16, 0, 0), ([5, 0, 1, 33], [15, 7, 16, 0], 4, 16, 2, 3), ([300], [77], 8, 64, 0, 5), ([1] * 70, [3 * i for i in range(70)], 2, 16, 0, 0),
    ([0, 0, 3, 0], [0, 0, 1022, 0], 2, 1024, 0, 0), ([1100, 950], [7, 300], 9, 32, 1, 2)]


@pytest.mark.parametrize("new,cached,Hkv,page,lead,tail", ROWS)
def test_rows_are_written_and_read_back(new, cached, Hkv, page, lead, tail):
    s = Step4(new, cached, Hkv, Hkv, 4, page, seed=len(new) + page, lead=lead, tail=tail)
    alloc = GuardedAllocator()
    none = [0] * s.B
    p, c = cache_on_gpu(s, alloc, s.pool(s.k, [None] * s.B, none), s.pool(s.v, [None] * s.B, none))
    packed = []
    for rows in (s.k, s.v):
        x = np.full((s.N, Hkv, D), np.nan)
        for b in range(s.B):
            x[s.start[b]:s.start[b + 1]] = rows[b][cached[b]:]
        packed.append(x)
    start, pos = up(s.start), up(np.array(cached, np.int32))
    B.l2a_cache_write(p, c, *(up(x, torch.bfloat16) for x in packed), start, pos)
    torch.cuda.synchronize()
    alloc.check()
    for rows, pool, scale in ((s.k, c.tensors[0], c.tensors[2]), (s.v, c.tensors[1], c.tensors[3])):
        x, e = s.pool(rows, [None] * s.B, none)  # the new rows and nothing else
        for b in range(s.B):
            for t in range(cached[b], cached[b] + new[b]):
                page_, at = s.place(b, t)
                x[page_, :, at], e[page_, :, at] = quantise4(rows[b][t])
        assert np.array_equal(pool.cpu().numpy(), x) and np.array_equal(scale.cpu().numpy(), e)
    back = [alloc((s.N, Hkv, D), torch.bfloat16).fill_(SENTINEL) for _ in range(2)]
    B.l2a_cache_read(p, c, start, pos, *back)
    torch.cuda.synchronize()
    alloc.check()
    for got, want in zip(back, packed):
        got = to_host(got)
        assert np.array_equal(got[lead:s.N - tail], dequantise4(*quantise4(want[lead:s.N - tail])))
        assert (got[:lead] == SENTINEL).all() and (got[s.N - tail:] == SENTINEL).all()


def through_cache(x):
    """x [N, 128] through a cache of one head and pages of 16: (bytes, exponents, values read back)."""
    n = len(x)
    p, pages = B.make_params(1, n, 1, 1, D, 4), -(-n // 16)
    c = B.alloc_cache(p, pages, 16, pages, fp4=True)
    c.tensors[4].copy_(torch.arange(pages, dtype=torch.int32))
    start, pos = up(np.array([0, n], np.int32)), up(np.zeros(1, np.int32))
    k = x.view(n, 1, D).cuda()
    back = [torch.empty_like(k) for _ in range(2)]
    B.l2a_cache_write(p, c, k, k, start, pos)
    B.l2a_cache_read(p, c, start, pos, *back)
    assert torch.equal(back[0].view(torch.int16), back[1].view(torch.int16))
    return c.tensors[0].cpu().numpy().reshape(-1, D // 2)[:n], c.tensors[2].cpu().numpy().reshape(-1, 4)[:n], to_host(back[0]).reshape(n, D)


def test_every_finite_bf16_number_is_rounded_to_nearest():
    """Every finite bf16 number as the largest of its block, beside numbers of all sizes below, ties among them."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    every = every[torch.isfinite(every)]
    g = torch.Generator().manual_seed(5)
    part = torch.randint(0, 65, (len(every), 31), generator=g) / 64.0 * torch.where(torch.rand(len(every), 31, generator=g) < 0.5, -1.0, 1.0)
    blocks = torch.cat([every[:, None], (every.float()[:, None] * part).bfloat16()], 1)
    blocks = torch.cat([blocks, torch.zeros(-len(blocks) % 4, 32, dtype=torch.bfloat16)])
    x = blocks.view(-1, D)
    code, e, back = through_cache(x)
    want_code, want_e = quantise4(x.double().numpy())
    assert np.array_equal(e, want_e) and np.array_equal(code, want_code)
    assert np.array_equal(back, dequantise4(code, e))  # exact, the largest and the smallest of them too


def test_blocks_that_are_no_numbers_are_nan_and_no_others():
    x = torch.randn(64, D, generator=torch.Generator().manual_seed(6)).bfloat16()
    bad = {(3, 5): np.nan, (3, 40): np.inf, (9, 127): -np.inf, (9, 0): np.nan, (63, 64): np.inf}
    for at, value in bad.items():
        x[at] = value
    code, e, back = through_cache(x)
    nan = np.zeros((64, 4), bool)
    for row, channel in bad:
        nan[row, channel // 32] = True
    assert np.array_equal(e == 255, nan) and np.array_equal(np.isnan(back), nan.repeat(32, 1))
    good = ~nan.repeat(32, 1)
    assert np.array_equal(back[good], dequantise4(*quantise4(np.nan_to_num(x.double().numpy())))[good])


# new, cached, Hq, Hkv, W, page and more
CASES = {
    "one token": ([1], [0], 1, 1, 4, 16, {}),
    "one behind many": ([1], [700], 28, 4, 100, 64, dict(f=1.0)),
    "steps": ([1, 1, 0, 1, 1], [0, 15, 9, 16, 333], 16, 2, 30, 16, dict(lead=1, tail=2)),
    "a decision per head": ([1, 1, 1], [40, 200, 129], 8, 2, 20, 32, dict(Hm=8, f=0.5)),
    "drafts": ([5, 3, 9], [100, 31, 500], 12, 1, 64, 16, dict(Hm=1, f=0.5)),
    "up to 128 rows": ([17, 30], [77, 150], 4, 1, 50, 64, dict(f=0.5)),
    "chunk of many rows": ([150], [333], 8, 2, 70, 16, dict(f=0.5)),
    "first chunks": ([130, 77], [0, 0], 4, 2, 40, 16, dict(Hm=4, f=0.3)),
    "mixed": ([100, 1, 1, 9], [65, 400, 31, 17], 16, 4, 33, 16, dict(f=0.4, lead=3, tail=1)),
    "nobody routed": ([40, 1], [100, 100], 4, 2, 16, 16, dict(f=0.0)),
    "all routed, no window": ([70, 2], [90, 300], 8, 1, 0, 256, dict(f=1.0, Hm=1)),
    "16 heads a group": ([3, 20], [50, 60], 16, 1, 20, 128, dict(f=0.6, Hm=16)),
}


@pytest.mark.parametrize("name", CASES)
def test_extend(check, name):
    new, cached, Hq, Hkv, W, page, more = CASES[name]
    check(Step4(new, cached, Hq, Hkv, W, page, seed=len(name), **more))


@pytest.mark.parametrize("flags", [B.L2A_FLAG_DENSE, B.L2A_FLAG_SKIP_LOCAL, B.L2A_FLAG_SKIP_GLOBAL, B.L2A_FLAG_DENSE | B.L2A_FLAG_SKIP_LOCAL])
@pytest.mark.parametrize("new", [[1, 1, 4], [90, 1, 40]])
def test_flags(check, flags, new):
    check(Step4(new, [100, 33, 0], 8, 2, 25, 16, f=0.5, seed=flags), flags)


@pytest.mark.parametrize("new,cached", [([5], [60]), ([40, 3], [33, 20]), ([140], [30])])
def test_blocks_that_are_nan_reach_the_rows_that_see_them_and_no_others(check, new, cached):
    s = Step4(new, cached, 4, 2, 12, 16, f=0.5, seed=9)
    s.k[0][cached[0] - 20, 1, 3] = np.nan
    s.v[0][cached[0] + 2, 0, 70] = np.inf
    s.v[0][-1, 1, 5] = np.nan
    check(s)


# up to 16 rows per KV head, for which there are tiles of 16 x 16: new, cached, Hq, Hkv, W, page and more
SIXTEEN = {
    "as many rows as fit": ([2, 1, 2], [300, 77, 0], 16, 2, 40, 16, dict(Hm=16, f=0.5)),
    "one head each, sixteen tokens": ([16, 3, 0, 16], [33, 1, 50, 200], 2, 2, 21, 32, dict(f=0.5, lead=2, tail=3)),
    "no window": ([4, 1], [95, 17], 4, 1, 0, 1024, dict(f=0.6)),
    "several tiles a workgroup": ([1] * 64, [(37 * i) % 150 for i in range(64)], 16, 8, 16, 16, dict(f=0.7)),
    "more KV heads than a plan of its own": ([1, 0, 2, 1] * 35, [(53 * i) % 170 for i in range(140)], 8, 4, 30, 16, dict(f=0.6)),
    "long and short": ([1] * 12, [0, 5000, 31, 32, 33, 1, 64, 2900, 16, 15, 17, 127], 4, 1, 100, 64, dict(f=0.8)),
}


@pytest.mark.parametrize("name", SIXTEEN)
def test_up_to_sixteen_rows(check, name):
    new, cached, Hq, Hkv, W, page, more = SIXTEEN[name]
    check(Step4(new, cached, Hq, Hkv, W, page, seed=len(name), **more))


def test_tiles_behind_one_with_nan_are_what_they_would_be(check):
    """Rows with a masked NaN among their keys are worked out one by one, while the workgroup's next tile has begun."""
    s = Step4([3] * 64, [(41 * i) % 90 for i in range(64)], 16, 8, 12, 16, f=0.6, seed=11)
    for b in range(0, 64, 3):
        s.v[b][-1, b % 8, 70] = np.nan      # the last token's, which the two before it must not see
        s.k[b][s.cached[b] + 1, (b + 1) % 8, 3] = np.inf
        s.v[b][s.cached[b] // 2, (b + 2) % 8, 127] = np.inf
    check(s)


def test_rows_outside_the_table_or_the_pool_are_skipped():
    p = B.make_params(2, 8, 2, 2, D, 4)
    c = B.alloc_cache(p, 3, 16, 2, fp4=True)
    for t in c.tensors[:4]:
        t.fill_(0x55)
    c.tensors[4].copy_(torch.tensor([[0, 7], [-3, 2]], dtype=torch.int32))
    k = torch.randn(8, 2, D, device="cuda").bfloat16()
    B.l2a_cache_write(p, c, k, k, up(np.array([0, 4, 8], np.int32)), up(np.array([14, 14], np.int32)))  # rows 14..17 of both
    rows = c.tensors[0].cpu().numpy()
    written = np.zeros((3, 16), bool)
    written[0, 14:] = written[2, :2] = True
    assert np.array_equal((rows != 0x55).any((1, 3)), written)


def test_values_of_every_element_and_scale_are_exact():
    """Every byte beside exponents of the whole range: what reading gives is the element times its power of two."""
    p = B.make_params(1, 64, 1, 1, D, 4)
    c = B.alloc_cache(p, 4, 16, 4, fp4=True)
    code = np.arange(64 * 64, dtype=np.int64).reshape(4, 1, 16, 64) * 7 % 256
    e = np.concatenate([np.linspace(2, 252, 255).astype(int), [255]]).reshape(4, 1, 16, 4)
    for t, x in zip(c.tensors[:4], (code, code, e, e)):
        t.copy_(up(x.astype(np.uint8)))
    c.tensors[4].copy_(torch.arange(4, dtype=torch.int32))
    k, v = (torch.empty(64, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.l2a_cache_read(p, c, up(np.array([0, 64], np.int32)), up(np.zeros(1, np.int32)), k, v)
    want = dequantise4(code.astype(np.uint8).reshape(64, 1, 64), e.astype(np.uint8).reshape(64, 1, 4))
    assert np.isnan(want[-1, 0, -32:]).all() and set(np.abs(want[:8]).ravel() / 2.0 ** np.floor(np.log2(np.abs(want[:8]).ravel() + 1e-300))) <= {0.0, 1.0, 1.5}
    for got in (k, v):
        got = to_host(got)
        assert np.array_equal(got, want, equal_nan=True) and np.array_equal(np.signbit(got[:63]), np.signbit(want[:63]))
    assert len(E2M1) == 8
