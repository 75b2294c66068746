"""The attention weights that cached rows receive, against the formula in 64 bits.

Tolerances.  A score is 128 products of bf16 numbers, exact in 32 bits, summed in 32 bits: off by at most 128 2^-24 sum |q k|.  Its exponential
takes a product, the log-sum-exp in units of log 2 and their difference, each rounded once (2^-24 of numbers up to |scale s| + |lse|, and log2 e
itself), and is good to 2^-22.  So a term is off by its 2^-24 (128 scale sum |q k| + 6 (|scale s| + |lse|) + 8); a sum of n terms besides by n 2^-24 of
the sum, and the decayed old weight by two roundings.
"""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator, to_host
from tests.fp4_helpers import make_step, whole_cache
from tests.paged_helpers import D, near, up

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
GONE = -77.0


def log_sums(s, k, scale, f, rng):
    """lse [Hq, N] as the attention leaves it: -inf where a token is not routed; routed at random, by head."""
    lse = np.full((s.Hq, s.N), -np.inf, np.float32)
    for b in range(s.B):
        for i in range(s.new[b]):
            t, token = s.cached[b] + i, s.start[b] + i
            for h in range(s.Hq):
                if rng.random() < f:
                    x = k[b][:t + 1, h // (s.Hq // s.Hkv)] @ s.q[token, h] * scale
                    m = np.fmax.reduce(x)
                    with np.errstate(invalid="ignore"):
                        lse[h, token] = m + np.log(np.nansum(np.exp(x - m)))
    return lse


def reference(s, k, lse, decay, old, scale):
    """-> weights and tolerances [pages, Hkv, page]; rows that are not written: GONE, 0."""
    G = s.Hq // s.Hkv
    out, tol = np.full((s.pages, s.Hkv, s.page), GONE), np.zeros((s.pages, s.Hkv, s.page))
    for b in range(s.B):
        if s.new[b] == 0:
            continue
        n = s.cached[b] + s.new[b]
        for hk in range(s.Hkv):
            w, e = np.zeros(n), np.zeros(n)
            terms = 0
            for i in range(s.new[b]):
                t, token = s.cached[b] + i, s.start[b] + i
                for h in range(hk * G, hk * G + G):
                    if not np.isfinite(lse[h, token]):
                        continue
                    x = k[b][:t + 1, hk] @ s.q[token, h] * scale
                    size = np.abs(k[b][:t + 1, hk]) @ np.abs(s.q[token, h]) * scale
                    p = np.exp(x - float(lse[h, token]))
                    w[:t + 1] += p
                    e[:t + 1] += p * ULP * (128 * size + 6 * (np.abs(x) + abs(lse[h, token])) + 8)
                    terms += 1
            e += terms * ULP * w
            for j in range(n):
                page, at = s.place(b, j)
                before = decay * old[page, hk, at] if j < s.cached[b] and old is not None and decay else 0.0
                out[page, hk, at] = w[j] + before
                tol[page, hk, at] = e[j] + 2 * ULP * (w[j] + abs(before))
    return out, tol


def check(s, f=0.5, decay=1.0, with_old=True, in_place=False, scale=None, max_new=None, lse=None, change=None):
    alloc = GuardedAllocator()
    p, c, k, _ = whole_cache(s, alloc)
    p = s.params(0, scale)
    scale = D ** -0.5 if scale is None else scale
    rng = np.random.default_rng(3)
    lse = log_sums(s, k, scale, f, rng) if lse is None else lse
    old = rng.exponential(size=(s.pages, s.Hkv, s.page)).astype(np.float32)
    want, tol = reference(s, k, lse, np.float32(decay), old if with_old else None, scale)
    if change:  # what must not matter
        change(old, lse)
    q = s.q.copy()
    used = np.zeros(s.N, bool)
    used[s.start[0]:s.start[-1]] = True
    q[~used] = np.nan
    weight_in = alloc((s.pages, s.Hkv, s.page)).copy_(up(old))
    weight = weight_in if in_place else alloc((s.pages, s.Hkv, s.page)).fill_(GONE)
    lse_gpu = alloc((s.Hq, s.N)).copy_(up(lse))
    if not used.all():
        lse_gpu[:, ~torch.from_numpy(used).cuda()] = float("nan")
    max_new = max(max(s.new), 1) if max_new is None else max_new
    ws = B.alloc_weights_workspace(p, c, max_new, alloc)
    if ws is not None:
        ws.fill_(255)
    B.l2a_cache_weights(p, c, up(q, torch.bfloat16), up(s.start), up(np.array(s.cached, np.int32)), lse_gpu, max_new, decay, weight_in if with_old else None, weight, ws)
    torch.cuda.synchronize()
    alloc.check()
    if in_place:
        want = np.where(want == GONE, old, want)
    near("weights", to_host(weight), want, tol)
    return weight


CASES = {  # bits, new, cached, Hq, Hkv, page, routed, more
    "one token": (16, [1], [0], 1, 1, 16, 1.0, {}),
    "one routed, one not": (8, [1, 1], [5, 5], 4, 2, 16, 0.5, {}),
    "nobody routed": (4, [3, 1], [40, 2], 8, 2, 16, 0.0, {}),
    "steps": (16, [1, 1, 0, 1, 1], [0, 31, 9, 32, 333], 16, 2, 16, 0.7, dict(lead=2, tail=3)),
    "steps e4m3": (8, [1, 1, 0, 1, 1], [63, 64, 65, 700, 15], 28, 4, 64, 0.7, {}),
    "steps e2m1": (4, [1, 1, 0, 1, 1], [127, 128, 129, 255, 256], 32, 8, 32, 0.7, {}),
    "drafts": (16, [5, 2, 9], [100, 31, 500], 12, 1, 16, 0.5, {}),
    "32 rows": (4, [8, 32], [77, 0], 4, 1, 64, 1.0, {}),
    "33 rows": (16, [33, 11], [77, 200], 3, 1, 64, 1.0, {}),
    "chunk": (16, [150], [333], 8, 2, 16, 0.5, {}),
    "chunk e4m3": (8, [260, 1], [255, 900], 4, 2, 32, 0.3, dict(lead=1)),
    "chunk e2m1": (4, [300], [512], 4, 1, 128, 0.6, {}),
    "first chunks": (16, [257, 64, 256], [0, 0, 0], 4, 2, 16, 0.4, {}),
    "mixed": (8, [200, 1, 1, 9, 0], [65, 400, 31, 17, 50], 16, 4, 16, 0.4, dict(lead=3, tail=1)),
    "sparse": (4, [400], [100], 2, 1, 16, 0.02, {}),
    "16 heads a group": (16, [3, 40], [50, 60], 16, 1, 128, 0.6, {}),
}


@pytest.mark.parametrize("name", CASES)
def test_weights(name):
    bits, new, cached, Hq, Hkv, page, f, more = CASES[name]
    check(make_step(bits, new, cached, Hq, Hkv, 10, page, seed=len(name), **more), f)


@pytest.mark.parametrize("decay,with_old,in_place", [(0.0, True, False), (0.5, True, True), (1.0, False, False), (0.0, False, True), (1.0, True, True), (0.9, True, False)])
@pytest.mark.parametrize("new", [[1, 2], [120, 1]])
def test_old_weights(new, decay, with_old, in_place):
    check(make_step(16, new, [70, 33], 4, 2, 10, 16, seed=1), 0.5, decay, with_old, in_place)


@pytest.mark.parametrize("decay,with_old,in_place", [(0.0, True, False), (0.5, True, True), (1.0, False, False), (0.0, False, True), (0.9, True, False)])
@pytest.mark.parametrize("bits,new,Hq,Hkv,page", [(4, [1, 0, 2], 16, 2, 16), (8, [2, 1, 1], 16, 2, 1024), (8, [8, 1, 5], 10, 5, 32), (4, [16, 9, 16], 3, 3, 64), (4, [1, 1, 1], 16, 1, 16)])
def test_up_to_sixteen_rows(bits, new, Hq, Hkv, page, decay, with_old, in_place):
    check(make_step(bits, new, [70, 129, 0], Hq, Hkv, 10, page, seed=page, lead=1, tail=2), 0.6, decay, with_old, in_place)


@pytest.mark.parametrize("new", [[2, 1], [90, 3]])
def test_what_must_not_matter(new):
    """Old weights of the new tokens' rows, and all of them where nothing of them stays; log-sum-exps that are no finite numbers count as not routed."""
    s = make_step(8, new, [50, 31], 4, 2, 10, 16, seed=2)

    def spoil(old, lse):
        for b in range(2):
            for t in range(s.cached[b], s.cached[b] + s.new[b]):
                old[s.place(b, t)[0], :, s.place(b, t)[1]] = np.nan
        lse[np.isneginf(lse)] = np.array([np.nan, np.inf, -np.inf], np.float32)[np.arange(np.isneginf(lse).sum()) % 3]
    check(s, 0.5, change=spoil)

    def spoil_all(old, lse):
        old[...] = np.nan
    check(s, 0.5, decay=0.0, change=spoil_all)


@pytest.mark.parametrize("bits,new", [(16, [1]), (16, [70]), (4, [2]), (4, [70])])
def test_keys_that_are_no_numbers_have_weights_of_their_own(bits, new):
    s = make_step(bits, new, [64], 4, 2, 10, 16, seed=3)
    s.k[0][7, 1, 9] = np.nan
    s.k[0][40, 0, 100] = np.inf
    s.k[0][-1, 0, 0] = np.nan
    alloc = GuardedAllocator()
    p, c, k, _ = whole_cache(s, alloc)
    clean = [np.where(np.isfinite(x), x, 0.0) for x in k]
    lse = log_sums(s, clean, D ** -0.5, 1.0, np.random.default_rng(4))
    weight = torch.full((s.pages, s.Hkv, s.page), GONE, device="cuda")
    B.l2a_cache_weights(p, c, up(s.q, torch.bfloat16), up(s.start), up(np.array(s.cached, np.int32)), up(lse), new[0], 1.0, None, weight)
    want, tol = reference(s, clean, lse, 1.0, None, D ** -0.5)
    got = to_host(weight)
    spoilt = np.zeros(got.shape, bool)
    for t, h in ((7, 1), (40, 0), (len(s.k[0]) - 1, 0)):
        spoilt[s.place(0, t)[0], h, s.place(0, t)[1]] = True
    # (an infinite key: infinite or no scores, weights of 0, infinity or NaN)
    assert np.isnan(got[s.place(0, 7)[0], 1, s.place(0, 7)[1]]) and np.isnan(got[s.place(0, len(s.k[0]) - 1)[0], 0, s.place(0, len(s.k[0]) - 1)[1]])
    near("the others", np.where(spoilt, 0, got), np.where(spoilt, 0, want), tol)


def test_behind_the_attention():
    """With the log-sum-exps that l2a_attn_extend leaves, the weights of a routed token's heads add up to their number.  (Each log-sum-exp is off by up to
    log(1 + 2^-8) + 4e-5 and every weight with it.)"""
    s = make_step(4, [3, 200, 1], [300, 100, 777], 8, 2, 50, 16, f=0.4, seed=5)
    alloc = GuardedAllocator()
    p, c, k, v = whole_cache(s, alloc)
    q, start, pos = up(s.q, torch.bfloat16), up(s.start), up(np.array(s.cached, np.int32))
    lse = torch.empty(s.Hq, s.N, device="cuda")
    O = torch.empty(s.N, s.Hq, D, dtype=torch.bfloat16, device="cuda")
    B.l2a_attn_extend(p, c, q, start, pos, up(s.mask), 200, O, lse_global=lse)
    weight = alloc((s.pages, s.Hkv, s.page)).zero_()
    B.l2a_cache_weights(p, c, q, start, pos, lse, 200, 1.0, None, weight)
    got = to_host(weight)
    for b in range(3):
        routed = (s.mask[0, s.start[b]:s.start[b + 1]] != 0).sum()
        for hk in range(2):
            total = sum(got[s.place(b, t)[0], hk, s.place(b, t)[1]] for t in range(s.cached[b] + s.new[b]))
            assert abs(total - 4 * routed) <= 4 * routed * (2.0 ** -8 + 2e-4), (b, hk, total, routed)


def test_scale_and_max_new():
    s = make_step(16, [6, 40], [33, 64], 4, 1, 10, 16, seed=6)
    check(s, 0.5, scale=0.3)
    check(s, 0.5, max_new=1000)
    # more new tokens than were announced are cut off
    p, c, k, _ = whole_cache(s, GuardedAllocator())
    lse = log_sums(s, k, D ** -0.5, 1.0, np.random.default_rng(5))
    weight = torch.full((s.pages, s.Hkv, s.page), GONE, device="cuda")
    B.l2a_cache_weights(p, c, up(s.q, torch.bfloat16), up(s.start), up(np.array(s.cached, np.int32)), up(lse), 6, 1.0, None, weight)
    s.new = [6, 6]
    want, tol = reference(s, k, lse, 1.0, None, D ** -0.5)
    near("cut off", to_host(weight), want, tol)


@pytest.mark.parametrize("sequences", [1025, 2100])
def test_many_sequences(sequences):
    """More than a workgroup's plan takes at a time."""
    check(make_step(8, [1 + i % 2 for i in range(sequences)], [(7 * i) % 40 for i in range(sequences)], 2, 1, 10, 16, seed=8), 0.8)


@pytest.mark.parametrize("most", [1, 50])
def test_damaged_device_data_stays_inside_the_tensors(most):
    rng = np.random.default_rng(9)
    s = make_step(4, [20, 1, 30], [40, 100, 7], 4, 2, 10, 16, seed=9)
    alloc = GuardedAllocator()
    p, c, _, _ = whole_cache(s, alloc)
    weight = alloc((s.pages, s.Hkv, s.page)).zero_()
    ws = B.alloc_weights_workspace(p, c, most, alloc)
    lse = up(rng.standard_normal((s.Hq, s.N)).astype(np.float32))
    big = np.array([-2 ** 31, -5, -1, 0, 3, 50, 51, 52, 10 ** 6, 2 ** 31 - 1], np.int32)
    for i in range(40):
        c.tensors[4].copy_(up(rng.choice(big, s.table.shape)))
        start, pos = up(rng.choice(big, s.B + 1)), up(rng.choice(big, s.B))
        B.l2a_cache_weights(p, c, up(s.q, torch.bfloat16), start, pos, lse, most, 1.0, weight, weight, ws)
    torch.cuda.synchronize()
    alloc.check()
