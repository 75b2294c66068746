"""The operators of long generations at the sizes where their work is shared out and their places pass 32 bits, and rotary positions in a training step."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator, Layer, to_host
from tests.fp4_helpers import Step4, cache_on_gpu, dequantise4, quantise4, whole_cache
from tests.paged_helpers import D, near, up
from tests.test_gpu_cache_evict import reference as evicted
from tests.test_gpu_rope import frequencies, reference as turned

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24


def test_a_pool_in_four_bits_beyond_four_gigabytes():
    """Pages at the end of pools of 4.3 GB each: 64-bit places throughout."""
    page, Hkv = 1024, 8
    s = Step4([40, 1], [1500, 2047], 16, Hkv, 300, page, f=0.5, seed=12)
    far = 2 ** 32 // (page * Hkv * 64) + 40
    p = s.params()
    c = B.alloc_cache(p, far, page, s.max_pages, fp4=True)
    assert c.tensors[0].numel() > 2 ** 32
    for t in c.tensors[:4]:
        t[far - s.pages:].zero_()
    move = lambda table: np.where((table >= 0) & (table < s.pages), table + far - s.pages, table).astype(np.int32)  # noqa: E731
    c.tensors[4].copy_(up(move(s.table)))
    start, pos = up(s.start), up(np.array(s.cached, np.int32))
    full = [up(np.concatenate([np.zeros((0, Hkv, D))] + x), torch.bfloat16) for x in (s.k, s.v)]
    lens = np.array([len(x) for x in s.k])
    pw = B.make_params(s.B, int(lens.sum()), 16, Hkv, D, 300)
    all_start, zero = up(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)), torch.zeros(s.B, dtype=torch.int32, device="cuda")
    B.l2a_cache_write(pw, c, *full, all_start, zero)
    back = [torch.empty_like(x) for x in full]
    B.l2a_cache_read(pw, c, all_start, zero, *back)
    for got, rows in zip(back, (s.k, s.v)):
        assert np.array_equal(to_host(got), np.concatenate([dequantise4(*quantise4(x)) for x in rows]))
    # the others beside a small pool with the same rows
    alloc = GuardedAllocator()
    (k, kq), (v, vq) = s.held(s.k), s.held(s.v)
    _, near_c = cache_on_gpu(s, alloc, s.pool(s.k, kq), s.pool(s.v, vq))
    q, mask = up(s.q, torch.bfloat16), up(s.mask)
    rows, keep = up(np.array([1024, 2000], np.int32)), up(np.array([300, 1700], np.int32))
    outs = []
    for cache, first in ((c, far - s.pages), (near_c, 0)):
        O, lse = torch.empty(s.N, 16, D, dtype=torch.bfloat16, device="cuda"), torch.empty(16, s.N, device="cuda")
        B.l2a_attn_extend(p, cache, q, start, pos, mask, 40, O, lse_global=lse)
        weight = torch.zeros(cache.pages, Hkv, page, device="cuda")
        B.l2a_cache_weights(p, cache, q, start, pos, lse, 40, 1.0, None, weight)
        kept = torch.zeros(2, Hkv, 2000, dtype=torch.int32, device="cuda")
        B.l2a_cache_evict(p, cache, rows, keep, 2000, weight, weight, kept)
        used, at = (torch.tensor([s.place(b, t)[i] for b, n in enumerate(lens) for t in range(n)]) for i in range(2))  # (rows of nobody differ)
        outs.append([O, lse, kept] + [t[first + used, :, at] for t in (weight, *cache.tensors[:4])])
        assert weight[:first].count_nonzero() == 0
    assert all(torch.equal(x, y) for x, y in zip(*outs))


@pytest.mark.parametrize("new,cached,Hq,Hkv,f,dtype", [
    ([700, 1, 1, 40], [9000, 30000, 511, 3000], 28, 4, 0.5, "fp4"), ([3000], [0], 12, 1, 1.0, "bf16"), ([1, 2000, 1], [70000, 5000, 300], 8, 2, 0.2, "fp8"),
    ([1] * 60, [37 * i * i % 20000 for i in range(60)], 32, 8, 0.7, "bf16"), ([5] * 30, [911 * i % 15000 for i in range(30)], 16, 16, 1.0, "fp8"), ([9] * 200, [100 + i for i in range(200)], 64, 8, 0.9, "fp4"),
    ([1500], [40000], 28, 4, 0.003, "bf16"), ([64] * 20, [256 * i for i in range(20)], 8, 8, 0.5, "fp4"),
    ([1] * 60, [37 * i * i % 20000 for i in range(60)], 32, 8, 0.7, "fp4"), ([4, 2, 1] * 10, [911 * i % 15000 for i in range(30)], 32, 8, 0.8, "fp4"), ([1] * 40, [701 * i % 18000 for i in range(40)], 16, 1, 0.9, "fp8"),
    ([5] * 30, [911 * i % 15000 for i in range(30)], 32, 8, 0.9, "fp4"), ([7] * 20, [911 * i % 15000 for i in range(20)], 32, 8, 0.9, "fp8")])
def test_weights_of_long_caches(new, cached, Hq, Hkv, f, dtype):
    """Against the formula in 64 bits on the GPU; log-sum-exps of random numbers' size (weights are then below 2^10 / keys)."""
    page, scale, G = 64, D ** -0.5, Hq // Hkv
    g = torch.Generator(device="cuda").manual_seed(len(new) + Hq)
    N, nseq = sum(new), len(new)
    held = [-(-(n + c) // page) for n, c in zip(new, cached)]
    p = B.make_params(nseq, N, Hq, Hkv, D, 10)
    c = B.alloc_cache(p, sum(held), page, max(held), dtype == "fp8", fp4=dtype == "fp4")
    table = torch.zeros(nseq, max(held), dtype=torch.int32)
    order, at = torch.randperm(sum(held), generator=torch.Generator().manual_seed(1)).int(), 0
    for b, n in enumerate(held):
        table[b, :n], at = order[at:at + n], at + n
    c.tensors[4].copy_(table)
    lens = [n + x for n, x in zip(new, cached)]
    k = torch.randn(sum(lens), Hkv, D, generator=g, device="cuda").bfloat16()
    begins = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    pw, zero = B.make_params(nseq, sum(lens), Hq, Hkv, D, 10), torch.zeros(nseq, dtype=torch.int32, device="cuda")
    B.l2a_cache_write(pw, c, k, k, up(begins), zero)
    B.l2a_cache_read(pw, c, up(begins), zero, k, torch.empty_like(k))  # as the cache holds it
    q = torch.randn(N, Hq, D, generator=g, device="cuda").bfloat16()
    first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    keys = torch.cat([x + 1.0 + torch.arange(n, device="cuda") for n, x in zip(new, cached)])
    lse = keys.log() + 0.5 + 0.1 * torch.randn(Hq, N, generator=g, device="cuda")
    lse[torch.rand(1, N, generator=g, device="cuda").expand(Hq, N) >= f] = -np.inf
    old = torch.rand(sum(held), Hkv, page, generator=g, device="cuda")
    weight = torch.full_like(old, -77.0)
    B.l2a_cache_weights(p, c, q, up(first), up(np.array(cached, np.int32)), lse, max(new), 0.5, old, weight)
    for b in range(nseq):
        t = torch.arange(new[b], device="cuda") + cached[b]
        key = torch.arange(lens[b], device="cuda")
        pages = table[b, :held[b]].long().cuda()
        got, was = (x[pages].transpose(0, 1).flatten(1)[:, :lens[b]].double() for x in (weight, old))
        for hk in range(Hkv):
            kb = k[begins[b]:begins[b + 1], hk].double()
            want = torch.where(key < cached[b], 0.5 * was[hk], 0.0)
            tol = 2 * ULP * want
            for h in range(hk * G, hk * G + G):
                ls = lse[h, first[b]:first[b + 1]].double()
                on = torch.isfinite(ls)
                qb, ls = q[first[b]:first[b + 1], h][on].double(), ls[on][:, None]
                x = qb @ kb.t() * scale
                e = torch.where(key <= t[on][:, None], torch.exp(x - ls), 0.0)
                want += e.sum(0)
                # (see test_gpu_cache_weights.py; sum |q k| scale is no larger than the products of the lengths)
                size = qb.norm(dim=1, keepdim=True) * kb.norm(dim=1) * scale
                tol += ULP * ((e * (128 * size + 6 * (x.abs() + ls.abs()) + 8)).sum(0) + int(on.sum()) * G * e.sum(0))
            assert bool(((got[hk] - want).abs() <= tol + 2 * ULP * want).all()), (b, hk, float(((got[hk] - want).abs() - tol).max()))
        rest = weight[pages].transpose(0, 1).flatten(1)[:, lens[b]:]
        assert bool((rest == -77.0).all())


def test_evictions_of_many_sequences_of_all_lengths():
    """Some with fewer rows than a workgroup takes, some with several times as many, in one call; some that give nothing up."""
    lengths = [10, 20000, 8192, 8193, 17, 30000, 16384, 9000]
    rows, keep = [10, 19999, 8192, 8193, 0, 100, 16384, 9000], [3, 7000, 8192, 8192, 0, 50, 0, 4500]
    s = Step4([0] * 8, lengths, 1, 1, 4, 256, seed=3, tail=1)
    alloc = GuardedAllocator()
    p, c, _, _ = whole_cache(s, alloc)
    w = np.round(np.random.default_rng(4).exponential(size=(s.pages, 1, s.page)), 2).astype(np.float32)  # with ties
    weight, kept = alloc(w.shape).copy_(up(w)), alloc((8, 1, 20000), torch.int32).fill_(-9)
    B.l2a_cache_evict(p, c, up(np.array(rows, np.int32)), up(np.array(keep, np.int32)), 20000, weight, weight, kept)
    torch.cuda.synchronize()
    alloc.check()
    for b in range(8):
        mine = np.array([w[s.place(b, j)[0], 0, s.place(b, j)[1]] for j in range(rows[b])])
        source = evicted(mine, keep[b])
        assert kept[b, 0, :keep[b]].tolist() == source and bool((kept[b, 0, keep[b]:] == -9).all()), b


def test_more_tokens_than_a_launch_takes():
    """Rotations of 2^26 tokens and more: several launches, places beyond 32 bits."""
    T = 2 ** 26 + 2 ** 23 + 5
    p = B.make_params(1, T, 1, 1, 64, 4, dtype=B.L2A_BF16, flags=B.L2A_FLAG_SCALAR)
    k = torch.empty(1, T, 1, 64, dtype=torch.bfloat16, device="cuda")
    ends = [slice(0, 300), slice(2 ** 26 - 150, 2 ** 26 + 150), slice(T - 300, T)]
    g = torch.Generator(device="cuda").manual_seed(1)
    k.fill_(1.0)
    for e in ends:
        k[:, e] = torch.randn(1, 300, 1, 64, generator=g, device="cuda").bfloat16()
    before = [to_host(k[0, e]) for e in ends]
    pos = torch.arange(T, device="cuda", dtype=torch.int32).view(1, T)
    freq = frequencies(32)
    B.l2a_rope(p, B.make_rotary(up(freq), (32,)), None, k, pos, None, k)
    for e, x in zip(ends, before):
        want, size = turned(x, np.arange(T)[e][None], freq, (32,), False, False)
        tol = size * 1e-6
        near(str(e), to_host(k[0, e]), want, tol + 2.0 ** -8 * (np.abs(want) + tol))


@pytest.mark.parametrize("adjacent", [False, True])
def test_a_training_step_with_rotary_positions(adjacent):
    """Queries and keys turned, the layer forward and backward, their gradients turned back: against 64-bit autograd of the whole, within the 1e-4 of the layer's
    fp32 results."""
    T, Hq, Hkv, W, n = 50, 4, 2, 12, 48
    g = torch.Generator().manual_seed(5)
    q, k, v, dO = (torch.randn(1, T, h, 128, generator=g, dtype=torch.float64).float().double() for h in (Hq, Hkv, Hkv, Hq))
    mask = torch.rand(1, 1, T, generator=g) < 0.4
    pos = torch.stack([torch.arange(T), torch.arange(T) % 7])
    freq = torch.from_numpy(frequencies(n, 1e4))

    def turn(x):
        angle = pos[torch.tensor([0] * 20 + [1] * 28)].t().double() * freq.double()
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if adjacent else (x[..., :n], x[..., n:2 * n])
        both = (a * c - b * s, b * c + a * s)
        y = torch.stack(both, -1).flatten(-2) if adjacent else torch.cat(both, -1)
        return torch.cat([y, x[..., 2 * n:]], -1)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    qt, kt = turn(leaves[0]), turn(leaves[1])
    scores = torch.stack([qt[0, :, h] @ kt[0, :, h // 2].t() for h in range(Hq)]) * 128 ** -0.5
    t, j = torch.arange(T)[:, None], torch.arange(T)
    parts = [torch.softmax(scores.masked_fill(~keep, -np.inf), -1) for keep in ((j <= t) & (j >= t - W), j <= t)]
    p = parts[0] + parts[1] * mask[0, 0][:, None]
    O = torch.stack([p[h] @ leaves[2][0, :, h // 2] for h in range(Hq)], 1)[None]
    (O * dO).sum().backward()

    par = B.make_params(1, T, Hq, Hkv, 128, W, 1, B.L2A_FP32)
    gpu = [x.float().cuda() for x in (q, k, v)]
    turned_ = [torch.empty_like(x) for x in gpu[:2]]
    where = pos.int().cuda()
    forward, back = (B.make_rotary(freq.cuda(), (20, 28), adjacent, inverse) for inverse in (False, True))
    B.l2a_rope(par, forward, gpu[0], gpu[1], where, *turned_)
    layer = Layer(par, *turned_, gpu[2], mask.to(torch.uint8).cuda())
    layer.route()
    layer.forward()
    layer.backward(dO.float().cuda())
    B.l2a_rope(par, back, layer.dq, layer.dk, where, layer.dq, layer.dk)
    for name, got, want in (("O", layer.O, O), ("dq", layer.dq, leaves[0].grad), ("dk", layer.dk, leaves[1].grad), ("dv", layer.dv, leaves[2].grad)):
        near(name, to_host(got), want.detach().numpy(), np.full(want.shape, 1e-4))
