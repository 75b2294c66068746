"""Plain 64-bit forms of the operators on a paged KV cache, and one whole comparison with the kernels, for the GPU tests.

Tolerances.  A weight enters the matrix cores rounded to bf16, p (1 + d) with |d| <= 2^-8, and the rounded weights are what the sum is
divided by: s' - s = sum p d (v - s) / sum p (1 + d), at most 2^-8 / (1 - 2^-8) E|v - s| with E the mean under the weights.  For the
row's own weights a routed row's a has its own such bound.  The result is rounded once, 2^-8 of it.  Scores: 128 products summed in
32 bits, exponentials to a few units in the last place of 32 bits: relative 2e-5 of a weight, which moves a mean of v by at most
4e-5 E|v|.  A log-sum-exp is off by the relative error of its sum, log(1 + 2^-8) + 2e-5, and 32-bit rounding.
"""
import numpy as np
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator, to_host

D, BLOCK = 128, 32
HALF = 2.0 ** -8
WEIGHT = HALF / (1 - HALF)
SMALL = 4e-5


def e4m3_values():
    """The value of every e4m3 byte (NaN for 0x7f, 0xff), from its definition."""
    x = np.arange(256)
    s, e, m = x >> 7, x >> 3 & 15, x & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0)) * np.where(s == 1, -1.0, 1.0)
    v[(x & 127) == 127] = np.nan
    return v


E4M3 = e4m3_values()


def block_exponents(x):
    """[..., D] -> [..., D / 32]: the least e with amax <= 448 2^e, clamped; NaN does not count."""
    amax = np.nan_to_num(np.fmax.reduce(np.abs(x.reshape(*x.shape[:-1], -1, BLOCK)), -1))
    e = np.full(amax.shape, -118)
    for up in range(-117, 120):
        e[amax > 448.0 * 2.0 ** (up - 1)] = up
    return e


def quantise(x):
    """[..., D] without infinities -> e4m3 bytes and biased exponents; ties to the even byte."""
    e = block_exponents(x)
    y = x.reshape(*x.shape[:-1], -1, BLOCK) * 2.0 ** -e[..., None].astype(float)
    grid = E4M3[:127]  # ascending
    a = np.abs(y)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - grid[lo], grid[hi] - a
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0))
    code = np.where(np.isnan(y), 127, np.where(up, hi, lo)) | np.where(np.signbit(y), 128, 0)
    return code.astype(np.uint8).reshape(x.shape), (e + 127).astype(np.uint8)


def dequantise(code, exponents):
    v = E4M3[code].reshape(*code.shape[:-1], -1, BLOCK)
    return (v * 2.0 ** (exponents.astype(float) - 127.0)[..., None]).reshape(code.shape)


class Step:
    """A call's inputs on the host: sequences of new[b] tokens behind cached[b], in pages handed out in random order."""

    def __init__(self, new, cached, Hq, Hkv, W, page=16, fp8=False, Hm=1, f=0.3, seed=0, lead=0, tail=0, spare=3, scale=1.0, more_pages=2):
        self.new, self.cached, self.Hq, self.Hkv, self.W, self.page, self.fp8, self.Hm = list(new), list(cached), Hq, Hkv, W, page, fp8, Hm
        self.B, self.N = len(new), lead + sum(new) + tail
        self.start = lead + np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rng = np.random.default_rng(seed)
        normal = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32) * scale).bfloat16().double().numpy()  # noqa: E731
        self.k = [normal(c + n, Hkv, D) for n, c in zip(new, cached)]  # every sequence's rows, cached and new
        self.v = [normal(c + n, Hkv, D) for n, c in zip(new, cached)]
        self.q = normal(self.N, Hq, D)
        self.mask = (rng.random((Hm, self.N)) < f).astype(np.uint8) * 3
        held = [-(-len(x) // page) for x in self.k]
        self.max_pages, self.pages = max(held) + more_pages, sum(held) + spare
        order = rng.permutation(self.pages).astype(np.int32)
        self.table = np.where(rng.random((self.B, self.max_pages)) < 0.5, -1, 2 ** 31 - 1).astype(np.int32)  # entries nobody needs
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n

    def routed(self, token, head, flags=0):
        if flags & B.L2A_FLAG_DENSE:
            return True
        row = 0 if self.Hm == 1 else head if self.Hm == self.Hq else head // (self.Hq // self.Hkv)
        return self.mask[row, token] != 0

    def place(self, b, t):
        return self.table[b, t // self.page], t % self.page

    def params(self, flags=0, scale=None):
        return B.make_params(self.B, self.N, self.Hq, self.Hkv, D, self.W, self.Hm, B.L2A_BF16, flags, scale)

    def pool(self, rows, which, upto=None):
        """Pool bytes with every sequence's rows (of those before `upto`), NaN patterns elsewhere."""
        shape = (self.pages, self.Hkv, self.page)
        x = np.full(shape + (D,), 0xFF if self.fp8 else 0xFFFF, np.uint8 if self.fp8 else np.uint16)
        s = np.full(shape + (D // BLOCK,), 0xFF, np.uint8)
        for b, r in enumerate(rows):
            for t in range(len(r) if upto is None else upto[b]):
                p, at = self.place(b, t)
                if self.fp8:
                    x[p, :, at], s[p, :, at] = which[b][0][t], which[b][1][t]
                else:
                    x[p, :, at] = bits(r[t])
        return x, s

    def held(self, rows):
        """What the cache holds of the rows, in 64 bits: (values, quantised form)."""
        if not self.fp8:
            return rows, [None] * len(rows)
        q = [quantise(r) for r in rows]
        return [dequantise(*x) for x in q], q


def bits(x):
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().view(torch.int16).numpy().view(np.uint16)


def up(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return t.cuda() if dtype is None else t.to(dtype).cuda()


def cache_on_gpu(s, alloc, k, v):
    """k, v: (bytes, exponents) of the pools."""
    p = s.params()
    c = B.alloc_cache(p, s.pages, s.page, s.max_pages, s.fp8, alloc=alloc)
    for t, x in zip(c.tensors[:2], (k, v)):
        t.view(torch.uint8).copy_(up(x[0].view(np.uint8).reshape(*x[0].shape[:-1], -1)))
    if s.fp8:
        c.tensors[2].copy_(up(k[1]))
        c.tensors[3].copy_(up(v[1]))
    c.tensors[4].copy_(up(s.table))
    return p, c


def softmax_part(q, k, v, scale):
    """-> (weighted mean, E|v - mean|, E|v|, log-sum-exp), q [D], k, v [keys, D]."""
    sc = (k @ q) * scale
    m = np.fmax.reduce(sc)
    p = np.exp(sc - m)
    total = p.sum()
    mean = p @ v / total
    return mean, p @ np.abs(v - mean) / total, p @ np.abs(v) / total, m + np.log(total)


def reference(s, k, v, flags=0, scale=None):
    """S, A, their tolerances before the last rounding, log-sum-exps, all over [N, Hq(, D)]; rows of no sequence are NaN."""
    scale = D ** -0.5 if scale is None else scale
    G = s.Hq // s.Hkv
    full = lambda *t: np.full((s.N, s.Hq) + t, np.nan)  # noqa: E731
    S, A, tS, tA, ls, lg = full(D), full(D), full(D), full(D), full(), full()
    for b in range(s.B):
        for i in range(s.new[b]):
            token, t = s.start[b] + i, s.cached[b] + i
            for h in range(s.Hq):
                kb, vb = k[b][:, h // G], v[b][:, h // G]
                S[token, h], tS[token, h], ls[token, h] = 0, 0, -np.inf
                A[token, h], tA[token, h], lg[token, h] = 0, 0, -np.inf
                if not flags & B.L2A_FLAG_SKIP_LOCAL:
                    lo = max(t - s.W, 0)
                    mean, spread, size, lse = softmax_part(s.q[token, h], kb[lo:t + 1], vb[lo:t + 1], scale)
                    S[token, h], tS[token, h], ls[token, h] = mean, WEIGHT * spread + SMALL * size, lse
                if not flags & B.L2A_FLAG_SKIP_GLOBAL and s.routed(token, h, flags):
                    mean, spread, size, lse = softmax_part(s.q[token, h], kb[:t + 1], vb[:t + 1], scale)
                    A[token, h], tA[token, h], lg[token, h] = mean, WEIGHT * spread + SMALL * size, lse
    return S, A, tS, tA, ls, lg


def near(name, got, want, tol):
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want)))  # (infinities and NaN in the same places)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, tolerance {tol[bad][0]}"


SENTINEL = -77.0


def check_extend(s, flags=0, scale=None, max_new=None, optional=True):
    alloc = GuardedAllocator()
    (k, kq), (v, vq) = s.held(s.k), s.held(s.v)
    p, c = cache_on_gpu(s, alloc, s.pool(s.k, kq), s.pool(s.v, vq))
    p = s.params(flags, scale)
    q = s.q.copy()
    used = np.zeros(s.N, bool)
    used[s.start[0]:s.start[-1]] = True
    q[~used] = np.nan
    out = [alloc((s.N, s.Hq, D), torch.bfloat16).fill_(SENTINEL) for _ in range(3)]
    stats = [alloc((s.Hq, s.N)).fill_(SENTINEL) for _ in range(2)]
    max_new = max(max(s.new), 1) if max_new is None else max_new
    ws = B.alloc_extend_workspace(p, c, max_new, alloc).fill_(255)
    mask = None if flags & B.L2A_FLAG_DENSE else up(s.mask)
    more = dict(lse_local=stats[0], lse_global=stats[1], S_opt=out[1], A_opt=out[2]) if optional else {}
    B.l2a_attn_extend(p, c, up(q, torch.bfloat16), up(s.start), up(np.array(s.cached, np.int32)), mask, max_new, out[0], workspace=ws, **more)
    torch.cuda.synchronize()
    alloc.check()
    with np.errstate(invalid="ignore"):
        S, A, tS, tA, ls, lg = reference(s, k, v, flags, scale)
    O, So, Ao = (to_host(t) for t in out)
    outs = [("O", O, S + A, tS + tA)] + ([("S", So, S, tS), ("A", Ao, A, tA)] if optional else [])
    for name, got, want, tol in outs:
        assert (got[~used] == SENTINEL).all(), f"{name}: rows of no sequence were written"
        w = want[used]
        near(name, got[used], w, tol[used] + HALF * (np.abs(w) + tol[used]))
    if optional:
        for name, got, want in (("lse_local", stats[0], ls), ("lse_global", stats[1], lg)):
            got = to_host(got).T
            assert (got[~used] == SENTINEL).all(), f"{name}: rows of no sequence were written"
            w = want[used]
            near(name, got[used], w, np.full(w.shape, WEIGHT + SMALL) + 2.0 ** -22 * np.where(np.isfinite(w), np.abs(w), 0))
    return out, stats
