"""The operators of long generations together, as a server uses them: rotary positions, a cache in few bits, attention, the weights that rows receive, and
the eviction of those that receive least; captured into graphs, and on several streams."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import PagedCache, to_host
from tests.fp4_helpers import dequantise4, quantise4
from tests.paged_helpers import D, HALF, Step, dequantise, near, quantise, reference, up
from tests.test_gpu_cache_evict import reference as evicted
from tests.test_gpu_rope import frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_steps_of_a_server_with_a_bound(bits):
    Hq, Hkv, W, page, limit = 8, 2, 20, 16, 96
    p = B.make_params(2, 1, Hq, Hkv, D, W)
    cache = PagedCache(p, 16, page, 10, bits == 8, fp4=bits == 4, decay=1.0)
    freq = up(frequencies(64))
    rotary = B.make_rotary(freq, (64,))
    g = torch.Generator(device="cuda").manual_seed(bits)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    held = {16: lambda x: x, 8: lambda x: dequantise(*quantise(x)), 4: lambda x: dequantise4(*quantise4(x))}[bits]
    k, v = ([np.zeros((0, Hkv, D)) for _ in range(2)] for _ in range(2))
    seen, received, given_up = [0, 0], [0, 0], 0
    for i, new in enumerate([[100, 3], [1, 1], [9, 0], [1, 120], [1, 1], [33, 1], [1, 1], [1, 60], [50, 1], "end", [1, 70], [1, 1]]):
        if new == "end":
            cache.end(1)
            k[1], v[1], seen[1] = k[1][:0], v[1][:0], 0
            continue
        cached, N, at = [len(x) for x in k], sum(new), np.cumsum([0] + new)
        pos = cache.positions(new)
        assert pos.cpu().tolist() == [[t + j for t, n in zip(seen, new) for j in range(n)]]
        q, kn, vn = randn(N, Hq, D), randn(N, Hkv, D), randn(N, Hkv, D)
        B.l2a_rope(B.make_params(1, N, Hq, Hkv, D, W), rotary, q, kn, pos, q, kn)
        mask = (torch.rand(1, N, generator=g, device="cuda") < 0.5).to(torch.uint8)
        before = cache.weight.clone()
        O = cache.extend(new, q, kn, vn, mask)
        for have, rows in ((k, to_host(kn)), (v, to_host(vn))):
            for b in range(2):
                have[b] = np.concatenate([have[b], held(rows[at[b]:at[b + 1]])]) if new[b] else have[b]
        s = Step(new, cached, Hq, Hkv, W)
        s.q, s.mask = to_host(q), to_host(mask).reshape(1, -1)
        S, A, tS, tA, _, _ = reference(s, k, v)
        near(f"step {i}", to_host(O), S + A, tS + tA + HALF * (np.abs(S + A) + tS + tA))
        seen = [t + n for t, n in zip(seen, new)]

        def rows_of(pool, b, hk, n):
            return np.array([pool[cache.table[b, j // page], hk, j % page] for j in range(n)], np.float64)
        # every routed token's head hands out one (its log-sum-exp is off by up to log(1 + 2^-8) + 4e-5)
        after, before = to_host(cache.weight), to_host(before)
        for b in range(2):
            routed = int((s.mask[0, at[b]:at[b + 1]] != 0).sum()) * Hq // Hkv
            for hk in range(Hkv):
                gained = rows_of(after, b, hk, len(k[b])).sum() - rows_of(before, b, hk, cached[b]).sum()
                assert abs(gained - routed) <= routed * (2.0 ** -8 + 3e-4) + 1e-3, (i, b, hk)
        if (cache.length > limit).any():
            weights = [[rows_of(after, b, hk, len(k[b])) for hk in range(Hkv)] for b in range(2)]
            gone = cache.evict(limit)
            for b in range(2):
                rows = (len(k[b]) - W) // page * page if gone[b] else 0
                keep = rows - int(gone[b])
                assert len(k[b]) <= limit or (gone[b] % page == 0 and len(k[b]) - gone[b] in range(limit - page + 1, limit + 1))
                for have in (k, v):
                    x = have[b].copy()
                    for hk in range(Hkv):
                        x[:keep, hk] = have[b][evicted(weights[b][hk][:rows], keep), hk]
                    have[b] = np.concatenate([x[:keep], x[rows:]])
            given_up += int(gone.sum())
            assert (cache.length == [len(x) for x in k]).all() and sorted(cache.free + [int(x) for x in cache.table[cache.table >= 0]]) == list(range(16))
        for b in range(2):
            for got, want in zip(cache.read(b), (k[b], v[b])):
                assert np.array_equal(to_host(got), want), (i, b)
    assert given_up >= 200
    with pytest.raises(ValueError, match="window"):
        cache.evict(limit, recent=W - 1)
    with pytest.raises(ValueError, match="no attention weights"):
        PagedCache(p, 16, page, 10).evict(limit)


class Call:
    """A whole step's tensors at fixed addresses, filled anew for every replay."""

    def __init__(self, sequences, new, Hq, Hkv, W, most, bits, pages_each=40, rows=300, workspaces=None):
        self.N, self.most, self.rows_most = sum(new), most, rows
        self.p, self.one = B.make_params(sequences, self.N, Hq, Hkv, D, W), B.make_params(1, self.N, Hq, Hkv, D, W)
        self.c = B.alloc_cache(self.p, sequences * pages_each, 16, pages_each, bits == 8, fp4=bits == 4)
        self.table = torch.randperm(sequences * pages_each, generator=torch.Generator().manual_seed(1)).view(sequences, pages_each)
        self.c.tensors[4].copy_(self.table)
        e = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        self.q, self.k, self.v, self.O = e(self.N, Hq, D), e(self.N, Hkv, D), e(self.N, Hkv, D), e(self.N, Hq, D)
        self.qr, self.kr, self.lse = e(self.N, Hq, D), e(self.N, Hkv, D), e(Hq, self.N, t=torch.float32)
        self.mask, self.tokens = e(1, self.N, t=torch.uint8), e(2, self.N, t=torch.int32)
        self.start = up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        self.pos, self.rows, self.keep = (torch.zeros(sequences, dtype=torch.int32, device="cuda") for _ in range(3))
        shape = (sequences * pages_each, Hkv, 16)
        self.weight = e(*shape, t=torch.float32)
        self.kept = e(sequences, Hkv, rows, t=torch.int32)
        self.freq = up(frequencies(64))
        self.rotary = B.make_rotary(self.freq, (24, 40), adjacent=True)
        self.own = self.workspaces()

    def workspaces(self):
        return (B.alloc_extend_workspace(self.p, self.c, self.most), B.alloc_weights_workspace(self.p, self.c, self.most), B.alloc_evict_workspace(self.p, self.c, self.rows_most))

    def fill(self, i):
        g = torch.Generator(device="cuda").manual_seed(i)
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        for t in self.c.tensors[:2]:  # what is cached: bytes that are numbers in each of the types
            t.view(torch.uint8).copy_(torch.randint(0, 64, t.view(torch.uint8).shape, generator=g, device="cuda"))
        for t in self.c.tensors[2:4]:
            if t is not None:
                t.fill_(126)
        self.mask.copy_(torch.rand(self.mask.shape, generator=g, device="cuda") < 0.6)
        self.tokens.copy_(torch.randint(0, 9000, self.tokens.shape, generator=g, device="cuda"))
        self.pos.copy_(torch.randint(100, 400, self.pos.shape, generator=g, device="cuda"))
        self.rows.copy_(torch.randint(0, self.rows_most + 1, self.rows.shape, generator=g, device="cuda"))
        self.keep.copy_(self.rows // 2 + torch.randint(-40, 40, self.rows.shape, generator=g, device="cuda"))
        self.weight.copy_(torch.rand(self.weight.shape, generator=g, device="cuda"))
        for x in (self.O, self.lse, self.kept):
            x.fill_(7)

    def run(self, workspaces=None):
        extend, weights, evict = self.own if workspaces is None else workspaces
        B.l2a_rope(self.one, self.rotary, self.q, self.k, self.tokens, self.qr, self.kr)
        B.l2a_cache_write(self.p, self.c, self.kr, self.v, self.start, self.pos)
        B.l2a_attn_extend(self.p, self.c, self.qr, self.start, self.pos, self.mask, self.most, self.O, lse_global=self.lse, workspace=extend)
        B.l2a_cache_weights(self.p, self.c, self.qr, self.start, self.pos, self.lse, self.most, 0.75, self.weight, self.weight, weights)
        B.l2a_cache_evict(self.p, self.c, self.rows, self.keep, self.rows_most, self.weight, self.weight, self.kept, evict)

    def outputs(self):
        return [x.view(torch.uint8).clone() for x in (self.O, self.qr, self.kr, self.lse, self.weight, self.kept, *self.c.tensors[:4]) if x is not None]


CALLS = [dict(sequences=5, new=[1] * 5, Hq=16, Hkv=2, W=100, most=2, bits=4), dict(sequences=2, new=[30, 20], Hq=4, Hkv=2, W=60, most=64, bits=8),
         dict(sequences=3, new=[150, 1, 9], Hq=4, Hkv=1, W=100, most=160, bits=4), dict(sequences=140, new=[1] * 140, Hq=8, Hkv=4, W=30, most=4, bits=16)]


@pytest.mark.parametrize("which", range(len(CALLS)))
def test_captured_and_replayed(which):
    a, b = Call(**CALLS[which]), Call(**CALLS[(which + 1) % len(CALLS)])
    # two graphs that share their workspaces and run one after the other
    larger = lambda x, y: y if x is None or (y is not None and y.numel() > x.numel()) else x  # noqa: E731
    a.own = b.own = tuple(larger(x, y) for x, y in zip(a.own, b.own))
    graphs = []
    for c in (a, b):
        c.fill(0)
        c.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run()
    for i in range(1, 5):
        for c, graph in zip((a, b), graphs):
            c.fill(i)
            graph.replay()
            junk = torch.randn(1000, 1000, device="cuda").sum().item()  # eager work and a synchronization in between
            got = c.outputs()
            c.fill(i)
            c.run(c.workspaces())
            torch.cuda.synchronize()
            assert junk == junk and all(torch.equal(x, y) for x, y in zip(got, c.outputs())), f"replay {i}"


def test_calls_on_several_streams_at_once():
    calls = [Call(**c) for c in CALLS]
    wants = []
    for i, c in enumerate(calls):
        c.fill(i)
        c.run()
        wants.append(c.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for i, c in enumerate(calls):
            c.fill(i)
        torch.cuda.synchronize()
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.run()
        torch.cuda.synchronize()
        for c, want in zip(calls, wants):
            assert all(torch.equal(x, y) for x, y in zip(c.outputs(), want))


def test_tensors_that_do_not_fit_are_refused():
    c = Call(**CALLS[1])
    c.fill(0)
    good = dict(p=c.p, c=c.c, q=c.qr, seq_start=c.start, pos=c.pos, lse_global=c.lse, max_new=64, decay=1.0, weight_in=c.weight, weight=c.weight, workspace=c.own[1])
    B.l2a_cache_weights(**good)
    for name, x in [("q", c.q.float()), ("q", c.q[:-1]), ("seq_start", c.start[:-1]), ("pos", c.pos.long()), ("lse_global", c.lse[:, :-1]), ("lse_global", c.lse.double()), ("weight", c.weight[1:]),
                    ("weight", c.weight.cpu()), ("weight_in", c.weight.transpose(0, 1)), ("p", B.make_params(3, c.N, 4, 2, D, 60))]:
        with pytest.raises(ValueError):
            B.l2a_cache_weights(**{**good, name: x})
    good = dict(p=c.p, c=c.c, rows=c.rows, keep=c.keep, max_rows=c.rows_most, weight_in=c.weight, weight=c.weight, kept=c.kept, workspace=c.own[2])
    B.l2a_cache_evict(**good)
    for name, x in [("rows", c.rows.long()), ("keep", c.keep[:-1]), ("weight", c.weight.half()), ("kept", c.kept[..., 1:]), ("max_rows", 200), ("p", B.make_params(2, c.N, 4, 4, D, 60))]:
        with pytest.raises(ValueError):
            B.l2a_cache_evict(**{**good, name: x})
    with pytest.raises(B.L2AError):
        B.l2a_cache_evict(**{**good, "workspace": c.own[2][:16]})
    torch.cuda.synchronize()
