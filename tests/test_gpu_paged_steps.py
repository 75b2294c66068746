"""The operators on a paged KV cache as they are used: steps of a server (router, cache write, attention; rows read back, sequences that
end and others that take their pages), captured graphs, several streams, and beside the calls on one sequence's own tensors."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import PagedCache, to_host
from tests.paged_helpers import D, HALF, SMALL, WEIGHT, Step, dequantise, near, quantise, reference, up

pytestmark = pytest.mark.gpu


def step_reference(new, cached, Hq, Hkv, W, q, mask, k, v):
    """O of a step and its tolerance."""
    s = Step(new, cached, Hq, Hkv, W)
    s.q, s.mask = to_host(q), to_host(mask).reshape(1, -1)
    S, A, tS, tA, _, _ = reference(s, k, v)
    tol = tS + tA
    return S + A, tol + HALF * (np.abs(S + A) + tol)


@pytest.mark.parametrize("fp8", [False, True])
def test_steps_of_a_server(fp8):
    Hq, Hkv, W, C, page = 8, 2, 40, 64, 16
    cache = PagedCache(B.make_params(3, 1, Hq, Hkv, D, W), 24, page, 12, fp8)
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    w = torch.randn(C, generator=g, device="cuda")
    k, v = ([np.zeros((0, Hkv, D)) for _ in range(3)] for _ in range(2))
    for i, new in enumerate([[70, 1, 0], [1, 5, 33], [1, 1, 1], [1, 1, 1], "end", [1, 130, 1], [1, 0, 1], [6, 6, 6]]):
        if new == "end":  # sequence 1's pages go to others, later to a sequence that takes its place
            cache.end(1)
            k[1], v[1] = k[1][:0], v[1][:0]
            assert cache.read(1)[0].shape == (0, Hkv, D)
            continue
        cached, N = [len(x) for x in k], sum(new)
        q, kn, vn = randn(N, Hq, D), randn(N, Hkv, D), randn(N, Hkv, D)
        mask = torch.empty(1, 1, N, dtype=torch.uint8, device="cuda")
        B.l2a_router_decide(B.make_params(1, N, Hq, Hkv, D, W), randn(1, N, C), w, 0.0, 0.5, mask)
        O = cache.extend(new, q, kn, vn, mask)
        at = np.cumsum([0] + new)
        for have, rows in ((k, to_host(kn)), (v, to_host(vn))):
            for b in range(3):
                x = rows[at[b]:at[b + 1]]
                have[b] = np.concatenate([have[b], dequantise(*quantise(x)) if fp8 and len(x) else x])
        want, tol = step_reference(new, cached, Hq, Hkv, W, q, mask, k, v)
        near(f"step {i}", to_host(O), want, tol)
    for b in range(3):
        for got, want in zip(cache.read(b), (k[b], v[b])):
            assert np.array_equal(to_host(got), want)
    assert sorted(cache.free + [int(x) for x in cache.table[cache.table >= 0]]) == list(range(24))
    with pytest.raises(ValueError):
        cache.begin_step([200, 0, 0])


def test_beside_the_calls_on_one_sequence():
    """The prompt as one call of l2a_attn_fwd and as three chunks on pages, the next token as l2a_attn_decode and on pages."""
    T, Hq, Hkv, W = 201, 8, 2, 60
    g = torch.Generator(device="cuda").manual_seed(2)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    q, k, v = randn(T, Hq, D), randn(T, Hkv, D), randn(T, Hkv, D)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.4).to(torch.uint8)
    n = T - 1
    p = B.make_params(1, n, Hq, Hkv, D, W)
    row_idx, count, kblk, ws = B.alloc_route(p)
    B.l2a_route_compact(p, mask[:n].contiguous(), row_idx, count, kblk, ws)
    fwd = torch.empty(1, n, Hq, D, dtype=torch.bfloat16, device="cuda")
    ll, lg = (torch.empty(1, Hq, n, device="cuda") for _ in range(2))
    one = [x[None, :n].contiguous() for x in (q, k, v)]
    B.l2a_attn_fwd(p, *one, *one, row_idx, count, kblk, fwd, ll, lg, workspace=B.alloc_fwd_workspace(p))
    pd = B.make_params(1, T, Hq, Hkv, D, W)
    dec = torch.empty(1, Hq, D, dtype=torch.bfloat16, device="cuda")
    B.l2a_attn_decode(pd, q[None, n].contiguous(), k[None], v[None], up(np.array([n], np.int32)), mask[n:].view(1, 1).contiguous(), dec)
    cache = PagedCache(B.make_params(1, 1, Hq, Hkv, D, W), 20, 16, 20)
    ext = torch.cat([cache.extend([m], *(x[a:a + m].contiguous() for x in (q, k, v)), mask[a:a + m].view(1, m).contiguous())
                     for a, m in ((0, 90), (90, 4), (94, 106), (200, 1))])
    want, tol = step_reference([T], [0], Hq, Hkv, W, q, mask, [to_host(k)], [to_host(v)])
    near("pages", to_host(ext), want, tol)
    # The other two divide by the sum of the weights before their rounding: off by 2^-8 E|v|, not E|v - mean|
    S, A = reference_of_sizes(q, mask, k, v, W)
    size = S + A
    tol = (WEIGHT + SMALL) * size + HALF * (np.abs(want) + (WEIGHT + SMALL) * size)
    near("one call", to_host(fwd[0]), want[:n], 2 * tol[:n] + 0 * size[:n])  # (s is rounded before a is added: once more)
    near("decode", to_host(dec), want[n:], tol[n:])


def reference_of_sizes(q, mask, k, v, W):
    s = Step([len(q)], [0], q.shape[1], k.shape[1], W)
    s.q, s.mask = to_host(q), to_host(mask).reshape(1, -1)
    S, A, _, _, _, _ = reference(s, [to_host(k)], [np.abs(to_host(v))])
    return S, A


class Call:
    """A step's tensors at fixed addresses, filled anew for every replay."""

    def __init__(self, sequences, new, Hq, Hkv, W, most, fp8, pages_each=60, workspace=None):
        self.N, self.most, self.sequences = sum(new), most, sequences
        self.p = B.make_params(sequences, self.N, Hq, Hkv, D, W)
        self.c = B.alloc_cache(self.p, sequences * pages_each, 16, pages_each, fp8)
        for t in self.c.tensors[:2]:
            t.view(torch.uint8).zero_()
        for t in self.c.tensors[2:4]:
            if t is not None:
                t.fill_(127)
        self.c.tensors[4].copy_(torch.randperm(sequences * pages_each).view(sequences, pages_each))
        e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.q, self.k, self.v, self.O = e(self.N, Hq, D), e(self.N, Hkv, D), e(self.N, Hkv, D), e(self.N, Hq, D)
        self.mask = torch.empty(1, self.N, dtype=torch.uint8, device="cuda")
        self.start = up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        self.pos = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.workspace = B.alloc_extend_workspace(self.p, self.c, most) if workspace is None else workspace

    def fill(self, i):
        g = torch.Generator(device="cuda").manual_seed(i)
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        self.mask.copy_(torch.rand(self.mask.shape, generator=g, device="cuda") < 0.5)
        self.pos.copy_(torch.randint(0, 500, self.pos.shape, generator=g, device="cuda"))
        cut = torch.randint(0, 4, self.start.shape, generator=g, device="cuda").int()  # other lengths, too
        self.start[1:-1].sub_(0).copy_(torch.maximum(self.start[1:-1] - cut[1:-1], self.start[:-2]))

    def run(self, O=None, workspace=None):
        B.l2a_cache_write(self.p, self.c, self.k, self.v, self.start, self.pos)
        B.l2a_attn_extend(self.p, self.c, self.q, self.start, self.pos, self.mask, self.most, self.O if O is None else O,
                          workspace=self.workspace if workspace is None else workspace)


CALLS = [dict(sequences=5, new=[1] * 5, Hq=16, Hkv=2, W=100, most=8, fp8=False), dict(sequences=2, new=[30, 20], Hq=4, Hkv=2, W=60, most=64, fp8=True),
         dict(sequences=3, new=[150, 1, 9], Hq=4, Hkv=1, W=100, most=160, fp8=False), dict(sequences=140, new=[1] * 140, Hq=8, Hkv=4, W=30, most=4, fp8=True, pages_each=40)]


@pytest.mark.parametrize("which", range(len(CALLS)))
def test_captured_and_replayed(which):
    a = Call(**CALLS[which])
    # another graph, of another kind of call, that shares the workspace; the two run one after the other
    b = Call(**CALLS[(which + 1) % len(CALLS)])
    if b.workspace.numel() > a.workspace.numel():
        a.workspace = b.workspace
    b.workspace = a.workspace
    graphs = []
    for c in (a, b):
        c.fill(0)
        c.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run()
    for i in range(1, 6):
        for c, graph in zip((a, b), graphs):
            c.fill(i)
            c.O.fill_(7)
            graph.replay()
            junk = torch.randn(1000, 1000, device="cuda").sum().item()  # eager work and a synchronization in between
            got = c.O.clone()
            want = torch.full_like(c.O, 7)
            c.run(want, B.alloc_extend_workspace(c.p, c.c, c.most))
            torch.cuda.synchronize()
            assert junk == junk and torch.equal(got.view(torch.int16), want.view(torch.int16)), f"replay {i}"


def test_calls_on_two_streams_at_once():
    calls = [Call(**c) for c in CALLS]
    wants = []
    for i, c in enumerate(calls):
        c.fill(i)
        c.run()
        wants.append(c.O.clone())
        c.O.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c, want in zip(calls, wants):
        assert torch.equal(c.O.view(torch.int16), want.view(torch.int16))


def test_tensors_that_do_not_fit_are_refused():
    c = Call(**CALLS[0])
    c.fill(0)
    good = dict(p=c.p, c=c.c, q=c.q, seq_start=c.start, pos=c.pos, mask=c.mask, max_new=8, O=c.O, workspace=c.workspace)
    B.l2a_attn_extend(**good)
    bad = [("q", c.q.float()), ("q", c.q[:-1]), ("q", c.q.cpu()), ("q", c.q.transpose(0, 1)), ("O", c.O[:, :, :64]), ("seq_start", c.start[:-1]),
           ("seq_start", c.start.long()), ("pos", c.pos.cpu()), ("mask", c.mask.bool()), ("mask", c.mask[:, :-1]), ("workspace", c.workspace.cpu()),
           ("lse_local", torch.empty(3, device="cuda")), ("S_opt", c.O.float()), ("p", B.make_params(4, c.N, 16, 2, D, 100)), ("p", B.make_params(5, c.N, 16, 4, D, 100))]
    for name, x in bad:
        with pytest.raises(ValueError):
            B.l2a_attn_extend(**{**good, name: x})
    for call in (B.l2a_cache_write, lambda p, cc, k, v, s, at: B.l2a_cache_read(p, cc, s, at, k, v)):
        for k, v in ((c.k.float(), c.v), (c.k, c.v[:-1]), (c.k.cpu(), c.v)):
            with pytest.raises(ValueError):
                call(c.p, c.c, k, v, c.start, c.pos)
    with pytest.raises(B.L2AError):
        B.l2a_attn_extend(**{**good, "workspace": c.workspace[:1024]})
    torch.cuda.synchronize()
