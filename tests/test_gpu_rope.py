"""Rotary positions against the formula in 64 bits, and their gradient against the formula's and against differences.

Tolerances.  An angle in turns is off by 2^-52 of itself (two roundings in 64 bits; positions of 31 bits, frequencies up to 1: below 2^-23),
its fraction is rounded to 2^-25 of a turn, times two pi 2.3e-7 in all with the functions' own errors; cosine and sine are off by 4e-7 at most.  A result is two
products and a sum of numbers up to r = sqrt(x^2 + y^2) in 32 bits: 3 2^-24 r more.  bf16: rounded once, 2^-8 of the result.
"""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import GuardedAllocator, to_host
from tests.paged_helpers import near, up

pytestmark = pytest.mark.gpu

ANGLE = 6e-7
SENTINEL = -77.0


def frequencies(n, base=1e6):
    return np.array([base ** (-i / n) for i in range(n)], np.float32)


def reference(x, pos, freq, pairs, adjacent, inverse):
    """x [N, heads, D], pos [axes, N] -> turned, and the length of each element's pair (0 where copied)."""
    n = sum(pairs)
    axis = np.repeat(np.arange(len(pairs)), pairs)
    angle = pos[axis].T.astype(np.float64) * freq.astype(np.float64) * (-1 if inverse else 1)
    first = 2 * np.arange(n) if adjacent else np.arange(n)
    second = first + 1 if adjacent else first + n
    a, b, c, s = x[..., first], x[..., second], np.cos(angle)[:, None], np.sin(angle)[:, None]
    y, r = x.copy(), np.zeros(x.shape)
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    r[..., first] = r[..., second] = np.hypot(a, b)
    return y, r


def check(Bn, T, Hq, Hkv, D=128, dtype="bf16", pairs=(64,), adjacent=False, inverse=False, fused=False, in_place=False, pos=None, which="qk", seed=0):
    kind, t = (B.L2A_BF16, torch.bfloat16) if dtype == "bf16" else (B.L2A_FP32, torch.float32)
    rng = np.random.default_rng(seed)
    N, n = Bn * T, sum(pairs)
    p = B.make_params(Bn, T, Hq, Hkv, D, 4, dtype=kind, flags=B.L2A_FLAG_SCALAR if D == 64 and dtype == "bf16" else 0)
    pos = rng.integers(-3, 200000, (len(pairs), N)).astype(np.int32) if pos is None else pos
    freq = frequencies(n)
    alloc = GuardedAllocator()
    width = (Hq + 2 * Hkv + (1 if fused else 0)) * D if fused else 0
    tensors, outs, wants = [], [], []
    if fused:
        rows = alloc((Bn, T, width), t).copy_(torch.from_numpy(rng.standard_normal((Bn, T, width))))
        tensors = [rows[..., :Hq * D].unflatten(-1, (Hq, D)), rows[..., Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D))]
    else:
        tensors = [alloc((Bn, T, h, D), t).copy_(torch.from_numpy(rng.standard_normal((Bn, T, h, D)))) for h in (Hq, Hkv)]
    for x in tensors:
        wants.append(reference(to_host(x).reshape(N, -1, D), pos, freq, pairs, adjacent, inverse))
        outs.append(x if in_place else alloc((Bn, T, *x.shape[2:]), t).fill_(SENTINEL))
    if fused:
        rest = rows[..., (Hq + Hkv) * D:].clone()
    r = B.make_rotary(up(freq), pairs, adjacent, inverse)
    q, k = (tensors[0] if "q" in which else None), (tensors[1] if "k" in which else None)
    B.l2a_rope(p, r, q, k, up(pos), outs[0] if "q" in which else None, outs[1] if "k" in which else None)
    torch.cuda.synchronize()
    alloc.check()
    for name, out, (want, size) in zip("qk", outs, wants):
        if name not in which:
            assert in_place or bool((out == SENTINEL).all())
            continue
        tol = size * (ANGLE + 3 * 2.0 ** -24)
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol) * (size > 0)
        near(name, to_host(out).reshape(want.shape), want, tol)
    if fused:
        assert torch.equal(rows[..., (Hq + Hkv) * D:], rest)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("Bn,T,Hq,Hkv,pairs", [(1, 1, 1, 1, (64,)), (3, 7, 28, 4, (64,)), (1, 33, 12, 1, (24, 11, 13)), (2, 17, 16, 16, (32,)), (1, 5, 4, 2, (8,)), (5, 1, 32, 8, (1, 0, 3, 36)),
                                               (1, 700, 3, 3, (17, 39))])
def test_turned(Bn, T, Hq, Hkv, pairs, adjacent, dtype):
    check(Bn, T, Hq, Hkv, dtype=dtype, pairs=pairs, adjacent=adjacent, seed=T)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("adjacent,in_place", [(False, False), (True, True), (False, True)])
def test_layouts(dtype, adjacent, in_place):
    """Parts of a fused projection's rows, heads of 64 channels, one tensor of the two."""
    check(2, 9, 8, 2, dtype=dtype, adjacent=adjacent, fused=True, in_place=in_place)
    check(1, 40, 6, 3, 64, dtype, (32,), adjacent, in_place=in_place)
    check(1, 40, 6, 3, 64, dtype, (5, 11), adjacent, True, fused=True, in_place=in_place)
    for which in "qk":
        check(2, 9, 8, 2, dtype=dtype, adjacent=adjacent, which=which, in_place=in_place)


def test_far_positions():
    """Positions of all sizes, beside frequencies up to one: no fraction of the angle is lost."""
    pos = np.array([[0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 131071]], np.int32)
    for adjacent in (False, True):
        check(1, 8, 2, 1, dtype="fp32", pos=pos, adjacent=adjacent)


def test_there_and_back():
    """The gradient is the turn's transpose, the opposite turn: by the formula, by differences of the sum <turned, g> and by turning back."""
    p = B.make_params(1, 50, 3, 1, 128, 4, dtype=B.L2A_FP32)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, dout = (torch.randn(1, 50, 3, 128, generator=g, device="cuda") for _ in range(2))
    pos = torch.randint(0, 5000, (2, 50), generator=g, device="cuda").int()
    for adjacent in (False, True):
        forward, back = (B.make_rotary(up(frequencies(48)), (16, 32), adjacent, inverse) for inverse in (False, True))

        def turn(r, x):
            out = torch.empty_like(x)
            B.l2a_rope(p, r, x, None, pos, out, None)
            return out
        dq = turn(back, dout)
        again = to_host(turn(back, turn(forward, q)))
        near("back", again, to_host(q), 4 * ANGLE * np.full(again.shape, 6.0))
        # the sum is linear in q: differences of any step are the gradient, but for the sum's own roundings
        for i in range(20):
            at = (0, (7 * i) % 50, i % 3, (37 * i) % 128)
            d = torch.zeros_like(q)
            d[at] = 8.0
            hi, lo = ((turn(forward, q + sign * d).double() * dout.double()).sum().item() for sign in (1, -1))
            assert abs((hi - lo) / 16.0 - dq[at].item()) <= 2e-5, (adjacent, at)


def test_refusals():
    p = B.make_params(2, 6, 4, 2, 128, 4)
    e = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    freq, pos = e(64, t=torch.float32), e(1, 12, t=torch.int32)
    r = B.make_rotary(freq, (64,))
    q, k = e(2, 6, 4, 128), e(2, 6, 2, 128)
    B.l2a_rope(p, r, q, k, pos, q, k)
    B.l2a_rope(p, r, q.view(12, 4, 128), k, pos, q, k.view(12, 2, 128))
    wide = e(2, 7, 4, 128)
    for bad in (q.float(), q[:1], q.cpu(), q.transpose(1, 2), e(2, 6, 4, 256)[..., ::2], wide[:, :6], e(2, 6, 8, 128)[:, :, ::2], q[..., :64]):
        with pytest.raises(ValueError):
            B.l2a_rope(p, r, bad, k, pos, q, k)
        with pytest.raises(ValueError):
            B.l2a_rope(p, r, q, k, pos, bad, k)
    for bad in (pos.long(), pos[:, :5], pos.cpu()):
        with pytest.raises(ValueError):
            B.l2a_rope(p, r, q, k, bad, q, k)
    for args in ((freq.double(), (64,)), (freq, (32,)), (freq, (20, 20, 10, 10, 4)), (freq.view(8, 8), (64,)), (freq, ())):
        with pytest.raises(ValueError):
            B.make_rotary(*args)
    for args in ((None, None, None, None), (q, None, None, None), (None, k, q, None)):
        with pytest.raises(B.L2AError):
            B.l2a_rope(p, r, args[0], args[1], pos, args[2], args[3])
    with pytest.raises(B.L2AError):  # 12 pairs: not a multiple of 8
        B.l2a_rope(p, B.make_rotary(freq[:12].contiguous(), (12,)), q, k, pos, q, k)
    with pytest.raises(B.L2AError):  # misaligned
        B.l2a_rope(p, r, e(2 * 6 * 4 * 128 + 4)[4:].view(2, 6, 4, 128), k, pos, q, k)
