"""Plain 64-bit forms of a cache in 4 bits, and calls on one, for the GPU tests (paged_helpers.py has those of the other element types)."""
import numpy as np

from paper_2603_17484_amd import binding as B
from tests import paged_helpers
from tests.paged_helpers import BLOCK, D, Step, up

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def block_exponents4(x):
    """[..., D] -> [..., D / 32]: the least e with amax <= 6 2^e, clamped."""
    amax = np.nan_to_num(np.abs(x.reshape(*x.shape[:-1], -1, BLOCK)), posinf=0.0).max(-1)
    e = np.full(amax.shape, -125)
    for power in range(-124, 126):
        e[amax > 6.0 * 2.0 ** (power - 1)] = power
    return e


def quantise4(x):
    """[..., D] -> bytes [..., D / 2] and biased exponents; ties to the even element; a block with something that is no finite number: exponent 255."""
    e = block_exponents4(x)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    y = np.nan_to_num(blocks, nan=0.0, posinf=0.0, neginf=0.0) * 2.0 ** -e[..., None].astype(float)
    a = np.abs(y)
    hi = np.clip(np.searchsorted(E2M1, a), 0, 7)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - E2M1[lo], E2M1[hi] - a
    code = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo) | np.where(np.signbit(y), 8, 0)
    code = code.astype(np.uint8).reshape(x.shape)
    exponents = np.where(np.isfinite(blocks).all(-1), e + 127, 255).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, exponents


def dequantise4(code, exponents):
    both = np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], D)
    v = (E2M1[both & 7] * np.where(both > 7, -1.0, 1.0)).reshape(*code.shape[:-1], -1, BLOCK)
    scale = np.where(exponents == 255, np.nan, 2.0 ** (exponents.astype(float) - 127.0))
    return (v * scale[..., None]).reshape(both.shape)


class Step4(Step):
    """A Step on a cache in 4 bits."""
    bits = 4

    def pool(self, rows, which, upto=None):
        shape = (self.pages, self.Hkv, self.page)
        x, s = np.full(shape + (D // 2,), 0xFF, np.uint8), np.full(shape + (D // BLOCK,), 0xFF, np.uint8)
        for b, r in enumerate(rows):
            for t in range(len(r) if upto is None else upto[b]):
                p, at = self.place(b, t)
                x[p, :, at], s[p, :, at] = which[b][0][t], which[b][1][t]
        return x, s

    def held(self, rows):
        q = [quantise4(r) for r in rows]
        return [dequantise4(*x) for x in q], q


def make_step(bits, *args, **kw):
    return Step4(*args, **kw) if bits == 4 else Step(*args, fp8=bits == 8, **kw)


def cache_on_gpu(s, alloc, k, v):
    """k, v: (bytes, exponents) of the pools, of any element type."""
    if not isinstance(s, Step4):
        return paged_helpers.cache_on_gpu(s, alloc, k, v)
    p = s.params()
    c = B.alloc_cache(p, s.pages, s.page, s.max_pages, alloc=alloc, fp4=True)
    for t, x in zip(c.tensors[:4], (k[0], v[0], k[1], v[1])):
        t.copy_(up(x))
    c.tensors[4].copy_(up(s.table))
    return p, c


def whole_cache(s, alloc):
    """-> (params, cache with all rows of the sequences, K and V as the cache holds them in 64 bits)."""
    (k, kq), (v, vq) = s.held(s.k), s.held(s.v)
    return (*cache_on_gpu(s, alloc, s.pool(s.k, kq), s.pool(s.v, vq)), k, v)
