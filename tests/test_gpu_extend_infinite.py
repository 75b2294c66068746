"""An infinity among the values that all rows of a tile see is an infinity in their results, wherever the division of work cuts the tile."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import to_host
from tests.paged_helpers import D, HALF, SMALL, WEIGHT, near, up
from tests.test_gpu_paged import on_the_gpu

pytestmark = pytest.mark.gpu


# pieces of two blocks; segments, and what they leave; a tile of up to 128 rows beside one of more, and one of few
@pytest.mark.parametrize("new,cached,Hq,W", [(140, 6000, 2, 30), (300, 40000, 8, 100), (45, 30000, 8, 50), (9, 9000, 8, 50)])
@pytest.mark.parametrize("half", [0, 32])
def test_an_infinity_that_every_row_sees(new, cached, Hq, W, half):
    g = torch.Generator(device="cuda").manual_seed(new)
    page, keys = 64, cached + new
    pages = -(-keys // page)
    p = B.make_params(1, new, Hq, 1, D, W)
    c = B.alloc_cache(p, pages, page, pages)
    c.tensors[4][0] = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int32)
    order = c.tensors[4][0].long()
    k, v = (torch.randn(pages * page, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    spoilt, key = v.clone(), torch.arange(pages * page, device="cuda")
    seen = (key < cached - W) & (key % 64 // 32 * 32 == half)  # by every row's Global attention, out of every row's window
    spoilt[seen, 5] = torch.inf
    spoilt[seen & (key // 64 % 7 == 3), 70] = -torch.inf
    for pool, x in zip(c.tensors, (k, spoilt)):
        pool[order, 0] = x.view(pages, page, D)
    q = torch.randn(new, Hq, D, generator=g, device="cuda").bfloat16()
    mask = torch.ones(1, new, dtype=torch.uint8, device="cuda")
    O, S, A = (torch.empty_like(q) for _ in range(3))
    B.l2a_attn_extend(p, c, q, up(np.array([0, new], np.int32)), up(np.array([cached], np.int32)), mask, new, O, S_opt=S, A_opt=A)
    hi = (cached + torch.arange(new, device="cuda")).repeat_interleave(Hq)
    args = q.double().flatten(0, 1), k[:keys].double(), v[:keys].double()
    s, ds, es, _ = on_the_gpu(*args, hi - W, hi, D ** -0.5)
    a, da, ea, _ = on_the_gpu(*args, torch.zeros_like(hi), hi, D ** -0.5)
    a[:, 5], a[:, 70] = torch.inf, -torch.inf
    for name, got, want, tol in (("S", S, s, WEIGHT * ds + SMALL * es), ("A", A, a, WEIGHT * da + SMALL * ea), ("O", O, s + a, WEIGHT * (ds + da) + SMALL * (es + ea))):
        tol = tol + HALF * (want.nan_to_num(posinf=0, neginf=0).abs() + tol)
        near(name, to_host(got.flatten(0, 1)), want.cpu().numpy(), tol.cpu().numpy())
