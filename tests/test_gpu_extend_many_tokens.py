"""Short calls among so many packed tokens that a thread group per row is more than one launch takes: the same bits as without the tokens
that belong to nobody."""
import numpy as np
import pytest
import torch

from paper_2603_17484_amd import binding as B
from tests.paged_helpers import D, SENTINEL, up

pytestmark = pytest.mark.gpu


def test_rows_behind_the_first_launch():
    Hq, Hkv, W, new, cached = 16, 2, 50, [1, 5, 3], [700, 90, 0]
    page, pages_each, n = 16, 50, sum(new)
    N = 2 ** 24 // Hq + 40  # 2^24 rows of 256 threads
    g = torch.Generator(device="cuda").manual_seed(1)
    p = B.make_params(3, n, Hq, Hkv, D, W)
    c = B.alloc_cache(p, 3 * pages_each, page, pages_each)
    for t in c.tensors[:2]:
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    c.tensors[4].copy_(torch.randperm(3 * pages_each, generator=g, device="cuda").view(3, -1))
    q = torch.randn(n, Hq, D, generator=g, device="cuda").bfloat16()
    mask = torch.tensor([[1, 0, 1, 1, 0, 1, 1, 0, 1]], dtype=torch.uint8, device="cuda")
    start, pos = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), up(np.array(cached, np.int32))
    want = torch.empty_like(q)
    B.l2a_attn_extend(p, c, q, up(start), pos, mask, 5, want)
    big = torch.empty(N, Hq, D, dtype=torch.bfloat16, device="cuda")
    decisions = torch.empty(1, N, dtype=torch.uint8, device="cuda")
    O = torch.empty_like(big)
    pb = B.make_params(3, N, Hq, Hkv, D, W)
    workspace = B.alloc_extend_workspace(pb, c, 5)
    for lead in (0, 2 ** 23 // Hq - 4, N - n):  # in the first launch, at its end, behind it
        big[lead:lead + n], decisions[0, lead:lead + n] = q, mask[0]
        O.fill_(SENTINEL)
        B.l2a_attn_extend(pb, c, big, up(start + lead), pos, decisions, 5, O, workspace=workspace)
        assert torch.equal(O[lead:lead + n].view(torch.int16), want.view(torch.int16)), lead
        assert bool((O[:lead] == SENTINEL).all()) and bool((O[lead + n:] == SENTINEL).all())
