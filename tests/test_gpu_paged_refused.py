"""runner.PagedCache on the GPU after calls that were refused, and while a graph is captured: the next step is that of a cache that never saw them."""
import pytest
import torch

from paper_2603_17484_amd import binding as B
from paper_2603_17484_amd.runner import PagedCache
from tests.paged_helpers import D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
def test_steps_after_refused_ones(fp8):
    Hq, Hkv = 8, 2
    g = torch.Generator(device="cuda").manual_seed(7)

    def rows(n):
        q, k, v = (torch.randn(n, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
        return q, k, v, (torch.rand(1, n, generator=g, device="cuda") < 0.5).to(torch.uint8)
    p = B.make_params(2, 1, Hq, Hkv, D, 20)
    plain, tried = (PagedCache(p, 24, 16, 12, fp8) for _ in range(2))
    for new in ([40, 3], [2, 1], [0, 0], [30, 17], [1, 1]):
        q, k, v, mask = rows(sum(new))
        if sum(new):
            for bad in ((q, k, v, mask.bool()), (q, k.float(), v, mask), (q[:, :4], k, v, mask)):
                with pytest.raises(ValueError):
                    tried.extend(new, *bad)
            with pytest.raises(B.L2AError):
                tried.extend(new, q, k, v, mask, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                with pytest.raises(RuntimeError, match="captured"):
                    tried.extend(new, q, k, v, mask)
        want, got = plain.extend(new, q, k, v, mask), tried.extend(new, q, k, v, mask)
        assert got.shape == (sum(new), Hq, D) and torch.equal(got.view(torch.int16), want.view(torch.int16))
    for b in range(2):
        assert tried.length[b] == plain.length[b]
        assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(plain.read(b), tried.read(b)))
