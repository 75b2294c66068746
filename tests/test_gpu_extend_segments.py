"""Attention of short chunks behind long caches, whose division is mostly segments: a few blocks of every tile are left for the workgroups that
have none (tests/test_extend_segments.py looks at how even that is)."""
import pytest

from tests import test_gpu_paged as paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,cached,Hq,Hkv,W,f,fp8,page", [
    ([128], [65536], 28, 4, 512, 0.2, False, 64), ([128], [32768], 28, 4, 512, 0.5, True, 32), ([313], [17548], 12, 1, 100, 1.0, False, 16),
    ([96], [65536], 28, 4, 64, 0.2, False, 128), ([40], [32768], 32, 8, 0, 1.0, True, 64), ([191, 1, 70], [33548, 9000, 40000], 12, 1, 1024, 1.0, False, 64)])
def test_segments(new, cached, Hq, Hkv, W, f, fp8, page):
    paged.test_long_caches(new, cached, Hq, Hkv, W, f, fp8, page)
