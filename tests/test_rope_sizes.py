"""l2a_rope of heads of 64 channels in bf16, which is a form of its own there: the flag that the attention wants for them is none of its arguments."""
import pytest
import torch

from paper_2603_17484_amd import binding as B
from tests.paged_helpers import near, up
from tests.test_gpu_rope import ANGLE, frequencies, reference
from tests.test_long_abi import lib, rope, rotary  # noqa: F401
from tests.test_paged_abi import ALIGN, AT, SHAPE, UNSUPPORTED, params, ref


def test_heads_of_64_channels_are_no_error(lib):  # noqa: F811
    """(An error that is looked for behind the sizes: nothing is launched.)"""
    for flags in (0, B.L2A_FLAG_SCALAR):
        p = params(D=64, dtype=B.L2A_BF16, flags=flags)
        assert rope(lib, ref(p), ref(rotary(pairs=(20, 12, 0, 0), flags=4))) == UNSUPPORTED
        assert rope(lib, ref(p), ref(rotary(pairs=(20, 12, 0, 0))), q=AT + 8) == ALIGN
        assert rope(lib, ref(p), ref(rotary(pairs=(40, 24, 0, 0)))) == SHAPE  # 64 pairs are 128 channels
    assert rope(lib, ref(params(D=96, dtype=B.L2A_BF16)), ref(rotary())) == UNSUPPORTED
    assert rope(lib, ref(params(D=64, dtype=B.L2A_FP8)), ref(rotary())) == UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("adjacent", [False, True])
def test_heads_of_64_channels(adjacent):
    """Tolerance as in tests/test_gpu_rope.py."""
    import numpy as np
    p = B.make_params(2, 33, 6, 3, 64, 4)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn(2, 33, h, 64, generator=g, device="cuda").bfloat16() for h in (6, 3))
    pos = torch.randint(0, 100000, (2, 66), generator=g, device="cuda").int()
    freq = frequencies(32)
    outs = torch.empty_like(q), torch.empty_like(k)
    B.l2a_rope(p, B.make_rotary(up(freq), (20, 12), adjacent), q, k, pos, *outs)
    for name, x, y in zip("qk", (q, k), outs):
        want, size = reference(x.double().cpu().numpy().reshape(66, -1, 64), pos.cpu().numpy(), freq, (20, 12), adjacent, False)
        tol = size * (ANGLE + 3 * 2.0 ** -24)
        near(name, y.double().cpu().numpy().reshape(want.shape), want, tol + 2.0 ** -8 * (np.abs(want) + tol) * (size > 0))
