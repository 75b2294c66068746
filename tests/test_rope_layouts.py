"""Which tensors binding.l2a_rope takes, and the strides that it hands on, on the CPU: the library is replaced by one that notes what it was given."""
import ctypes

import pytest
import torch

from paper_2603_17484_amd import binding as B

SIZES = (2, 6, 4, 2, 128)  # B, T, Hq, Hkv, D


@pytest.fixture
def call(monkeypatch):
    """rope(q, k, q_out, k_out, **rotary's fields) -> the fields of the struct that the library was called with."""
    seen = []

    class Library:
        @staticmethod
        def l2a_rope(p, r, *args):
            r = ctypes.cast(r, ctypes.POINTER(B.l2a_rotary)).contents
            seen.append((r.q_stride, r.k_stride, r.q_out_stride, r.k_out_stride, r.axes, list(r.pairs), r.flags, r.freq))
            return 0
    monkeypatch.setattr(B, "lib", lambda: Library)
    monkeypatch.setattr(B, "_ptr", lambda t: t.data_ptr())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # the CPU's number
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    p = B.make_params(*SIZES, 4)
    freq, pos = torch.zeros(64), torch.zeros(2, 12, dtype=torch.int32)

    def rope(q, k, q_out, k_out, **fields):
        r = B.make_rotary(freq, (40, 24), True)
        for name, x in fields.items():
            setattr(r, name, x)
        B.l2a_rope(p, r, q, k, pos, q_out, k_out)
        assert seen[-1][4:] == (2, [40, 24, 0, 0], B.L2A_ROTARY_ADJACENT, freq.data_ptr())
        return seen[-1][:4]
    return rope


def e(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def test_layouts_that_are_taken(call):
    q, k = e(2, 6, 4, 128), e(2, 6, 2, 128)
    fused = e(2, 6, 8 * 128)
    parts = fused[..., :512].unflatten(-1, (4, 128)), fused[..., 512:768].unflatten(-1, (2, 128))
    assert call(q, k, q, k) == (0, 0, 0, 0)
    assert call(q.view(12, 4, 128), k.view(2, 6, 256), q.view(12, 512), k.view(-1)) == (0, 0, 0, 0)
    assert call(*parts, *parts) == (1024,) * 4
    assert call(*parts, q, k) == (1024, 1024, 0, 0)
    # one sequence's heads before the tokens is the same memory only where either is one
    assert B._token_rows(e(2, 4, 1, 128).transpose(1, 2), 2, 1, torch.bfloat16, 4, 128, -1, "q")[1] in (0, 512)


@pytest.mark.parametrize("shape", [(2, 4, 6, 128), (6, 2, 4, 128), (4, 2, 6, 128), (12, 128, 4), (2, 6, 128, 4), (6, 2, 512), (24, 256), (48, 128), (2, 3, 2, 4, 128)])
def test_other_layouts_of_as_many_entries_are_refused(call, shape):
    """Contiguous and of the right size, but not rows of tokens: head-major and sequence-minor tensors would be turned by other tokens' angles."""
    q, k = e(2, 6, 4, 128), e(2, 6, 2, 128)
    bad = e(*shape)
    assert bad.numel() == q.numel()
    for args in ((bad, k, q, k), (q, k, bad, k)):
        with pytest.raises(ValueError, match="must be"):
            call(*args)


def test_strides_follow_the_tensors(call):
    """What the struct says of strides is about C callers' tensors: with it, contiguous tensors would be read and written behind their ends."""
    q, k = e(2, 6, 4, 128), e(2, 6, 2, 128)
    for name in ("q_stride", "k_stride", "q_out_stride", "k_out_stride"):
        assert call(q, k, q, k, **{name: 4096}) == (0, 0, 0, 0)
