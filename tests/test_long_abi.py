"""Host-side checks of the calls for long generations (no GPU work): a cache in 4 bits, cached rows' weights, eviction, rotary positions.  Bad arguments
become error codes before anything is launched, and workspaces have the documented sizes."""
import ctypes
import os

import pytest
import torch

from paper_2603_17484_amd import binding as B
from tests.test_paged_abi import ALIGN, AT, BAD_CACHES, BAD_PARAMS, NULL, SHAPE, UNSUPPORTED, WORKSPACE, cache, params, ref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2603_17484_amd.build import build_lib
        build_lib()
    return B.lib()


def weights(lib, p, c, q=AT, start=AT, pos=AT, lse=AT, max_new=9, decay=1.0, old=AT, new=AT, ws=AT, size=1 << 40):
    return lib.l2a_cache_weights(p, c, q, start, pos, lse, max_new, decay, old, new, ws, size, None)


def evict(lib, p, c, rows=AT, keep=AT, max_rows=100, old=AT, new=AT, kept=AT, ws=AT, size=1 << 40):
    return lib.l2a_cache_evict(p, c, rows, keep, max_rows, old, new, kept, ws, size, None)


def rotary(**changed):
    r = B.l2a_rotary(2, (ctypes.c_int32 * 4)(40, 24, 0, 0), 0, 0, 0, 0, 0, AT)
    for name, x in changed.items():
        setattr(r, name, (ctypes.c_int32 * 4)(*x) if name == "pairs" else x)
    return r


def rope(lib, p, r, q=AT, k=2 * AT, pos=AT, q_out=3 * AT, k_out=4 * AT):
    return lib.l2a_rope(p, r, q, k, pos, q_out, k_out, None)


@pytest.mark.parametrize("changed,code", BAD_PARAMS)
def test_sizes_that_are_refused(lib, changed, code):
    p = params(**changed)
    assert weights(lib, ref(p), ref(cache())) == code and evict(lib, ref(p), ref(cache())) == code
    assert lib.l2a_weights_workspace_bytes(ref(p), ref(cache()), 9) == 0 and lib.l2a_evict_workspace_bytes(ref(p), ref(cache()), 9) == 0


@pytest.mark.parametrize("fp8,changed,code", BAD_CACHES)
def test_caches_that_are_refused(lib, fp8, changed, code):
    c = cache(fp8, **changed)
    assert weights(lib, ref(params()), ref(c)) == code and evict(lib, ref(params()), ref(c)) == code


@pytest.mark.parametrize("changed,code", [(dict(k_scale=None), NULL), (dict(v_scale=None), NULL), (dict(k_scale=AT + 4), ALIGN), (dict(v_scale=AT + 8), ALIGN), (dict(k=AT + 8), ALIGN),
                                          (dict(dtype=4), UNSUPPORTED)])
def test_caches_in_four_bits_that_are_refused(lib, changed, code):
    c = cache(True, **{"dtype": B.L2A_FP4, **changed})
    p = params()
    assert lib.l2a_cache_write(ref(p), ref(c), AT, AT, AT, AT, None) == code and lib.l2a_cache_read(ref(p), ref(c), AT, AT, AT, AT, None) == code
    assert lib.l2a_attn_extend(ref(p), ref(c), AT, AT, AT, AT, 9, AT, None, None, None, None, AT, 1 << 40, None) == code
    assert weights(lib, ref(p), ref(c)) == code and evict(lib, ref(p), ref(c)) == code


def test_arguments_of_weights_that_are_refused(lib):
    p, c = params(), cache()
    call = lambda **kw: weights(lib, ref(p), ref(c), **kw)  # noqa: E731
    for name in ("q", "start", "pos", "lse", "new"):
        assert call(**{name: None}) == NULL
    for name in ("start", "pos", "lse", "old", "new"):
        assert call(**{name: AT + 2}) == ALIGN
    assert call(q=AT + 8) == ALIGN
    for decay in (-0.1, float("nan"), float("inf")):
        assert call(decay=decay) == SHAPE
    assert call(max_new=0) == SHAPE and call(max_new=-3) == SHAPE
    assert weights(lib, None, ref(c)) == NULL and weights(lib, ref(p), None) == NULL
    need = lib.l2a_weights_workspace_bytes(ref(p), ref(c), 900)
    if need:
        assert call(max_new=900, size=need - 1) == WORKSPACE and call(max_new=900, ws=None) == WORKSPACE and call(max_new=900, ws=AT + 8) == ALIGN


def test_arguments_of_evict_that_are_refused(lib):
    p, c = params(), cache()
    call = lambda **kw: evict(lib, ref(p), ref(c), **kw)  # noqa: E731
    for name in ("rows", "keep", "old", "new"):
        assert call(**{name: None}) == NULL
    for name in ("rows", "keep", "old", "new", "kept"):
        assert call(**{name: AT + 2}) == ALIGN
    for most in (0, -1, 2 ** 24 + 1):
        assert call(max_rows=most) == SHAPE and lib.l2a_evict_workspace_bytes(ref(p), ref(c), most) == 0
    need = lib.l2a_evict_workspace_bytes(ref(p), ref(c), 100)
    assert need > 0 and call(size=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=AT + 8) == ALIGN
    assert evict(lib, None, ref(c)) == NULL and evict(lib, ref(p), None) == NULL


def test_arguments_of_rope_that_are_refused(lib):
    p = params()
    call = lambda r=None, **kw: rope(lib, ref(p), ref(rotary() if r is None else r), **kw)  # noqa: E731
    for kw in (dict(pos=None), dict(q=None, k=None), dict(q_out=None), dict(k_out=None)):
        assert call(**kw) == NULL
    assert rope(lib, None, ref(rotary())) == NULL and rope(lib, ref(p), None) == NULL and call(rotary(freq=None)) == NULL
    for name in ("q", "k", "q_out", "k_out"):
        assert call(**{name: AT + 8}) == ALIGN
    assert call(pos=AT + 2) == ALIGN and call(rotary(freq=AT + 1)) == ALIGN
    for changed in (dict(axes=0), dict(axes=5), dict(axes=-1), dict(pairs=(40, -8, 0, 0)), dict(pairs=(0, 0, 0, 0)), dict(pairs=(40, 25, 0, 0)), dict(pairs=(40, 32, 0, 0)), dict(pairs=(4, 8, 0, 0)),
                    dict(axes=1, pairs=(2 ** 31 - 8, 0, 0, 0)), dict(q_stride=8 * 128 - 8), dict(k_stride=1), dict(q_out_stride=-1024), dict(k_out_stride=2 * 128 + 4)):
        assert call(rotary(**changed)) == SHAPE, changed
    for changed, kw in ((dict(flags=4), {}), (dict(flags=-1), {}), (dict(q_stride=2048), dict(q_out=AT)), (dict(k_out_stride=512), dict(k_out=2 * AT))):
        assert call(rotary(**changed), **kw) == UNSUPPORTED, changed
    assert rope(lib, ref(params(dtype=B.L2A_FP8)), ref(rotary())) == UNSUPPORTED and rope(lib, ref(params(T=0)), ref(rotary())) == SHAPE
    assert rope(lib, ref(params(D=64, dtype=B.L2A_FP32)), ref(rotary())) == SHAPE  # 64 pairs are 128 channels


def test_struct_layout():
    assert ctypes.sizeof(B.l2a_rotary) == 48


def test_tensors_that_are_refused():
    e = lambda *s, t=torch.uint8: torch.empty(*s, dtype=t)  # noqa: E731
    k, table, s = e(4, 2, 16, 64), e(3, 5, t=torch.int32), e(4, 2, 16, 4)
    with pytest.raises(ValueError, match="GPU tensors"):  # (and nothing else is wrong with them)
        B.make_cache(k, k, table, s, s)
    for args in ((k, k, table), (k, k, table, s, None), (k, k, table, s, s[:2]), (k, e(4, 2, 16, 128), table, s, s), (k, k.to(torch.bfloat16), table, s, s), (k, k, table, e(4, 2, 16, 2), s)):
        with pytest.raises(ValueError, match="must be|have k_scale"):
            B.make_cache(*args)
    with pytest.raises(ValueError, match="8 bits or 4"):
        B.alloc_cache(params(), 4, 16, 3, True, device="cpu", fp4=True)
