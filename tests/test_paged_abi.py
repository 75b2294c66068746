"""Host-side checks of the calls on a paged KV cache (no GPU work): bad arguments become error codes before anything is launched, and
workspaces have the documented sizes."""
import ctypes
import os

import pytest
import torch

from paper_2603_17484_amd import binding as B

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = 0, -1, -2, -3, -4, -5
AT = 1 << 20  # an address that is never followed: every call below is refused


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2603_17484_amd.build import build_lib
        build_lib()
    return B.lib()


def params(**changed):
    p = B.make_params(3, 40, 8, 2, 128, 100)
    for name, x in changed.items():
        setattr(p, name, x)
    return p


def cache(fp8=False, **changed):
    c = B.l2a_cache(AT, AT, AT if fp8 else None, AT if fp8 else None, AT, 10, 16, 7, B.L2A_FP8 if fp8 else B.L2A_BF16)
    for name, x in changed.items():
        setattr(c, name, x)
    return c


def rows(lib, p, c, k=AT, v=AT, start=AT, pos=AT):
    a, b = lib.l2a_cache_write(p, c, k, v, start, pos, None), lib.l2a_cache_read(p, c, start, pos, k, v, None)
    assert a == b
    return a


def extend(lib, p, c, q=AT, start=AT, pos=AT, mask=AT, max_new=9, O=AT, ll=None, lg=None, S=None, A=None, ws=AT, size=None):
    size = lib.l2a_extend_workspace_bytes(p, c, max_new) if size is None else size
    return lib.l2a_attn_extend(p, c, q, start, pos, mask, max_new, O, ll, lg, S, A, ws, size, None)


def ref(x):
    return ctypes.byref(x)


BAD_PARAMS = [(dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(T=-4), SHAPE), (dict(Hq=0), SHAPE), (dict(Hkv=0), SHAPE), (dict(W=-1), SHAPE), (dict(Hkv=3), SHAPE),
              (dict(mask_heads=3), SHAPE), (dict(B=40000), SHAPE), (dict(T=2 ** 24 + 1), SHAPE), (dict(T=2 ** 31 - 1), SHAPE), (dict(softmax_scale=0.0), SHAPE),
              (dict(softmax_scale=float("nan")), SHAPE), (dict(D=64), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(dtype=B.L2A_FP32), UNSUPPORTED), (dict(dtype=B.L2A_FP8), UNSUPPORTED),
              (dict(Hq=34), UNSUPPORTED), (dict(flags=B.L2A_FLAG_SCALAR), UNSUPPORTED), (dict(flags=B.L2A_FLAG_RING_CACHE), UNSUPPORTED),
              (dict(flags=B.L2A_FLAG_RING_CACHE | B.L2A_FLAG_SKIP_GLOBAL), UNSUPPORTED), (dict(flags=B.L2A_FLAG_SKIP_LOCAL | B.L2A_FLAG_SKIP_GLOBAL), UNSUPPORTED)]
BAD_CACHES = [(False, dict(k=None), NULL), (False, dict(v=None), NULL), (False, dict(table=None), NULL), (True, dict(k_scale=None), NULL), (True, dict(v_scale=None), NULL),
              (False, dict(dtype=B.L2A_FP32), UNSUPPORTED), (False, dict(dtype=7), UNSUPPORTED), (False, dict(page_size=0), SHAPE), (False, dict(page_size=-16), SHAPE),
              (False, dict(page_size=8), SHAPE), (False, dict(page_size=48), SHAPE), (False, dict(page_size=2048), SHAPE), (False, dict(pages=0), SHAPE), (False, dict(max_pages=0), SHAPE),
              (False, dict(max_pages=2 ** 20 + 1), SHAPE), (False, dict(max_pages=2 ** 31 - 1, page_size=1024), SHAPE), (False, dict(k=AT + 8), ALIGN), (False, dict(v=AT + 2), ALIGN),
              (True, dict(k_scale=AT + 4), ALIGN), (True, dict(v_scale=AT + 8), ALIGN), (False, dict(table=AT + 2), ALIGN)]


@pytest.mark.parametrize("changed,code", BAD_PARAMS)
def test_sizes_that_are_refused(lib, changed, code):
    p = params(**changed)
    assert rows(lib, ref(p), ref(cache())) == code
    assert extend(lib, ref(p), ref(cache()), size=1 << 30) == code
    assert lib.l2a_extend_workspace_bytes(ref(p), ref(cache()), 9) == 0


@pytest.mark.parametrize("fp8,changed,code", BAD_CACHES)
def test_caches_that_are_refused(lib, fp8, changed, code):
    c = cache(fp8, **changed)
    assert rows(lib, ref(params()), ref(c)) == code
    assert extend(lib, ref(params()), ref(c), size=1 << 30) == code
    assert lib.l2a_extend_workspace_bytes(ref(params()), ref(c), 9) == 0


def test_pointers_that_are_refused(lib):
    p, c = params(), cache()
    assert rows(lib, None, ref(c)) == NULL and rows(lib, ref(p), None) == NULL
    assert extend(lib, None, ref(c), size=1 << 30) == NULL and extend(lib, ref(p), None, size=1 << 30) == NULL
    for name in ("k", "v", "start", "pos"):
        assert rows(lib, ref(p), ref(c), **{name: None}) == NULL
        assert rows(lib, ref(p), ref(c), **{name: AT + 2}) == ALIGN
    for name in ("q", "start", "pos", "mask", "O"):
        assert extend(lib, ref(p), ref(c), **{name: None}) == NULL
    for name in ("q", "O", "S", "A"):
        assert extend(lib, ref(p), ref(c), **{name: AT + 8}) == ALIGN
    for name in ("start", "pos", "ll", "lg"):
        assert extend(lib, ref(p), ref(c), **{name: AT + 2}) == ALIGN
    assert extend(lib, ref(p), ref(c), max_new=0) == SHAPE and extend(lib, ref(p), ref(c), max_new=-1, size=1 << 30) == SHAPE
    need = lib.l2a_extend_workspace_bytes(ref(p), ref(c), 9)
    assert extend(lib, ref(p), ref(c), size=need - 1) == WORKSPACE and extend(lib, ref(p), ref(c), ws=None) == WORKSPACE
    assert extend(lib, ref(p), ref(c), ws=AT + 8) == ALIGN
    dense = params(flags=B.L2A_FLAG_DENSE)  # no decisions needed: refused for the workspace only
    assert extend(lib, ref(dense), ref(c), mask=None, size=0) == WORKSPACE
    local = params(flags=B.L2A_FLAG_SKIP_GLOBAL)
    assert extend(lib, ref(local), ref(c), mask=None, size=0) == WORKSPACE


@pytest.mark.parametrize("T,Hq,Hkv,Bn,max_new", [(1, 1, 1, 1, 1), (64, 28, 4, 64, 1), (64, 28, 4, 64, 5), (80, 32, 8, 16, 18), (2048, 32, 8, 1, 2048), (700, 16, 1, 3, 2 ** 31 - 1)])
def test_workspace_bytes(lib, T, Hq, Hkv, Bn, max_new):
    p = B.make_params(Bn, T, Hq, Hkv, 128, 100)
    G, up = Hq // Hkv, lambda x: (x + 255) // 256 * 256
    most = max_new * G
    few, tile = most <= 128, 32 if most <= 32 else 128 if most <= 128 else 256
    tiles = 2 * Hkv * (T * G // tile + Bn)
    want = 256 + up(64 * tiles) + up(4 * 256) + up(12 * 256) + up(16 * Bn * Hkv) + up(2 * 256 * tile * 132 * 4) + 2 * up(T * Hq * 132 * 4)
    want += up(4 * T) + up(48 * Bn * Hkv) if few else 2 * up(4 * T * Hq)
    assert lib.l2a_extend_workspace_bytes(ref(p), ref(cache()), max_new) == want


def test_tensors_that_are_refused():
    e = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t)  # noqa: E731
    f8 = torch.float8_e4m3fn
    k, table, s = e(4, 2, 16, 128), e(3, 5, t=torch.int32), e(4, 2, 16, 4, t=torch.uint8)
    k8 = e(4, 2, 16, 128, t=f8)
    for tensors in ((k, k, table), (k8, k8, table, s, s)):
        with pytest.raises(ValueError, match="GPU tensors"):  # (and nothing else is wrong with them)
            B.make_cache(*tensors)
    for args in ((k, k[:3], table), (k.float(), k.float(), table), (k, k8, table), (k[0], k[0], table), (k, k, table.long()), (k, k, table[0]), (k8, k8, table),
                 (k8, k8, table, s, s[:2]), (k8, k8, table, s, s.int()), (k, k, table, s, s), (k8, k8, table, s, None)):
        with pytest.raises(ValueError, match="must be|have k_scale"):
            B.make_cache(*args)
