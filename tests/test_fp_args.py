"""Refusals of the floating-point experts' entry points: all on the host, before a device is touched (no GPU)."""
import ctypes as C

import pytest

import paper_2508_09204_b200 as moqe

P = 0x10000           # never dereferenced


@pytest.fixture(scope="module")
def L():
    import shutil
    from paper_2508_09204_b200 import build
    if shutil.which("nvcc"):
        build.build()
    return moqe.lib()


def test_quantize_rows(L):
    f = L.moqe_fp4_quantize_rows
    assert f(None, 4, 64, moqe.FP_MXFP4, P, P, None, None, None) == moqe.ERR_NULL
    assert f(P, -1, 64, moqe.FP_MXFP4, P, P, None, None, None) == moqe.ERR_SHAPE
    assert f(P, 4, 0, moqe.FP_MXFP4, P, P, None, None, None) == moqe.ERR_SHAPE
    assert f(P, 4, 60, moqe.FP_MXFP4, P, P, None, None, None) == moqe.ERR_UNSUPPORTED
    for fmt in (0, moqe.FP_BF16, 4, -1):
        assert f(P, 4, 64, fmt, P, P, None, None, None) == moqe.ERR_UNSUPPORTED
    assert f(P + 8, 4, 64, moqe.FP_NVFP4, P, P, P, P, None) == moqe.ERR_UNSUPPORTED
    assert f(P, 4, 64, moqe.FP_NVFP4, P + 4, P, P, P, None) == moqe.ERR_UNSUPPORTED
    assert f(P, 4, 64, moqe.FP_NVFP4, P, P, P + 2, P, None) == moqe.ERR_UNSUPPORTED
    assert f(P, 4, 64, moqe.FP_NVFP4, P, P, P, P + 8, None) == moqe.ERR_UNSUPPORTED
    assert f(None, 0, 64, moqe.FP_NVFP4, None, None, None, None, None) == moqe.OK


def test_experts(L):
    out = C.c_void_p()
    q = L.moqe_fp_quantize
    assert q(None, 8, 64, 1, None, C.byref(out)) == moqe.ERR_NULL
    assert q(P, 8, 64, 1, None, None) == moqe.ERR_NULL
    assert q(P, 0, 64, 1, None, C.byref(out)) == moqe.ERR_SHAPE
    assert q(P, 8, -8, 1, None, C.byref(out)) == moqe.ERR_SHAPE
    assert q(P, 8, 36, 1, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert q(P, 8, 64, 0, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert q(P, 8, 64, 4, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert q(P + 4, 8, 64, 1, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    i = L.moqe_fp_expert_import
    assert i(8, 64, 1, None, P, None, None, None, C.byref(out)) == moqe.ERR_NULL
    assert i(8, 64, 2, P, None, None, None, None, C.byref(out)) == moqe.ERR_NULL
    assert i(8, 64, 3, P, P, None, None, None, C.byref(out)) == moqe.ERR_NULL
    assert i(8, 64, 3, None, None, None, P + 2, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert i(8, 64, 1, P + 2, P, None, None, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert i(8, 64, 9, P, P, None, None, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert i(-8, 64, 1, P, P, None, None, None, C.byref(out)) == moqe.ERR_SHAPE
    assert L.moqe_fp_expert_export(None, None, None, None, None, None) == moqe.ERR_NULL
    assert L.moqe_fp_expert_info(None, None, None, None, None, None, None) == moqe.ERR_NULL
    assert L.moqe_fp_expert_destroy(None) == moqe.ERR_NULL


def test_sizes_beyond_the_indices(L):
    out = C.c_void_p()
    for N, K in ((8, (1 << 24) + 8), (8, (1 << 31) - 8), ((1 << 30) + 1, 64), ((1 << 31) - 1, 64)):
        for fmt in (moqe.FP_MXFP4, moqe.FP_NVFP4, moqe.FP_BF16):
            assert L.moqe_fp_quantize(P, N, K, fmt, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
            assert L.moqe_fp_expert_import(N, K, fmt, P, P, None, P, None, C.byref(out)) == moqe.ERR_UNSUPPORTED
    assert L.moqe_fp4_quantize_rows(P, 1, (1 << 24) + 8, moqe.FP_NVFP4, P, P, P, P, None) == moqe.ERR_UNSUPPORTED


def test_product(L):
    none = (C.c_void_p * 2)(None, None)
    for f in (lambda *a: L.moqe_routed_fpgemm(P, P, *a), lambda *a: L.moqe_routed_fpgemm_sorted(P, P, P, *a)):
        assert f(4, None, 1, P, P, 1 << 30, None) == moqe.ERR_NULL
        assert f(4, none, 1, P, P, 1 << 30, None) == moqe.ERR_NULL
        assert f(4, none, 0, P, P, 1 << 30, None) == moqe.ERR_SHAPE
        assert f(-1, none, 1, P, P, 1 << 30, None) == moqe.ERR_SHAPE
        assert f(4, none, 33, P, P, 1 << 30, None) == moqe.ERR_UNSUPPORTED
    assert L.moqe_routed_fpgemm_workspace(4, none, 1) == 0 and L.moqe_routed_fpgemm_workspace(4, None, 1) == 0
