"""Floating-point experts and stream captures: builds, imports and destructions in and beside them, and a process whose first calls are
captured ones."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_2508_09204_b200 as moqe
from test_gpu_expert_memory import RELAXED, THREAD_LOCAL, _Capture, _elsewhere, _runtime

pytestmark = pytest.mark.gpu
FORMATS = (moqe.FP_MXFP4, moqe.FP_NVFP4, moqe.FP_BF16)


def _weights(N=264, K=520):
    return torch.randn((N, K), device="cuda", generator=torch.Generator("cuda").manual_seed(N + K))


def _same(a, b):
    return all(p is q or torch.equal(p, q) for p, q in zip(moqe.moqe_fp_expert_export(a, values=True), moqe.moqe_fp_expert_export(b, values=True)))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("mode,same_thread", [(THREAD_LOCAL, False), (RELAXED, False), (RELAXED, True)])
def test_destroy_beside_a_capture(mode, same_thread, fmt):
    e = moqe.moqe_fp_quantize(_weights(), fmt)
    handle, e.handle = e.handle, None
    with _Capture(mode) as c:
        destroy = lambda: moqe.lib().moqe_fp_expert_destroy(handle)
        status = destroy() if same_thread else _elsewhere(destroy)
    assert status == moqe.OK and c.valid


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("what", ["quantize", "import"])
@pytest.mark.parametrize("mode,same_thread", [(THREAD_LOCAL, False), (RELAXED, True)])
def test_building_in_a_capture(mode, same_thread, what, fmt):
    """The expert's memory exists at once, and the graph fills it whenever it runs."""
    W = _weights()
    N, K = W.shape
    e = moqe.moqe_fp_quantize(W, fmt)
    arrays = moqe.moqe_fp_expert_export(e)
    ptr = [None if t is None else t.data_ptr() for t in arrays]
    out = ctypes.c_void_p()
    with _Capture(mode) as c:
        if what == "quantize":
            build = lambda: moqe.lib().moqe_fp_quantize(W.data_ptr(), N, K, fmt, c.handle, ctypes.byref(out))
        else:
            build = lambda: moqe.lib().moqe_fp_expert_import(N, K, fmt, *ptr, c.handle, ctypes.byref(out))
        status = build() if same_thread else _elsewhere(build)
    assert status == moqe.OK and c.valid
    run = ctypes.c_void_p()
    assert _runtime().cudaGraphInstantiate(ctypes.byref(run), c.graph, ctypes.c_ulonglong(0)) == 0
    built = moqe.FpExpert(out.value, N, K, fmt)
    for again in range(2):
        if again and what == "quantize":
            W.mul_(-3.0)
            e = moqe.moqe_fp_quantize(W, fmt)
        torch.cuda.synchronize()
        assert _runtime().cudaGraphLaunch(run, c.handle) == 0
        torch.cuda.synchronize()
        assert _same(built, e)
    _runtime().cudaGraphExecDestroy(run)
    _runtime().cudaGraphDestroy(c.graph)
    built.close()


def test_a_build_that_a_capture_does_not_allow():
    W = _weights()
    out = ctypes.c_void_p(7)
    with _Capture(THREAD_LOCAL) as c:
        status = moqe.lib().moqe_fp_quantize(W.data_ptr(), *W.shape, moqe.FP_NVFP4, c.handle, ctypes.byref(out))
    assert status == moqe.ERR_ALLOC and not c.valid and out.value == 7
    # the next call knows nothing of it
    assert _same(moqe.moqe_fp_quantize(W, moqe.FP_NVFP4), moqe.moqe_fp_quantize(W, moqe.FP_NVFP4))


def test_building_beside_a_capture():
    W = _weights()
    side = torch.cuda.Stream()
    out = ctypes.c_void_p()
    with _Capture(THREAD_LOCAL) as c:
        status = _elsewhere(lambda: moqe.lib().moqe_fp_quantize(W.data_ptr(), *W.shape, moqe.FP_MXFP4, side.cuda_stream, ctypes.byref(out)))
    assert status == moqe.OK and c.valid
    torch.cuda.synchronize()
    assert _same(moqe.FpExpert(out.value, *W.shape, moqe.FP_MXFP4), moqe.moqe_fp_quantize(W, moqe.FP_MXFP4))


_FIRST_CALLS = """
import sys, torch
import paper_2508_09204_b200 as moqe
M, N, K = (int(a) for a in sys.argv[1:4])
g = torch.Generator("cuda").manual_seed(1)
X = torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16)
W = torch.randn((N, K), device="cuda", generator=g) * 0.05
ids = (torch.arange(M, device="cuda") % 3).to(torch.int32)
torch.cuda.synchronize()
experts, out, graph = [], {}, torch.cuda.CUDAGraph()

def step():
    out["rows"] = moqe.moqe_fp4_quantize_rows(X, moqe.FP_NVFP4, values=True)
    out["Y"] = moqe.moqe_routed_fpgemm(X, ids, experts)
    out["export"] = moqe.moqe_fp_expert_export(experts[1], values=True)
    return [t for o in ("rows", "export") for t in out[o]] + [out["Y"]]

with torch.cuda.graph(graph, capture_error_mode="relaxed"):
    experts += [moqe.moqe_fp_quantize(W, f) for f in (moqe.FP_MXFP4, moqe.FP_NVFP4, moqe.FP_BF16)]
    captured = step()
graph.replay()
torch.cuda.synchronize()
want = step()
assert moqe.moqe_async_status() == moqe.OK
assert all(torch.equal(a, b) for a, b in zip(captured, want)), [bool(torch.equal(a, b)) for a, b in zip(captured, want)]
X.mul_(-2.0)
graph.replay()
assert torch.equal(captured[-1], step()[-1]) and moqe.moqe_async_status() == moqe.OK
"""


@pytest.mark.parametrize("M,N,K", [(1, 512, 1024), (40, 1000, 4096), (2400, 2048, 4096)])
def test_the_first_calls_of_a_process_are_captured(M, N, K):
    """Builds, rows, a product by each kernel and an export, with nothing of them run before."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_CALLS, str(M), str(N), str(K)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
