"""What the floating-point experts' calls refuse on the host, before the library or a device sees it (no GPU): tensors of another type, size,
layout or device, experts of several devices."""
import ctypes as C

import pytest
import torch

import paper_2508_09204_b200 as moqe

N, K, M = 64, 128, 6


class OnDevice(torch.Tensor):
    """A CPU tensor that says it is on a device."""
    is_cuda = True
    at = 0

    def get_device(self):
        return self.at


def on(t, device=0):
    t = t.as_subclass(OnDevice)
    t.at = device
    return t


class FakeExpert(moqe.FpExpert):
    def __init__(self):
        self.handle, self.N, self.K, self.format = C.c_void_p(0x1000), N, K, moqe.FP_NVFP4

    def close(self):
        pass


@pytest.fixture
def calls(monkeypatch):
    """The library calls that were reached, by name."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: (seen.append(name), 256 if name.endswith("workspace") else b"" if name.endswith("str") else 0)[1]
    monkeypatch.setattr(moqe, "_lib", Library())
    monkeypatch.setattr(moqe, "_stream", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    return seen


def good():
    return {"X": on(torch.zeros((M, K), dtype=torch.bfloat16)), "rows": on(torch.zeros(M, dtype=torch.int32)), "offsets": on(torch.zeros(3, dtype=torch.int32)),
            "experts": [FakeExpert(), FakeExpert()], "Y": on(torch.zeros((M, N), dtype=torch.bfloat16)), "workspace": on(torch.zeros(256, dtype=torch.uint8))}


def by_ids(a):
    return moqe.moqe_routed_fpgemm(a["X"], a["rows"], a["experts"], Y=a["Y"], workspace=a["workspace"])


def by_sort(a):
    return moqe.moqe_routed_fpgemm_sorted(a["X"], a["rows"], a["offsets"], a["experts"], a["Y"], a["workspace"])


BAD = {
    "X of another type": ("X", lambda t: on(t.float())),
    "X of another K": ("X", lambda t: on(torch.zeros((M, K - 8), dtype=torch.bfloat16))),
    "X flat": ("X", lambda t: on(t.reshape(-1))),
    "X on the host": ("X", lambda t: torch.zeros((M, K), dtype=torch.bfloat16)),
    "X on another device": ("X", lambda t: on(t.clone(), 1)),
    "rows of another type": ("rows", lambda t: on(t.long())),
    "too few rows": ("rows", lambda t: on(t[:-1].clone())),
    "rows on another device": ("rows", lambda t: on(t.clone(), 1)),
    "no experts": ("experts", lambda e: []),
    "Y of another type": ("Y", lambda t: on(t.float())),
    "Y of another N": ("Y", lambda t: on(torch.zeros((M, N - 8), dtype=torch.bfloat16))),
    "Y of too few rows": ("Y", lambda t: on(t[:-1].clone())),
    "Y turned round": ("Y", lambda t: on(torch.zeros((N, M), dtype=torch.bfloat16).t())),
    "Y flat": ("Y", lambda t: on(t.reshape(-1))),
    "Y on the host": ("Y", lambda t: torch.zeros((M, N), dtype=torch.bfloat16)),
    "Y on another device": ("Y", lambda t: on(t.clone(), 1)),
    "a workspace with gaps": ("workspace", lambda t: on(torch.zeros(512, dtype=torch.uint8)[::2])),
    "a workspace on the host": ("workspace", lambda t: torch.zeros(256, dtype=torch.uint8)),
    "a workspace on another device": ("workspace", lambda t: on(t.clone(), 1)),
    "too few offsets": ("offsets", lambda t: on(t[:-1].clone())),
    "offsets of another type": ("offsets", lambda t: on(t.float())),
    "offsets on another device": ("offsets", lambda t: on(t.clone(), 1)),
}


@pytest.mark.parametrize("what", BAD)
@pytest.mark.parametrize("call", [by_ids, by_sort])
def test_refused(calls, what, call):
    name, spoil = BAD[what]
    if name == "offsets" and call is by_ids:
        return
    a = good()
    a[name] = spoil(a[name])
    with pytest.raises((ValueError, moqe.MoqeError)):
        call(a)
    assert not [c for c in calls if not c.endswith(("workspace", "status_str"))]


@pytest.mark.parametrize("call", [by_ids, by_sort])
def test_taken(calls, call):
    a = good()
    assert call(a) is a["Y"] and len([c for c in calls if c.startswith("moqe_routed_fpgemm")]) == 1
    # outputs, places and offsets with more behind them; rows with gaps are copied
    a["Y"] = on(torch.zeros((M + 2, N), dtype=torch.bfloat16))
    a["X"] = on(torch.zeros((M, 2 * K), dtype=torch.bfloat16)[:, ::2])
    call(a)
    if call is by_sort:
        a["rows"], a["offsets"] = on(torch.zeros(M + 5, dtype=torch.int32)), on(torch.zeros(9, dtype=torch.int32))
        call(a)


def test_sources_on_another_device(calls):
    for f in (lambda: moqe.moqe_fp4_quantize_rows(on(torch.zeros((M, K), dtype=torch.bfloat16), 1), moqe.FP_MXFP4),
              lambda: moqe.moqe_fp_quantize(on(torch.zeros((N, K)), 1), moqe.FP_MXFP4),
              lambda: moqe.moqe_fp_expert_import(moqe.FP_BF16, values=on(torch.zeros((N, K), dtype=torch.bfloat16), 1)),
              lambda: moqe.moqe_fp_expert_import(moqe.FP_MXFP4, codes=on(torch.zeros((N, K // 2), dtype=torch.uint8)),
                                                 scales=on(torch.zeros((N, K // 32), dtype=torch.uint8), 1)),
              lambda: moqe.moqe_fp_expert_import(moqe.FP_NVFP4, codes=on(torch.zeros((N, K // 2), dtype=torch.uint8)),
                                                 scales=on(torch.zeros((N, K // 16), dtype=torch.uint8)), outer=on(torch.zeros(N), 1))):
        with pytest.raises(ValueError):
            f()
    assert not calls


class _Expert(C.Structure):
    """The head of the library's struct; what lies behind it is not looked at by the checks."""
    _fields_ = [("N", C.c_int), ("K", C.c_int), ("format", C.c_int), ("Np", C.c_int), ("KB", C.c_int), ("device", C.c_int), ("rest", C.c_uint64 * 8)]


def test_experts_of_two_devices():
    import shutil
    from paper_2508_09204_b200 import build
    if shutil.which("nvcc"):
        build.build()
    L, p = moqe.lib(), 0x10000
    e = [_Expert(N, K, moqe.FP_NVFP4, 128, 1, d) for d in (0, 1)]
    both = (C.c_void_p * 2)(*(C.addressof(x) for x in e))
    assert L.moqe_routed_fpgemm(p, p, M, both, 2, p, p, 1 << 40, None) == moqe.ERR_MISMATCH
    assert L.moqe_routed_fpgemm_sorted(p, p, p, M, both, 2, p, p, 1 << 40, None) == moqe.ERR_MISMATCH
