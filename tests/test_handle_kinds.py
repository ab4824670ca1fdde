"""Integer, floating-point and parked experts have handles of different layouts: a call that is given one kind for another refuses it on
the host, before the library sees it (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2508_09204_b200 as moqe


def _made(cls, **members):
    """One without the library's help; its handle is never dereferenced."""
    e = cls.__new__(cls)
    e.handle = None                    # (nothing to destroy)
    for k, v in {"N": 64, "K": 64, "bits": 4, "group": 0, "sym": True, "format": moqe.FP_MXFP4, **members}.items():
        setattr(e, k, v)
    return e


@pytest.fixture
def library(monkeypatch):
    """A library in which every call is a mistake."""
    class Untouchable:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError(f"{name} was reached")
            return call
    monkeypatch.setattr(moqe, "_lib", Untouchable())
    monkeypatch.setattr(moqe, "_stream", lambda: 0)
    monkeypatch.setattr(moqe, "_dev", lambda t, dtype, name: t)


INT, FP, HOST = (lambda: _made(moqe.Expert)), (lambda: _made(moqe.FpExpert)), (lambda: _made(moqe.HostExpert))
X, Y = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((4, 64), dtype=torch.bfloat16)
IDS, OFFSETS, WS = torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)


@pytest.mark.parametrize("call", [
    lambda i, f, h: moqe.moqe_routed_fpgemm(X, IDS, [f, i], Y=Y, workspace=WS),
    lambda i, f, h: moqe.moqe_routed_fpgemm(X, IDS, [i]),
    lambda i, f, h: moqe.moqe_routed_fpgemm_sorted(X, IDS, OFFSETS, [i, f], Y, WS),
    lambda i, f, h: moqe.moqe_routed_fpgemm_workspace(4, [f, f, i]),
    lambda i, f, h: moqe.moqe_fp_expert_export(i),
    lambda i, f, h: moqe.moqe_routed_qgemm(X, IDS, [i, f], Y=Y, workspace=WS),
    lambda i, f, h: moqe.moqe_routed_qgemm_kernel(4, [f]),
    lambda i, f, h: moqe.moqe_routed_qgemm_sorted(X, IDS, OFFSETS, [f, i], Y, WS),
    lambda i, f, h: moqe.moqe_routed_qgemm_sorted_gated(X, IDS, OFFSETS, [i], [f], Y, WS),
    lambda i, f, h: moqe.moqe_routed_qgemm_sorted_residual(X, IDS, OFFSETS, [f], Y, Y, WS),
    lambda i, f, h: moqe.moqe_routed_qgemm_sorted_multi([X, X], IDS, OFFSETS, [[i], [f]], [Y, Y], WS),
    lambda i, f, h: moqe.moqe_expert_offload(f),
    lambda i, f, h: moqe.moqe_expert_export(f),
    lambda i, f, h: moqe.moqe_expert_prefetch(i),
    lambda i, f, h: moqe.moqe_expert_host_save(f, "nowhere"),
    lambda i, f, h: moqe.moqe_routed_qgemm_kernel(4, [h]),
])
def test_another_kind_is_refused(library, call):
    with pytest.raises(ValueError, match="expected"):
        call(INT(), FP(), HOST())


def test_handles_of_the_right_kind():
    i, f = INT(), FP()
    closed = list(moqe._handles([i]))                          # (the library's own refusal)
    i.handle, f.handle = C.c_void_p(0x1000), C.c_void_p(0x2000)
    got = list(moqe._handles([i, i])), list(moqe._handles([f], moqe.FpExpert))
    i.handle = f.handle = None
    assert got == ([0x1000] * 2, [0x2000]) and closed == [0]
