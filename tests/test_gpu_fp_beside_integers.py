"""Integer and floating-point experts on memory that both use as their workspace: the integer product's has to be cleared in between."""
import numpy as np
import pytest
import torch

import paper_2508_09204_b200 as moqe
from test_gpu_fp_gemm import BF, MX, NV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [4, 24, 40, 300])
def test_one_workspace_cleared_in_between(M):
    g = torch.Generator("cuda").manual_seed(M)
    N, K = 1024, 2048
    W = torch.randn((N, K), device="cuda", generator=g) * 0.02
    ints = [moqe.moqe_quantize_rtn(W, 8, 0, True), moqe.moqe_quantize_rtn(W, 4, 128, False)]
    floats = [moqe.moqe_fp_quantize(W, f) for f in (MX, NV, BF)]
    X = torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16)
    ids = torch.from_numpy(np.random.default_rng(M).integers(0, 5, M).astype(np.int32)).cuda()
    _, perm, offsets = moqe.moqe_permute(None, ids, 5)
    sizes = moqe.moqe_routed_qgemm_workspace(M, N, K, 2), moqe.moqe_routed_fpgemm_workspace(M, floats)
    apart = [moqe.alloc_workspace(n) for n in sizes]
    want = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    moqe.moqe_routed_qgemm_workspace_clear(apart[0], M, N, K, 2)
    moqe.moqe_routed_qgemm_sorted(X, perm, offsets, ints, want, apart[0])
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[2:], floats, want, apart[1])
    both = moqe.alloc_workspace(max(sizes))
    for _ in range(5):
        Y = torch.full_like(want, float("nan"))
        moqe.moqe_routed_qgemm_workspace_clear(both, M, N, K, 2)
        moqe.moqe_routed_qgemm_sorted(X, perm, offsets, ints, Y, both)
        moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[2:], floats, Y, both)
        assert torch.equal(Y, want)
    assert moqe.moqe_async_status() == moqe.OK
