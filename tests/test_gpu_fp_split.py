"""Tiles of the floating-point experts' product that workers share along k: whoever comes last reads what the others have parked, with
all of its lanes.  Sums are exact, so that every repeat has to give the definition's bits."""
import numpy as np
import pytest
import torch

import paper_2508_09204_b200 as moqe
from fp_exact import exact_product, on_grid
from test_gpu_fp_gemm import BF, MX, NV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,formats", [
    (16, 136, 16384, [MX]),                                # two tiles, many workers to each
    (40, 1000, 8200, [NV, BF]),                            # eight tiles of either kind, shares that end inside of them
    (128, 264, 11008, [BF, MX, NV]),
    (600, 4096, 8192, [NV, BF]),                           # pairs of SMs
])
def test_shared_tiles_repeat_exactly(M, N, K, formats):
    g = np.random.default_rng(M + K)
    E = len(formats)
    X = torch.from_numpy(on_grid(g, M, K)).cuda().to(torch.bfloat16)
    W = [torch.from_numpy(on_grid(g, N, K)).cuda() for _ in formats]
    ids = torch.arange(M, device="cuda", dtype=torch.int32) % E
    want = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        want[ids == e] = exact_product(X[ids == e], W[e])
    experts = [moqe.moqe_fp_quantize(w, f) for w, f in zip(W, formats)]
    _, perm, offsets = moqe.moqe_permute(None, ids, E)
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, experts))
    outs = [torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(25)]
    ws.fill_(255)                                          # parked sums that nobody has written are NaN
    for Y in outs:
        moqe.moqe_routed_fpgemm_sorted(X, perm, offsets, experts, Y, ws)
    assert moqe.moqe_async_status() == moqe.OK
    assert all(torch.equal(Y, want) for Y in outs)
