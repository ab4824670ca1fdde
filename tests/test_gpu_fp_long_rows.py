"""Long rows, to the bit: a part of a row that goes missing is a small part of its sum of magnitudes, but not of an exact sum, and all of
it where the rest of the row is zeros.  Every k-block, both sides of the row kernels' limits, short last blocks."""
import numpy as np
import pytest
import torch

import paper_2508_09204_b200 as moqe
from fp_exact import exact_product, on_grid
from test_gpu_fp_gemm import BF, MX, NV

pytestmark = pytest.mark.gpu


def _windows(M, K, parts):
    """[M][K]: where row m is not zero.  Row m mod len(parts) has parts[...] = (first k, number of k)."""
    at = np.zeros((M, K), bool)
    for m in range(M):
        k, n = parts[m % len(parts)]
        at[m, k:k + n] = True
    return at


def _seams(K):
    """The first and the last k, what is left behind whole blocks of 16, 32, 64 and 256 k, and both sides of every multiple of 256 x a power of
    two: among them what a thread, a warp, a block of threads and a stage of the ring hold."""
    out = [(0, 8), (K - 8, 8)]
    for b in (16, 32, 64, 256):
        if K % b and K // b:
            out += [(K // b * b, K % b), (K // b * b - 8, 8)]
    b = 256
    while b < K:
        for k in range(b, K, b if b >= 4096 else K):
            out += [(k - 8, 16), (k, 8)]
        b *= 2
    for k in (3 * 8192, 3 * 4096, 1536 * 16):
        if k + 8 <= K:
            out += [(k - 8, 16)]
    return [(k, min(n, K - k)) for k, n in out]


def _run(fmt, x, w, chunk=None):
    """Rows x by one expert w, in calls of `chunk` rows."""
    X, W = (torch.from_numpy(a).cuda() for a in (x, w))
    X = X.to(torch.bfloat16)
    e = moqe.moqe_fp_quantize(W, fmt)
    want = exact_product(X, W)
    M = X.shape[0]
    chunk = chunk or M
    ids = torch.zeros(chunk, dtype=torch.int32, device="cuda")
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(chunk, [e]))
    for m in range(0, M, chunk):
        rows = X[m:m + chunk]
        ws.fill_(255)
        Y = moqe.moqe_routed_fpgemm(rows, ids[:rows.shape[0]], [e], workspace=ws)
        assert moqe.moqe_async_status() == moqe.OK
        off = (Y != want[m:m + chunk]).any(1)
        assert not bool(off.any()), f"rows {(m + torch.nonzero(off)[:, 0]).tolist()[:8]} of {M}"
    return want


@pytest.mark.parametrize("fmt", [MX, NV, BF])
@pytest.mark.parametrize("chunk,N,K", [
    (1, 40, 4104), (1, 72, 18952), (1, 40, 65544), (1, 8, 131080),         # a row alone: its own kernel, and beyond what that holds
    (8, 264, 11016), (16, 136, 65544), (100, 136, 18952),                  # a block for each row
])
def test_every_part_of_few_rows(fmt, chunk, N, K):
    g = np.random.default_rng(K + chunk)
    parts = _seams(K) + [(int(k), 264) for k in g.integers(0, K - 264, 8)]
    M = -(-len(parts) // chunk) * chunk
    w = on_grid(g, N, K)
    want = _run(fmt, on_grid(g, M, K, at=_windows(M, K, parts)), w, chunk)
    assert bool((want != 0).any(1).all())                                  # (a part that is left out shows)
    _run(fmt, on_grid(g, min(chunk, 4), K), w)                             # whole rows


@pytest.mark.parametrize("fmt", [MX, NV, BF])
@pytest.mark.parametrize("M,N,K", [
    (300, 136, 32768), (300, 136, 32776), (276, 136, 32760), (1100, 264, 8200),  # the ring's rows, on both sides of its limits
    (4400, 136, 2056), (4500, 136, 2048), (9100, 136, 1000), (20000, 136, 456),
    (1100, 2056, 8200), (520, 4096, 4104),                                 # pairs of SMs
])
def test_every_part_of_many_rows(fmt, M, N, K):
    g = np.random.default_rng(M + K)
    parts = _seams(K) + [(k, min(256, K - k)) for k in range(0, K, 256)]
    w = on_grid(g, N, K)
    x = on_grid(g, M, K, at=_windows(M, K, parts))
    x[len(parts):len(parts) + 40] = on_grid(g, min(40, M - len(parts)), K)  # whole rows among them
    want = _run(fmt, x, w)
    assert bool((want != 0).any(1).all())


@pytest.mark.parametrize("M,N,K", [(24, 264, 32776), (300, 520, 18952), (1200, 136, 8200)])
def test_formats_beside_each_other(M, N, K):
    g = np.random.default_rng(M)
    formats = [NV, BF, MX]
    parts = _seams(K)
    X = torch.from_numpy(on_grid(g, M, K, at=_windows(M, K, parts))).cuda().to(torch.bfloat16)
    W = [torch.from_numpy(on_grid(g, N, K)).cuda() for _ in formats]
    ids = torch.from_numpy(g.integers(0, 3, M).astype(np.int32)).cuda()
    Y = moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(w, f) for w, f in zip(W, formats)])
    assert moqe.moqe_async_status() == moqe.OK
    for e, w in enumerate(W):
        assert torch.equal(Y[ids == e], exact_product(X[ids == e], w))
