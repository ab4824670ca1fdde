"""What a product sees of a row is exactly what moqe_fp4_quantize_rows gives: rows that quantize to the same numbers have the same outputs,
bit for bit, in both formats and all rows."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe
from test_gpu_fp_gemm import MX, NV, _bf16, _expert

pytestmark = pytest.mark.gpu


def _held(g, M, K, fmt):
    """[M][K]: numbers the format holds, which quantize to themselves, and others that quantize to the same: a 6 under every scale stays as
    it is, what else a block has moves by up to a twentieth, less than half of any step, but not beyond the 6."""
    size = R.BLOCK[fmt]
    nb = -(-K // size)
    v = R.E2M1[g.integers(0, 8, (M, nb, size))]
    v[:, :, 0] = 6.0
    if fmt == MX:
        scale = 2.0 ** g.integers(-6, 7, (M, nb))
        outer = 1.0
    else:
        scale = R.E4M3[g.integers(40, 120, (M, nb))]                       # 2^-2 .. 240
        scale[:, 0] = R.E4M3[g.integers(115, 122, M)]                      # the row's largest: 6 times 176 .. 288, so that its row scale is
        scale = np.minimum(scale, scale[:, :1])
        outer = 2.0 ** g.integers(-20, 20, (M, 1, 1))                       # this one
    sign = np.where(g.random(v.shape) < 0.5, -1.0, 1.0)
    near = np.minimum(v * np.where(np.arange(size) == 0, 1.0, 1 + 0.05 * g.uniform(-1, 1, v.shape)), 6.0)
    flat = lambda a: (a * sign * scale[:, :, None] * outer).reshape(M, nb * size)[:, :K]
    return flat(v), flat(near)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N,K", [(1, 264, 1000), (50, 264, 1000), (5, 40, 4104), (300, 520, 2056), (1200, 136, 8200)])
def test_rows_that_quantize_alike(fmt, M, N, K):
    g = np.random.default_rng(M + K + fmt)
    held, near = _held(g, M, K, fmt)
    H, X = _bf16(held), _bf16(near)
    assert np.array_equal(H.double().cpu().numpy(), held)                 # (bf16 holds them)
    a, b = moqe.moqe_fp4_quantize_rows(H, fmt, values=True), moqe.moqe_fp4_quantize_rows(X, fmt, values=True)
    assert all(p is q or torch.equal(p, q) for p, q in zip(a, b)) and torch.equal(a[3], H)
    again = moqe.moqe_fp4_quantize_rows(a[3], fmt, values=True)
    assert all(p is q or torch.equal(p, q) for p, q in zip(a, again))
    e, _ = _expert(M, N, K, fmt)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    Y = moqe.moqe_routed_fpgemm(H, ids, [e])
    assert bool(Y.isfinite().all()) and bool((Y != 0).any(1).all())
    for rows in (X, a[3], b[3]):
        assert torch.equal(moqe.moqe_routed_fpgemm(rows, ids, [e]), Y)
    assert moqe.moqe_async_status() == moqe.OK
