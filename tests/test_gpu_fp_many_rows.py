"""Rows in a 4-bit format, as many as an int counts."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [2 ** 31 - 1, 2 ** 31 - 4])
def test_as_many_rows_as_an_int_counts(M):
    K = 8
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("34 GB of rows")
    X = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 2 ** 30 - 1, 2 ** 30, M - 5, M - 4, M - 3, M - 2, M - 1], device="cuda")
    X[at] = torch.from_numpy(np.random.default_rng(1).standard_normal((at.numel(), K)).astype(np.float32)).cuda().to(torch.bfloat16)
    scales = torch.full((M + 64,), 7, dtype=torch.uint8, device="cuda")
    codes = torch.full((M * K // 2 + 64,), 7, dtype=torch.uint8, device="cuda")
    for fmt in (moqe.FP_MXFP4, moqe.FP_NVFP4):
        codes[-64 - 64 * K:].fill_(7)
        scales[-128:].fill_(7)
        st = moqe.lib().moqe_fp4_quantize_rows(X.data_ptr(), M, K, fmt, codes.data_ptr(), scales.data_ptr(), None, None, moqe._stream())
        assert st == moqe.OK and moqe.moqe_async_status() == moqe.OK
        wc, wb, _, _ = R.encode(X[at].float().cpu().numpy(), fmt)
        assert np.array_equal(scales[at].cpu().numpy(), wb[:, 0])
        assert np.array_equal(codes[:M * K // 2].view(M, K // 2)[at].cpu().numpy(), R.pack(wc))
        zero, = R.encode(np.zeros((1, K), np.float32), fmt)[1][0]
        assert bool((scales[2 ** 30 + 1:2 ** 30 + 65] == int(zero)).all()) and bool((scales[M - 45:M - 5] == int(zero)).all())
        assert bool((scales[M:] == 7).all()) and bool((codes[M * K // 2:] == 7).all())
    del X, scales, codes
    torch.cuda.empty_cache()
