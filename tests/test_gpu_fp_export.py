"""Values of imported experts: code * scale * outer is rounded to bf16 once, whatever fp32 number the outer scale is."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe

pytestmark = pytest.mark.gpu


def nearest_bf16(v):
    """v (64 bits, exact) to the nearest bf16 number, ties to even, as float32."""
    _, e = np.frexp(v)
    step = np.exp2(np.maximum(e - 8, -133).astype(np.float64))          # (below 2^-126 the steps stay as they are)
    with np.errstate(invalid="ignore", over="ignore"):
        r = np.rint(v / step) * step
        return np.where(np.abs(r) >= 2.0 ** 128, np.copysign(np.inf, v), r).astype(np.float32)


def near_ties(g, power, n=2048):
    """Outer scales, and for each the scale byte under which a code of 3 comes as near to the middle of two bf16 numbers as fp32 allows:
    nearer than fp32's own rounding of the product, where that happens."""
    byte = g.integers(8, 127, n)
    a = 3.0 * R.E4M3[byte]
    middle = (2 * g.integers(128, 256, n) + 1) * 2.0 ** -8                # of two neighbours in [1, 2)
    outer = (middle / a).astype(np.float32)
    # (a few last places around it)
    outer = (outer.view(np.uint32) + g.integers(-2, 3, n).astype(np.uint32)).view(np.float32)
    return byte.astype(np.uint8), np.ldexp(outer, power).astype(np.float32)


@pytest.mark.parametrize("power", [0, 60, -60, 120, -100, -126, -133])
def test_values_are_rounded_once(power):
    g = np.random.default_rng(power + 200)
    byte, outer = near_ties(g, power)
    N, K = byte.size, 16
    codes = np.tile(np.array([5, 13] + list(range(14)), np.uint8), (N, 1))                # 3, -3 and all others
    scales = byte[:, None]
    e = moqe.moqe_fp_expert_import(moqe.FP_NVFP4, torch.from_numpy(R.pack(codes)).cuda(), torch.from_numpy(scales).cuda(), torch.from_numpy(outer).cuda())
    got = moqe.moqe_fp_expert_export(e, values=True)[3].float().cpu().numpy()
    exact = R.decode(R.pack(codes), scales, outer, R.NVFP4)                              # (30 bits at most)
    want = nearest_bf16(exact)
    if power == 0:
        with np.errstate(over="ignore"):
            twice = nearest_bf16(exact.astype(np.float32).astype(np.float64))
        assert int((twice != want).sum()) > 50                                           # rounding to fp32 in between shows
    assert np.array_equal(got.view(np.uint32) << 1, want.view(np.uint32) << 1)           # (zeros of either sign)
    assert np.array_equal(np.signbit(got)[want != 0], np.signbit(want)[want != 0])


def test_signs_and_no_numbers():
    codes = np.tile(np.arange(16, dtype=np.uint8), (6, 1))
    scales = np.array([56, 56, 56, 127, 0, 126], np.uint8)[:, None]
    outer = np.array([-1.5, np.inf, np.nan, 1.0, 1.0, 3e38], np.float32)
    e = moqe.moqe_fp_expert_import(moqe.FP_NVFP4, torch.from_numpy(R.pack(codes)).cuda(), torch.from_numpy(scales).cuda(), torch.from_numpy(outer).cuda())
    got = moqe.moqe_fp_expert_export(e, values=True)[3].float().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = nearest_bf16(R.decode(R.pack(codes), scales, outer, R.NVFP4))
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(np.signbit(got[0]), np.signbit(-1.5 * np.where(np.arange(16) < 8, 1.0, -1.0)))
