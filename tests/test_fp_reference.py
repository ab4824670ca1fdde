"""Pins of the 64-bit reference of the microscaled formats, by hand-worked values and properties (no GPU)."""
import numpy as np
import pytest

import fp_reference as R


def test_grids():
    assert len(R.E4M3) == 127 and R.E4M3[-1] == 448.0 and R.E4M3[8] == 2.0 ** -6 and np.all(np.diff(R.E4M3) > 0)
    # ties go to the even code
    assert list(R.nearest(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9]), R.E2M1)) == [0, 2, 2, 4, 4, 6, 6, 7]


def test_mxfp4_by_hand():
    x = np.zeros((1, 40), np.float32)
    x[0, :6] = [7.0, -6.0, 0.3, 0.25, -0.0, 5.0]        # largest 7: 2^(2 - 2) = 1
    x[0, 32:34] = [0.375, 0.1]                           # largest 0.375 = 1.5 * 2^-2: scale 2^-4
    codes, byte, outer, v = R.encode(x, R.MXFP4)
    assert list(byte[0]) == [127, 123] and outer is None
    assert list(codes[0, :6]) == [7, 15, 1, 0, 8, 6]
    assert list(v[0, :6]) == [6, -6, 0.5, 0, 0, 4] and list(v[0, 32:34]) == [0.375, 0.09375]
    assert np.array_equal(R.decode(R.pack(codes), byte, None, R.MXFP4), v)


def test_nvfp4_by_hand():
    x = np.zeros((2, 24), np.float32)
    x[0, 0], x[0, 16], x[0, 17] = 1536.0, 6.0, -1.0       # row scale 2^(10 - 10); scales 256 and 1
    codes, byte, outer, v = R.encode(x, R.NVFP4)
    assert list(outer) == [1.0, 1.0] and list(R.E4M3[byte[0]]) == [256.0, 1.0] and list(R.E4M3[byte[1]]) == [0, 0]
    assert v[0, 0] == 1536.0 and v[0, 16] == 6.0 and v[0, 17] == -1.0


@pytest.mark.parametrize("fmt", [R.MXFP4, R.NVFP4])
def test_properties(fmt):
    rng = np.random.default_rng(fmt)
    x = (rng.standard_normal((64, 72)) * np.exp(4 * rng.standard_normal((64, 1)))).astype(np.float32)
    codes, byte, outer, v = R.encode(x, fmt)
    # a power of two goes through, and so does what is on the grid already
    c2, b2, _, v2 = R.encode(np.ldexp(x, 3), fmt)
    assert np.array_equal(c2, codes) and np.array_equal(v2, 8 * v)
    assert np.array_equal(R.decode(R.pack(codes), byte, outer, fmt), v)
    # no number moves by more than half of the widest step, which is 2 scales, but where it is beyond 6 of them
    blocks = [(k, min(k + R.BLOCK[fmt], 72)) for k in range(0, 72, R.BLOCK[fmt])]
    for i, (a, b) in enumerate(blocks):
        scale = (2.0 ** (byte[:, i].astype(float) - 127) if fmt == R.MXFP4 else R.E4M3[byte[:, i]] * outer)[:, None]
        d = np.abs(v[:, a:b] - x[:, a:b].astype(np.float64))
        assert np.all((d <= scale) | (np.abs(x[:, a:b]) > 6 * scale))
    y = x.copy()
    y[3, 5], y[4, 70] = np.inf, np.nan
    cn, bn, on, vn = R.encode(y, fmt)
    nan = 255 if fmt == R.MXFP4 else 127
    assert bn[3, 5 // R.BLOCK[fmt]] == nan and bn[4, 70 // R.BLOCK[fmt]] == nan and (bn == nan).sum() == 2
    assert np.isnan(vn[3, :R.BLOCK[fmt]]).all() and not np.isnan(vn[3, R.BLOCK[fmt]:]).any()
