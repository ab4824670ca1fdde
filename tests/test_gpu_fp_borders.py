"""fp32 weights in the last places around every border: of the codes under every e4m3 scale, and of the scales themselves."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe
from test_gpu_fp_formats import _check

pytestmark = pytest.mark.gpu
MARKS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
STEPS = (-3, -2, -1, 0, 1, 2, 3)


def _stepped(v, step):
    """fp32 numbers some last places off positive ones that fp32 holds."""
    bits = v.astype(np.float32).view(np.uint32).astype(np.int64) + step
    return np.maximum(bits, 0).astype(np.uint32).view(np.float32)


def _build(rows, power):
    W = np.ldexp(np.array(rows, dtype=np.float32), power)
    e = moqe.moqe_fp_quantize(torch.from_numpy(W).cuda(), moqe.FP_NVFP4)
    _check(*moqe.moqe_fp_expert_export(e, values=True), R.encode(W, moqe.FP_NVFP4))


@pytest.mark.parametrize("power", [0, -100, 110])
def test_codes(power):
    rows = []
    for b in range(1, 127):
        s = R.E4M3[b]
        if 6 * s >= 2048:
            continue
        for step in STEPS:
            near = _stepped(MARKS * s, step)
            rows.append(np.concatenate([[6 * s], near, -near, [0], [1536], 15 * [0]]))       # the row's scale is 1
    _build(rows, power)


@pytest.mark.parametrize("power", [0, -100, 110])
def test_scales(power):
    """A block's largest number around six times the middle of two e4m3 numbers, the subnormal ones among them."""
    rows = []
    for b in range(126):
        middle = (R.E4M3[b] + R.E4M3[b + 1]) / 2
        if 6 * middle >= 2048:
            continue
        for step in STEPS:
            top = _stepped(np.array([6 * middle]), step)[0]
            rows.append(np.concatenate([[top, -top / 2, top / 3], 13 * [top / 7], [1536], 15 * [0]]))
    _build(rows, power)


def test_random_numbers_near_borders():
    """Any quotient's neighbourhood: random scales times random marks, off by a few last places of the product."""
    g = np.random.default_rng(3)
    n = 20000
    tops = R.E4M3[g.integers(1, 115, n)]
    rows = np.zeros((n, 32), np.float32)
    rows[:, 0] = 6 * tops * g.uniform(0.97, 1.0, n)                                           # the scale is the nearest e4m3 number
    s = R.E4M3[R.nearest(rows[:, 0].astype(np.float64) / 6, R.E4M3)]
    for i in range(1, 16):
        rows[:, i] = _stepped(MARKS[g.integers(0, 7, n)] * s, g.integers(-2, 3, n)) * np.where(g.random(n) < 0.5, -1, 1)
    rows[:, 1:16] = np.where(np.abs(rows[:, 1:16]) <= rows[:, :1], rows[:, 1:16], 0)
    rows[:, 16] = 1536
    _build(rows, 0)
