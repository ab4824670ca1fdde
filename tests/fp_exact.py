"""Inputs that the 4-bit formats hold as they are and whose products sum exactly in fp32, in any order: outputs are compared to the bit,
where a tolerance that grows with the sum of magnitudes would let parts of a long row go missing."""
import numpy as np
import torch


def on_grid(g, R, K, at=None):
    """fp32 [R][K]: e2m1 numbers with a 6 (either sign) in every 16 k, the last, short ones too, times 1 or 2 for every 32 k; `at` [R][K]: zero
    elsewhere (with a 6 still in every 16 k that has any).  MXFP4's scale is the factor, NVFP4's block scale and row scale multiply to it:
    both formats, and bf16, hold these numbers exactly."""
    v = g.choice(np.array([0, .5, 1, 1.5, 2, -.5, -1, -1.5, -2]), (R, K))
    pad = -K % 16
    inside = np.pad(np.ones((R, K), bool) if at is None else at, ((0, 0), (0, pad))).reshape(R, -1, 16)
    order = np.where(inside, g.random(inside.shape), -1.0)
    six = np.zeros(inside.shape, bool)
    np.put_along_axis(six, order.argmax(2)[:, :, None], True, 2)
    six = (six & inside).reshape(R, -1)[:, :K]
    v = np.where(six, g.choice([6.0, -6.0], (R, K)), v)
    if at is not None:
        v = np.where(at, v, 0.0)
    return (v * np.repeat(2.0 ** g.integers(0, 2, (R, -(-K // 32))), 32, 1)[:, :K]).astype(np.float32)


def exact_product(X, W):
    """X . W^T of numbers `on_grid` gave, rounded to bf16 once.  Every product is a multiple of 2^-2; as long as their magnitudes sum to less
    than 2^21, every partial sum is a multiple of 2^-2 with at most 23 bits, which fp32 holds."""
    x, w = X.double(), W.double()
    assert float((x.abs() @ w.abs().t()).max()) < 2.0 ** 21
    return (x @ w.t()).float().to(torch.bfloat16)
