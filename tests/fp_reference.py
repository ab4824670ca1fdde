"""The floating-point experts' formats and product from their definitions, in numpy and 64 bits (no code of the library)."""
import numpy as np

MXFP4, NVFP4, BF16 = 1, 2, 3
BLOCK = {MXFP4: 32, NVFP4: 16}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([i * 2.0 ** -9 for i in range(8)] + [(8 + i) * 2.0 ** (e - 3) for e in range(-6, 9) for i in range(8)][:119])


def nearest(q, grid):
    """Index of the grid number nearest to each q >= 0, the even one of two equally near ones."""
    i = np.clip(np.searchsorted(grid, q, side="right") - 1, 0, len(grid) - 2)
    below, above = q - grid[i], grid[i + 1] - q
    return i + ((above < below) | ((above == below) & (i % 2 == 1)))


def floor_log2(a):
    return np.frexp(a)[1] - 1


def encode(x, fmt):
    """x [R][K] (float32 numbers) -> codes uint8 [R][K] (one a byte), scale bytes [R][blocks], outer [R] or None, values [R][K]."""
    x = np.asarray(x, dtype=np.float64)
    R, K = x.shape
    size = BLOCK[fmt]
    nb = -(-K // size)
    pad = np.zeros((R, nb * size))
    pad[:, :K] = x
    b = pad.reshape(R, nb, size)
    finite = np.isfinite(b)
    bad = ~finite.all(2)
    mag = np.where(finite, np.abs(b), 0.0)
    outer = np.ones(R)
    if fmt == NVFP4:
        A = mag.max((1, 2), initial=0.0)
        outer = np.where(A > 0, 2.0 ** np.maximum(floor_log2(np.where(A > 0, A, 1.0)) - 10, -126.0), 1.0)
    amax = mag.max(2, initial=0.0)
    if fmt == MXFP4:
        e = np.where(amax > 0, np.maximum(floor_log2(np.where(amax > 0, amax, 1.0)) - 2, -127), -127)
        byte, s, nan = e + 127, 2.0 ** e, 255
    else:
        byte = nearest(amax / outer[:, None] / 6.0, E4M3)
        s, nan = E4M3[byte], 127
    whole = s * outer[:, None]
    q = np.where(whole[:, :, None] > 0, mag / np.where(whole > 0, whole, 1.0)[:, :, None], 0.0)
    sign = np.signbit(b)
    codes = nearest(q, E2M1) + 8 * sign
    values = E2M1[codes & 7] * np.where(sign, -1.0, 1.0) * whole[:, :, None]
    codes, byte = np.where(bad[:, :, None], 0, codes), np.where(bad, nan, byte)
    values = np.where(bad[:, :, None], np.nan, values)
    flat = lambda a: a.reshape(R, nb * size)[:, :K]
    return flat(codes).astype(np.uint8), byte.astype(np.uint8), (outer if fmt == NVFP4 else None), flat(values)


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def decode(packed, byte, outer, fmt):
    """Values of canonical arrays."""
    c = np.stack((packed & 15, packed >> 4), 2).reshape(packed.shape[0], -1).astype(np.int64)
    v = E2M1[c & 7] * np.where(c >= 8, -1.0, 1.0)
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127)) if fmt == MXFP4 else np.where(byte >= 127, np.nan, E4M3[np.minimum(byte, 126)])
    v = v * np.repeat(s, BLOCK[fmt], 1)[:, :c.shape[1]]
    return v if outer is None else v * outer[:, None].astype(np.float64)


def product(xq, wq):
    """Exact sums and what bounds an fp32 accumulation's error: (y, sum of the products' magnitudes)."""
    return xq @ wq.T, np.abs(xq) @ np.abs(wq).T


def tolerance(y, mags, K):
    """bf16 rounds by at most 2^-8 of the value.  The sums are fp32: an MMA takes 16 k at least and adds them to the accumulator, with
    at most 2^-22 of the sum of magnitudes lost at each of the K / 16 + 1 additions (alignment and rounding of its terms), and a few
    more where CTAs share a tile or scales are applied."""
    acc = (K / 16 + 8) * 2.0 ** -22 * mags
    return 2.0 ** -8 * np.abs(y) + 2 * acc + 1e-38
