"""Microscaled 4-bit rows and experts against their definitions in 64 bits: codes, scales, row scales and values bit for bit."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe

pytestmark = pytest.mark.gpu
FORMATS = [moqe.FP_MXFP4, moqe.FP_NVFP4]


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _rows(seed, M, K):
    """Rows of all kinds: ordinary ones, wide ranges, zeros, numbers near the ends of the type, ties."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((M, K)).astype(np.float32)
    kind = np.arange(M) % 8
    x[kind == 1] *= np.exp(6 * g.standard_normal((np.sum(kind == 1), K))).astype(np.float32)
    x[kind == 2] = 0.0
    x[kind == 3] *= 1e-38
    x[kind == 4] *= 1e37
    x[kind == 5] = (g.integers(-28, 29, (np.sum(kind == 5), K)) * 0.25).astype(np.float32)          # many ties
    x[kind == 6, :K // 2] = -0.0
    return x


def _check(codes, scales, outer, values, want):
    wc, wb, wo, wv = want
    assert np.array_equal(scales.cpu().numpy(), wb)
    assert np.array_equal(codes.cpu().numpy(), R.pack(wc))
    if wo is None:
        assert outer is None
    else:
        assert np.array_equal(outer.cpu().numpy().astype(np.float64), wo)
    if values is not None:
        # (code * scale * outer has 6 bits at most: bf16 rounds it only among its subnormals, and beyond its largest number)
        with np.errstate(over="ignore"):
            rounded = torch.from_numpy(wv.astype(np.float32)).to(torch.bfloat16)
        assert np.array_equal(values.float().cpu().numpy(), rounded.float().numpy(), equal_nan=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,K", [(1, 8), (1, 32), (3, 40), (9, 264), (16, 1032), (5, 4096), (33, 2056), (2, 18944), (257, 72)])
def test_rows(fmt, M, K):
    X = _dev(_rows(K, M, K)).to(torch.bfloat16)
    got = moqe.moqe_fp4_quantize_rows(X, fmt, values=True)
    _check(*got, R.encode(X.float().cpu().numpy(), fmt))
    again = moqe.moqe_fp4_quantize_rows(X, fmt)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]) and again[3] is None


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bf16_number(fmt):
    """Every finite bf16 number as a row's only one, and beside one 64 times as large."""
    bits = np.arange(65536, dtype=np.uint32)
    v = (bits << 16).view(np.float32)
    v = v[np.isfinite(v)]
    x = np.zeros((v.size, 32), np.float32)
    x[:, 0] = v
    big = np.clip(v.astype(np.float64) * 64, -3.3e38, 3.3e38).astype(np.float32)
    y = x.copy()
    y[:, 1] = big
    for a in (x, y):
        X = _dev(a).to(torch.bfloat16)
        _check(*moqe.moqe_fp4_quantize_rows(X, fmt, values=True), R.encode(X.float().cpu().numpy(), fmt))


@pytest.mark.parametrize("fmt", FORMATS)
def test_infinities_and_nan(fmt):
    x = _rows(3, 16, 200)
    x[0, 5], x[1, 199], x[2, 64], x[5, :] = np.inf, np.nan, -np.inf, np.nan
    X = _dev(x).to(torch.bfloat16)
    _check(*moqe.moqe_fp4_quantize_rows(X, fmt, values=True), R.encode(X.float().cpu().numpy(), fmt))


def test_rows_of_a_view_and_nothing():
    X = torch.randn(64, 128, device="cuda").to(torch.bfloat16)
    for fmt in FORMATS:
        a = moqe.moqe_fp4_quantize_rows(X[:, :64], fmt, values=True)             # (the binding makes it contiguous)
        b = moqe.moqe_fp4_quantize_rows(X[:, :64].contiguous(), fmt, values=True)
        assert all(p is q or torch.equal(p, q) for p, q in zip(a, b))
        assert moqe.moqe_fp4_quantize_rows(X[:0], fmt)[0].shape == (0, 64)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("N,K", [(8, 8), (128, 256), (136, 264), (1, 4096), (520, 1000), (24, 11008), (16, 18944)])
def test_experts(fmt, N, K):
    W = _rows(N + K, N, K)
    W[0, :min(K, 7)] = np.nextafter(np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]), np.float32(9))[:min(K, 7)]   # just beyond the borders
    e = moqe.moqe_fp_quantize(_dev(W), fmt)
    assert (e.N, e.K, e.format) == (N, K, fmt) and e.code_bytes == N * K // 2 and e.alloc_bytes >= e.code_bytes
    want = R.encode(W, fmt)
    got = moqe.moqe_fp_expert_export(e, values=True)
    _check(*got, want)
    # through the canonical arrays and back
    f = moqe.moqe_fp_expert_import(fmt, codes=got[0], scales=got[1], outer=got[2])
    for a, b in zip(moqe.moqe_fp_expert_export(f, values=True), got):
        assert a is b or torch.equal(a, b)


@pytest.mark.parametrize("fmt", FORMATS)
def test_expert_borders(fmt):
    """fp32 weights a unit of the last place around every border, under every scale that NVFP4 has near a row's top."""
    g = np.random.default_rng(5)
    border = np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    W = np.zeros((1024, 32), np.float32)
    for half in (0, 16):
        top = g.uniform(3, 6, 1024).astype(np.float32)
        W[:, half] = top
        for i, b in enumerate(border):
            # the nearest e4m3 number under the row's scale, then its multiples by the border, and their neighbours
            s = R.E4M3[R.nearest(top.astype(np.float64) * 256 / 6, R.E4M3)] / 256 if fmt == R.NVFP4 else np.ones(1024)
            m = (b * s).astype(np.float32)
            W[:, half + 1 + i] = m
            W[:, half + 8 + i] = np.nextafter(m, np.float32(0) if i % 2 else np.float32(99))
    got = moqe.moqe_fp_expert_export(moqe.moqe_fp_quantize(_dev(W), fmt), values=True)
    _check(*got, R.encode(W, fmt))


@pytest.mark.parametrize("N,K", [(8, 8), (130, 72), (256, 4096)])
def test_bf16_expert(N, K):
    W = _dev(np.random.default_rng(1).standard_normal((N, K)).astype(np.float32))
    e = moqe.moqe_fp_quantize(W, moqe.FP_BF16)
    codes, scales, outer, values = moqe.moqe_fp_expert_export(e)
    assert codes is None and scales is None and outer is None
    assert torch.equal(values.view(torch.int16), W.to(torch.bfloat16).view(torch.int16))
    f = moqe.moqe_fp_expert_import(moqe.FP_BF16, values=values)
    assert torch.equal(moqe.moqe_fp_expert_export(f)[3].view(torch.int16), values.view(torch.int16))
    assert e.code_bytes == 2 * N * K and e.meta_bytes == 0


def test_any_outer_can_be_imported():
    g = np.random.default_rng(2)
    codes = g.integers(0, 256, (40, 24), dtype=np.uint8)
    scales = g.integers(0, 128, (40, 3), dtype=np.uint8)
    outer = g.standard_normal(40).astype(np.float32)
    e = moqe.moqe_fp_expert_import(moqe.FP_NVFP4, _dev(codes), _dev(scales), _dev(outer))
    c, s, o, v = moqe.moqe_fp_expert_export(e, values=True)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales) and np.array_equal(o.cpu().numpy(), outer)
    want = R.decode(codes, scales, outer, R.NVFP4)
    got = v.float().cpu().numpy()
    ok = ~np.isnan(want)
    assert np.array_equal(np.isnan(got), ~ok) and np.all(np.abs(got[ok] - want[ok]) <= np.abs(want[ok]) * (2.0 ** -8 + 2.0 ** -22))
    # without one: 1; the scales' top bit is not looked at
    f = moqe.moqe_fp_expert_import(moqe.FP_NVFP4, _dev(codes), _dev(scales | 128))
    c, s, o, _ = moqe.moqe_fp_expert_export(f)
    assert np.array_equal(s.cpu().numpy(), scales) and bool((o == 1).all())


def test_refusals_of_the_binding():
    W = torch.zeros(16, 64, device="cuda")
    e = moqe.moqe_fp_quantize(W, moqe.FP_MXFP4)
    b = moqe.moqe_fp_quantize(W, moqe.FP_BF16)
    buf = torch.zeros(4096, device="cuda").data_ptr()
    L = moqe.lib()
    assert L.moqe_fp_expert_export(e.handle, None, None, buf, None, None) == moqe.ERR_UNSUPPORTED
    assert L.moqe_fp_expert_export(b.handle, buf, None, None, None, None) == moqe.ERR_UNSUPPORTED
    assert L.moqe_fp_expert_export(e.handle, buf + 2, None, None, None, None) == moqe.ERR_UNSUPPORTED
    assert L.moqe_fp_expert_export(e.handle, None, None, None, None, None) == moqe.OK
    with pytest.raises(ValueError):
        moqe.moqe_fp4_quantize_rows(torch.zeros(2, 64, device="cuda"), moqe.FP_MXFP4)
    with pytest.raises(ValueError):
        moqe.moqe_fp_quantize(W.half(), moqe.FP_MXFP4)
    with pytest.raises(moqe.MoqeError):
        moqe.moqe_fp_expert_import(moqe.FP_MXFP4, codes=torch.zeros(8, 32, dtype=torch.uint8, device="cuda"),
                                   scales=torch.zeros(8, 3, dtype=torch.uint8, device="cuda"))
    with pytest.raises(moqe.MoqeError):
        moqe.moqe_fp_expert_import(moqe.FP_BF16)


@pytest.mark.parametrize("power", [0, -60, -125, 90])
def test_every_tie_under_every_scale(power):
    """NVFP4: each block's largest number makes its scale, the others are its half way marks and their bf16 neighbours on both sides."""
    marks = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows = []
    for b in range(1, 127):
        s = (b & 7) * 2.0 ** -9 if b < 8 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7)
        if 6 * s >= 2048:
            continue
        ties = (marks * s).astype(np.float32).view(np.uint32)
        assert np.array_equal(ties & 0xFFFF, 0 * ties)                       # (seven bits: bf16 has them)
        for step in (-0x10000, 0, 0x10000):
            near = (ties.astype(np.int64) + step).astype(np.uint32).view(np.float32)
            rows.append(np.concatenate([[6 * s], near, -near, [0], [1536], 15 * [0]]))    # the row's scale is 1
    X = torch.from_numpy(np.ldexp(np.array(rows, dtype=np.float32), power)).to(torch.bfloat16).cuda()
    _check(*moqe.moqe_fp4_quantize_rows(X, moqe.FP_NVFP4, values=True), R.encode(X.float().cpu().numpy(), moqe.FP_NVFP4))
