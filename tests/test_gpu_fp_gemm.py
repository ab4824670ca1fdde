"""The routed product of floating-point experts against 64 bits: formats and mixtures, ragged and empty segments, odd sizes, one row to
thousands; what else a serving loop does with it (graphs, streams, a sort shared with integer experts)."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe

pytestmark = pytest.mark.gpu
MX, NV, BF = moqe.FP_MXFP4, moqe.FP_NVFP4, moqe.FP_BF16


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _bf16(a):
    return _dev(a.astype(np.float32)).to(torch.bfloat16)


def _expert(seed, N, K, fmt):
    """(handle, its weights in 64 bits)"""
    W = (np.random.default_rng(seed).standard_normal((N, K)) * 0.02).astype(np.float32)
    e = moqe.moqe_fp_quantize(_dev(W), fmt)
    if fmt == BF:
        return e, _dev(W).to(torch.bfloat16).double()
    return e, _dev(R.encode(W, fmt)[3])


def _quantized(X, fmt):
    return X.double() if fmt == BF else _dev(R.encode(X.float().cpu().numpy(), fmt)[3])


def _check(Y, X, ids, weights, formats):
    """Every row against the exact product (on the device, in 64 bits)."""
    K = X.shape[1]
    for e, (w, f) in enumerate(zip(weights, formats)):
        rows = torch.nonzero(ids == e)[:, 0]
        if rows.numel() == 0:
            continue
        xq = _quantized(X[rows], f)
        y, mags = xq @ w.t(), xq.abs() @ w.abs().t()
        tol = 2.0 ** -8 * y.abs() + 2 * (K / 16 + 8) * 2.0 ** -22 * mags + 1e-38                # fp_reference.tolerance
        bad = ~((Y[rows].double() - y).abs() <= tol)
        assert not bool(bad.any()), f"expert {e} (format {f}): {int(bad.sum())} of {bad.numel()} off, first {torch.nonzero(bad)[0].tolist()}: " \
                                    f"{Y[rows].double()[bad][0].item()} for {y[bad][0].item()}"


def _case(seed, M, N, K, formats, counts=None):
    g = np.random.default_rng(seed)
    E = len(formats)
    ids = g.integers(0, E, M) if counts is None else np.repeat(np.arange(E), counts)
    g.shuffle(ids)
    X = _bf16(g.standard_normal((M, K)) * np.exp(g.standard_normal((M, 1))))
    return X, _dev(ids.astype(np.int32)), [_expert(seed * 100 + e, N, K, f) for e, f in enumerate(formats)]


@pytest.mark.parametrize("fmt", [MX, NV, BF])
@pytest.mark.parametrize("M,N,K", [(1, 8, 8), (1, 128, 64), (1, 4096, 4096), (5, 136, 72), (16, 256, 256), (17, 128, 520), (33, 1000, 264), (64, 384, 1024),
                                   (65, 8, 4104), (128, 128, 2048), (129, 264, 512), (300, 520, 1032), (1000, 640, 776)])
def test_one_expert(fmt, M, N, K):
    X, ids, ex = _case(M + N + K, M, N, K, [fmt])
    Y = moqe.moqe_routed_fpgemm(X, ids, [e for e, _ in ex])
    assert moqe.moqe_async_status() == moqe.OK
    _check(Y, X, ids, [w for _, w in ex], [fmt])


@pytest.mark.parametrize("M,N,K,formats,counts", [
    (3, 256, 512, [MX, NV, BF], None),
    (16, 1024, 1024, [MX, NV, BF], [5, 0, 11]),
    (16, 11008, 4096, [MX, NV, BF], None),                       # work split along k
    (96, 512, 3584, [NV, MX], [0, 96]),
    (200, 200, 400, [BF, MX, NV, MX, NV], [1, 127, 0, 71, 1]),
    (777, 1000, 2056, [NV, BF, MX], [544, 155, 78]),
    (2500, 1536, 512, [MX, BF], None),                           # whole tiles dealt out in turn
    (700, 256, 256, [MX] * 16 + [NV] * 15 + [BF], None),          # as many experts as there may be
    (40, 136, 136, [NV] * 32, [0] * 31 + [40]),
])
def test_mixtures(M, N, K, formats, counts):
    X, ids, ex = _case(M + K, M, N, K, formats, counts)
    handles = [e for e, _ in ex]
    Y = moqe.moqe_routed_fpgemm(X, ids, handles)
    assert moqe.moqe_async_status() == moqe.OK
    _check(Y, X, ids, [w for _, w in ex], formats)
    # the same bits again, on a workspace full of NaNs, and through the sorted call
    ws = torch.full((moqe.moqe_routed_fpgemm_workspace(M, handles),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(moqe.moqe_routed_fpgemm(X, ids, handles, workspace=ws).view(torch.int16), Y.view(torch.int16))
    _, perm, offsets = moqe.moqe_permute(None, ids, len(formats))
    Z = torch.full_like(Y, float("nan"))
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets, handles, Z, ws)
    assert torch.equal(Z.view(torch.int16), Y.view(torch.int16))
    assert moqe.moqe_async_status() == moqe.OK


def test_quantized_rows_are_what_the_product_sees():
    """The product of rows equals that of their quantized values, bit for bit."""
    for fmt in (MX, NV):
        X, ids, ex = _case(7, 50, 264, 1000, [fmt])
        V = moqe.moqe_fp4_quantize_rows(X, fmt, values=True)[3]
        e = [ex[0][0]]
        a, b = moqe.moqe_routed_fpgemm(X, ids, e), moqe.moqe_routed_fpgemm(V, ids, e)
        if fmt == MX:
            # (a block whose largest number was rounded up across a power of two has another scale the second time)
            again = moqe.moqe_fp4_quantize_rows(V, fmt, values=True)[3]
            same = (again == V).all(1)
            assert bool(same.any())
            a, b = a[same], b[same]
            assert torch.equal(a, b)


def test_infinities_and_nan_stay_in_their_rows():
    for fmt in (MX, NV, BF):
        X, ids, ex = _case(11, 40, 136, 520, [fmt])
        clean = moqe.moqe_routed_fpgemm(X, ids, [ex[0][0]])
        X2 = X.clone()
        X2[3, 7], X2[17, 519], X2[39, 0] = float("nan"), float("inf"), float("-inf")
        Y = moqe.moqe_routed_fpgemm(X2, ids, [ex[0][0]])
        dirty = torch.zeros(40, dtype=torch.bool, device="cuda")
        dirty[[3, 17, 39]] = True
        assert torch.equal(Y[~dirty], clean[~dirty])
        if fmt != BF:
            assert bool(torch.isnan(Y[dirty]).all())
        else:
            assert bool(torch.isnan(Y[3]).all()) and not bool(torch.isfinite(Y[17]).any())


def test_weights_that_are_no_numbers_stay_in_their_channels():
    for fmt in (MX, NV):
        g = np.random.default_rng(4)
        W = g.standard_normal((200, 264)).astype(np.float32)
        W2 = W.copy()
        W2[5, 100], W2[199, 263] = np.nan, np.inf
        X, ids = _bf16(g.standard_normal((20, 264))), torch.zeros(20, dtype=torch.int32, device="cuda")
        a = moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(W), fmt)])
        b = moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(W2), fmt)])
        bad = torch.zeros(200, dtype=torch.bool, device="cuda")
        bad[[5, 199]] = True
        assert bool(torch.isnan(b[:, bad]).all()) and torch.equal(a[:, ~bad], b[:, ~bad])


def test_large_and_small_numbers():
    """Row scales, block scales and an imported outer at the ends of their ranges."""
    g = np.random.default_rng(8)
    X = _bf16(g.standard_normal((24, 512)) * np.exp2(np.arange(24) * 4.0 - 46)[:, None])
    ids = torch.zeros(24, dtype=torch.int32, device="cuda")
    for fmt in (MX, NV):
        W = (g.standard_normal((64, 512)) * np.exp2(np.arange(64) - 32.0)[:, None]).astype(np.float32)
        Y = moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(W), fmt)])
        _check(Y, X, ids, [_dev(R.encode(W, fmt)[3])], [fmt])
    codes, scales = g.integers(0, 256, (64, 256), dtype=np.uint8), g.integers(1, 126, (64, 32), dtype=np.uint8)
    outer = (g.standard_normal(64) * 0.37).astype(np.float32)
    e = moqe.moqe_fp_expert_import(NV, _dev(codes), _dev(scales), _dev(outer))
    _check(moqe.moqe_routed_fpgemm(X, ids, [e]), X, ids, [_dev(R.decode(codes, scales, outer, NV))], [NV])


def test_rows_of_nobody():
    """Ids outside [0, E) give zeros in the one-call form; the sorted form leaves rows outside its offsets alone."""
    X, ids, ex = _case(21, 90, 264, 512, [MX, NV])
    ids[::7] = -3
    ids[1::11] = 2
    handles = [e for e, _ in ex]
    Y = moqe.moqe_routed_fpgemm(X, ids, handles, Y=torch.full((90, 264), 5.0, dtype=torch.bfloat16, device="cuda"))
    assert moqe.moqe_async_status() == moqe.ERR_EXPERT_ID
    _check(Y, X, ids, [w for _, w in ex], [MX, NV])
    out = (ids < 0) | (ids > 1)
    assert bool((Y[out] == 0).all())
    _, perm, offsets = moqe.moqe_permute(None, ids, 2)
    assert moqe.moqe_async_status() == moqe.ERR_EXPERT_ID
    Z = torch.full_like(Y, 5.0)
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(90, handles))
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets, handles, Z, ws)
    assert torch.equal(Z[~out], Y[~out]) and bool((Z[out] == 5).all())


def test_nothing_to_do():
    X, ids, ex = _case(5, 4, 64, 64, [MX])
    assert moqe.moqe_routed_fpgemm(X[:0], ids[:0], [ex[0][0]]).shape == (0, 64)
    Y = torch.full((4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(4, [ex[0][0]]))
    perm = torch.arange(4, dtype=torch.int32, device="cuda")
    for off in ([0, 0], [2, 2], [4, 4]):
        moqe.moqe_routed_fpgemm_sorted(X, perm, torch.tensor(off, dtype=torch.int32, device="cuda"), [ex[0][0]], Y, ws)
    assert bool((Y == 3).all()) and moqe.moqe_async_status() == moqe.OK


@pytest.mark.parametrize("M", [30, 300])
def test_one_sort_for_integer_and_floating_point_experts(M):
    g = np.random.default_rng(M)
    N, K = 384, 512
    W = (g.standard_normal((N, K)) * 0.02).astype(np.float32)
    ints = [moqe.moqe_quantize_rtn(_dev(W), 8, 0, True), moqe.moqe_quantize_rtn(_dev(W), 4, 128, False)]
    floats = [_expert(1, N, K, MX), _expert(2, N, K, NV), _expert(3, N, K, BF)]
    ids = _dev(g.integers(0, 5, M).astype(np.int32))
    X = _bf16(g.standard_normal((M, K)))
    _, perm, offsets = moqe.moqe_permute(None, ids, 5)
    Y = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = moqe.alloc_workspace(moqe.moqe_routed_qgemm_workspace(M, N, K, 2))
    moqe.moqe_routed_qgemm_workspace_clear(ws, M, N, K, 2)
    handles = [e for e, _ in floats]
    fws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, handles))
    moqe.moqe_routed_qgemm_sorted(X, perm, offsets, ints, Y, ws)
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[2:], handles, Y, fws)
    assert moqe.moqe_async_status() == moqe.OK
    low = ids < 2
    want = moqe.moqe_routed_qgemm(X[low].contiguous(), ids[low].contiguous(), ints)
    # (other rows beside them, another kernel perhaps: within the product's own tolerance)
    assert torch.allclose(Y[low].float(), want.float(), rtol=1e-2, atol=2e-3)
    _check(Y, X, torch.where(ids >= 2, ids - 2, -1), [w for _, w in floats], [MX, NV, BF])


def test_a_block_captured_and_replayed():
    """Sort, gate and up, their product, down: one graph, replayed on new inputs and new routing, two calls on one workspace."""
    M, H, F = 48, 512, 1408
    formats = [MX, NV, BF]
    gate, up = [[_expert(10 * i + e, F, H, f) for e, f in enumerate(formats)] for i in (1, 2)]
    down = [_expert(30 + e, H, F, f) for e, f in enumerate(formats)]
    X, ids, _ = _case(1, M, 64, H, formats)
    A, B, Y = (torch.empty((M, n), dtype=torch.bfloat16, device="cuda") for n in (F, F, H))
    h = [[e for e, _ in l] for l in (gate, up, down)]
    ws = moqe.alloc_workspace(max(moqe.moqe_routed_fpgemm_workspace(M, x) for x in h))

    def step():
        _, perm, offsets = moqe.moqe_permute(None, ids, 3)
        moqe.moqe_routed_fpgemm_sorted(X, perm, offsets, h[0], A, ws)
        moqe.moqe_routed_fpgemm_sorted(X, perm, offsets, h[1], B, ws)
        C = (torch.nn.functional.silu(A.float()) * B.float()).to(torch.bfloat16)
        moqe.moqe_routed_fpgemm_sorted(C, perm, offsets, h[2], Y, ws)
        return C

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C = step()
    for seed in (2, 3, 4):
        X2, ids2, _ = _case(seed, M, 64, H, formats)
        X.copy_(X2)
        ids.copy_(ids2)
        for t in (A, B, Y):
            t.fill_(float("nan"))
        graph.replay()
        assert moqe.moqe_async_status() == moqe.OK
        _check(A, X, ids, [w for _, w in gate], formats)
        _check(B, X, ids, [w for _, w in up], formats)
        _check(Y, C, ids, [w for _, w in down], formats)
        got = Y.clone()
        step()
        assert torch.equal(got, Y)


def test_two_streams_with_workspaces_of_their_own():
    X, ids, ex = _case(9, 130, 1024, 2048, [MX, NV, BF])
    handles = [e for e, _ in ex]
    want = moqe.moqe_routed_fpgemm(X, ids, handles)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                out[i].append(moqe.moqe_routed_fpgemm(X, ids, handles))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for o in out for y in o) and moqe.moqe_async_status() == moqe.OK


def test_refusals():
    X, ids, ex = _case(6, 4, 64, 64, [MX])
    other = _expert(1, 64, 128, MX)[0]
    narrow = _expert(1, 12, 64, MX)[0]
    e = ex[0][0]
    L = moqe.lib()
    from array import array
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(4, [e]))
    Y = torch.full((4, 64), 7.0, dtype=torch.bfloat16, device="cuda")

    def call(experts, x=X.data_ptr(), y=Y.data_ptr(), w=ws.data_ptr(), size=ws.numel()):
        a = array("Q", [q.address for q in experts])
        return L.moqe_routed_fpgemm(x, ids.data_ptr(), 4, a.buffer_info()[0], len(experts), y, w, size, None)

    assert call([e, other]) == moqe.ERR_MISMATCH
    assert call([narrow]) == moqe.ERR_UNSUPPORTED                    # N % 8
    assert call([e], x=None) == moqe.ERR_NULL and call([e], y=None) == moqe.ERR_NULL
    assert call([e], x=X.data_ptr() + 8) == moqe.ERR_UNSUPPORTED and call([e], y=Y.data_ptr() + 2) == moqe.ERR_UNSUPPORTED
    assert call([e], w=None) == moqe.ERR_WORKSPACE and call([e], w=ws.data_ptr() + 16) == moqe.ERR_WORKSPACE
    assert call([e], size=moqe.moqe_routed_fpgemm_workspace(4, [e]) - 1) == moqe.ERR_WORKSPACE
    assert bool((Y == 7).all())
    with pytest.raises(moqe.MoqeError):
        moqe.moqe_routed_fpgemm(X, ids[:3], [e])
    with pytest.raises(moqe.MoqeError):
        moqe.moqe_routed_fpgemm(X, ids, [])
