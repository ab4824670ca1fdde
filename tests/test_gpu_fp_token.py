"""One row through the floating-point experts (a sequence's decode step), and a few of a small layer: every format, short and long rows,
odd sizes."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe
from test_gpu_fp_gemm import BF, MX, NV, _bf16, _check, _dev, _expert

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [MX, NV, BF])
@pytest.mark.parametrize("N,K", [(8, 8), (8, 16), (24, 24), (32, 40), (136, 72), (128, 256), (1000, 264), (264, 4096), (4096, 1032), (512, 3584), (64, 18944),
                                 (40, 65544), (8, 131072)])
def test_shapes(fmt, N, K):
    g = np.random.default_rng(N + K + fmt)
    X = _bf16(g.standard_normal((1, K)) * np.where(g.random(K) < 0.01, 30.0, 1.0))
    e, w = _expert(N + K, N, K, fmt)
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = moqe.moqe_routed_fpgemm(X, ids, [e])
    assert moqe.moqe_async_status() == moqe.OK
    _check(Y, X, ids, [w], [fmt])
    assert torch.equal(Y, moqe.moqe_routed_fpgemm(X, ids, [e]))


@pytest.mark.parametrize("M,N,K,formats", [(2, 4096, 1024, [MX, NV]), (5, 1000, 264, [BF, NV, MX]), (16, 264, 1032, [NV, MX, NV]), (64, 520, 136, [MX, BF]),
                                           (200, 8, 64, [NV, MX, BF]), (33, 136, 72, [MX] * 31 + [NV])])
def test_a_few_rows(M, N, K, formats):
    g = np.random.default_rng(M)
    ex = [_expert(M + e, N, K, f) for e, f in enumerate(formats)]
    X = _bf16(g.standard_normal((M, K)))
    ids = _dev(g.integers(-1, len(formats) + 1, M).astype(np.int32))
    Y = moqe.moqe_routed_fpgemm(X, ids, [e for e, _ in ex])
    moqe.moqe_async_status()
    _check(Y, X, ids, [w for _, w in ex], formats)
    assert bool((Y[(ids < 0) | (ids >= len(formats))] == 0).all())
    _, perm, offsets = moqe.moqe_permute(None, ids, len(formats))
    moqe.moqe_async_status()
    Z = torch.full_like(Y, 4.0)
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, [ex[1][0]]))
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[1:3], [ex[1][0]], Z, ws)
    assert torch.equal(Z[ids == 1], Y[ids == 1]) and bool((Z[ids != 1] == 4).all())


def test_routing():
    formats = [BF, MX, NV, NV, MX]
    ex = [_expert(e, 264, 520, f) for e, f in enumerate(formats)]
    h = [e for e, _ in ex]
    X = _bf16(np.random.default_rng(1).standard_normal((1, 520)))
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(1, h))
    for i in range(5):
        ids = torch.tensor([i], dtype=torch.int32, device="cuda")
        _check(moqe.moqe_routed_fpgemm(X, ids, h, workspace=ws), X, ids, [w for _, w in ex], formats)
    for i in (-1, 5):
        ids = torch.tensor([i], dtype=torch.int32, device="cuda")
        assert bool((moqe.moqe_routed_fpgemm(X, ids, h, Y=torch.full((1, 264), 2.0, dtype=torch.bfloat16, device="cuda")) == 0).all())
        assert moqe.moqe_async_status() == moqe.ERR_EXPERT_ID
    # inner experts of a sort; a segment that the row is not in
    _, perm, offsets = moqe.moqe_permute(None, torch.tensor([3], dtype=torch.int32, device="cuda"), 5)
    Y = torch.full((1, 264), 2.0, dtype=torch.bfloat16, device="cuda")
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[:4], h[:3], Y, ws)
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[4:], h[4:], Y, ws)
    assert bool((Y == 2).all())
    moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[2:5], h[2:4], Y, ws)
    _check(Y, X, torch.tensor([1], device="cuda"), [w for _, w in ex[2:4]], formats[2:4])


def test_every_pair_of_codes():
    """Weights and activations that take every e2m1 value in every pairing: exact sums."""
    grid = np.concatenate([R.E2M1, -R.E2M1])
    K = 512
    x = np.tile(np.repeat(grid, 16), 2)[None, :K]
    W = np.stack([np.roll(np.tile(grid, 32), s) for s in range(16)])[:, :K]
    W[:, ::16] = 6.0
    x[:, 5::16] = 6.0                                          # every block has its largest number, so that its scale is known
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    for fmt in (MX, NV):
        X = _bf16(x)
        w = R.encode(W.astype(np.float32), fmt)[3]
        xq = R.encode(X.float().cpu().numpy(), fmt)[3]
        want = torch.from_numpy((xq @ w.T).astype(np.float32)).to(torch.bfloat16)
        got = moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(W.astype(np.float32)), fmt)])
        # (sums of multiples of 2^-4 below 2^15 are exact in fp32 whatever their order: only the rounding to bf16 is left)
        assert torch.equal(got.cpu(), want)


def test_infinities_nan_and_extreme_scales():
    g = np.random.default_rng(2)
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    for fmt in (MX, NV, BF):
        W = g.standard_normal((72, 200)).astype(np.float32)
        W2 = W.copy()
        W2[9, 100], W2[71, 199] = np.nan, np.inf
        X = _bf16(g.standard_normal((1, 200)))
        a, b = (moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(w), fmt)])[0] for w in (W, W2))
        bad = torch.zeros(72, dtype=torch.bool, device="cuda")
        bad[[9, 71]] = True
        assert not bool(torch.isfinite(b[bad]).any()) and torch.equal(a[~bad], b[~bad])
        X[0, 150] = float("nan")
        assert bool(torch.isnan(moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(W), fmt)])).all())
    for fmt in (MX, NV):
        for up, down in ((100.0, -100.0), (-100.0, 100.0), (40.0, 40.0), (-60.0, -60.0)):
            W = (g.standard_normal((40, 264)) * 2.0 ** up).astype(np.float32)
            X = _bf16(g.standard_normal((1, 264)) * 2.0 ** down)
            Y = moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(_dev(W), fmt)])
            _check(Y, X, ids, [_dev(R.encode(W, fmt)[3])], [fmt])


def test_decoding_step_in_a_graph():
    """One sequence's block, captured: the routing changes between replays."""
    H, F = 1024, 2816
    formats = [MX, NV, BF]
    gate, down = [_expert(e, F, H, f) for e, f in enumerate(formats)], [_expert(9 + e, H, F, f) for e, f in enumerate(formats)]
    hg, hd = [e for e, _ in gate], [e for e, _ in down]
    X = _bf16(np.random.default_rng(3).standard_normal((1, H)))
    logits = torch.zeros((1, 3), device="cuda")
    A, Y = torch.empty((1, F), dtype=torch.bfloat16, device="cuda"), torch.empty((1, H), dtype=torch.bfloat16, device="cuda")
    ws = moqe.alloc_workspace(max(moqe.moqe_routed_fpgemm_workspace(1, h) for h in (hg, hd)))

    def step():
        _, _, perm, offsets = moqe.moqe_route_permute(logits, None, 1)
        moqe.moqe_routed_fpgemm_sorted(X, perm, offsets, hg, A, ws)
        moqe.moqe_routed_fpgemm_sorted(A, perm, offsets, hd, Y, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for e in (2, 0, 1, 1, 0):
        logits.zero_()
        logits[0, e] = 1.0
        Y.fill_(float("nan"))
        graph.replay()
        ids = torch.tensor([e], dtype=torch.int32, device="cuda")
        _check(A, X, ids, [w for _, w in gate], formats)
        _check(Y, A, ids, [w for _, w in down], formats)
    assert moqe.moqe_async_status() == moqe.OK
