"""Floating-point experts where they can go wrong: odd numbers of channel tiles under pairs of SMs, formats that change inside a worker's
share, memory beside outputs and workspaces, segments that do not begin at row 0, graphs that share a workspace, long rows."""
import numpy as np
import pytest
import torch

import fp_reference as R
import paper_2508_09204_b200 as moqe
from test_gpu_fp_gemm import BF, MX, NV, _bf16, _case, _check, _dev, _expert

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,formats,counts", [
    (2600, 1544, 264, [BF, NV, MX, NV], None),                   # 13 channel tiles: a pair's last one is half empty
    (3000, 648, 520, [NV, BF, NV, MX], [2000, 600, 399, 1]),
    (2304, 4096, 136, [MX], None),                               # one k-block to a tile
    (1300, 3584, 1032, [BF], None),
    (1041, 2048, 2056, [NV, MX], [1040, 1]),                     # five equal token tiles, and one row
    (5000, 1000, 72, [MX, NV, BF, BF, NV, MX], [0, 4000, 1, 0, 999, 0]),
    (70000, 8, 64, [NV, MX], None),
    (129, 8, 128, [MX] * 32, None),
    (16, 136, 65544, [NV, MX, BF], None),                        # rows beyond a block's registers
    (1, 8, 131072, [NV], None),
    (127, 4096, 512, [BF, MX], [63, 64]),
])
def test_shapes(M, N, K, formats, counts):
    X, ids, ex = _case(M + N, M, N, K, formats, counts)
    Y = moqe.moqe_routed_fpgemm(X, ids, [e for e, _ in ex])
    assert moqe.moqe_async_status() == moqe.OK
    _check(Y, X, ids, [w for _, w in ex], formats)


@pytest.mark.parametrize("M", [7, 60, 100, 400, 2000])
def test_nothing_beside_the_outputs_is_written(M):
    N, K = 1032, 520
    X, ids, ex = _case(M, M, N, K, [NV, BF, MX])
    handles = [e for e, _ in ex]
    n = moqe.moqe_routed_fpgemm_workspace(M, handles)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    big = torch.full((M + 16, N), 9.0, dtype=torch.bfloat16, device="cuda")
    moqe.moqe_routed_fpgemm(X, ids, handles, Y=big[8:8 + M], workspace=ws[:n])
    assert moqe.moqe_async_status() == moqe.OK
    assert bool((big[:8] == 9).all()) and bool((big[8 + M:] == 9).all()) and bool((ws[n:] == 0x5A).all())
    _check(big[8:8 + M], X, ids, [w for _, w in ex], [NV, BF, MX])
    # rows in a 4-bit format: outputs that are slices of larger buffers
    for fmt in (MX, NV):
        nb = -(-K // R.BLOCK[fmt])
        codes, scales = torch.full((M * K // 2 + 32,), 7, dtype=torch.uint8, device="cuda"), torch.full((M * nb + 32,), 7, dtype=torch.uint8, device="cuda")
        outer, values = torch.full((M + 8,), 7.0, device="cuda"), torch.full((M * K + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        for v in (values.data_ptr(), None):
            assert moqe.lib().moqe_fp4_quantize_rows(X.data_ptr(), M, K, fmt, codes.data_ptr(), scales.data_ptr(), outer.data_ptr(), v, st) == moqe.OK
        assert all(bool((t[-k:] == 7).all()) for t, k in ((codes, 32), (scales, 32), (outer, 8), (values, 16)))
        assert fmt == NV or bool((outer == 7).all())                       # MXFP4 has no row scale
        got = moqe.moqe_fp4_quantize_rows(X, fmt, values=True)
        assert torch.equal(codes[:-32].view(M, -1), got[0]) and torch.equal(scales[:-32].view(M, -1), got[1]) and torch.equal(values[:-16].view(M, K), got[3])


@pytest.mark.parametrize("M", [20, 90, 700, 3000])
def test_segments_that_do_not_begin_at_row_0(M):
    N, K = 1544, 392
    X, ids, ex = _case(M, M, N, K, [MX, NV, BF, NV])
    handles = [e for e, _ in ex]
    _, perm, offsets = moqe.moqe_permute(None, ids, 4)
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, handles))
    for a, b in ((1, 3), (2, 4), (1, 2), (3, 4)):
        Y = torch.full((M, N), 3.0, dtype=torch.bfloat16, device="cuda")
        moqe.moqe_routed_fpgemm_sorted(X, perm, offsets[a:b + 1], handles[a:b], Y, ws)
        inside = (ids >= a) & (ids < b)
        assert bool((Y[~inside] == 3).all())
        _check(Y, X, torch.where(inside, ids - a, -1), [w for _, w in ex[a:b]], [MX, NV, BF, NV][a:b])
    assert moqe.moqe_async_status() == moqe.OK


def test_two_graphs_on_one_workspace():
    """Captured calls of other sizes and formats, replayed in turn on one workspace and between eager calls."""
    cases = [(_case(1, 16, 1024, 2048, [MX, NV])), (_case(2, 300, 1024, 1032, [BF, NV, MX])), (_case(3, 2100, 1160, 264, [NV, BF]))]
    formats = [[MX, NV], [BF, NV, MX], [NV, BF]]
    ws = moqe.alloc_workspace(max(moqe.moqe_routed_fpgemm_workspace(c[0].shape[0], [e for e, _ in c[2]]) for c in cases))
    out, graphs = [], []
    for X, ids, ex in cases:
        h = [e for e, _ in ex]
        Y = torch.empty((X.shape[0], ex[0][0].N), dtype=torch.bfloat16, device="cuda")
        moqe.moqe_routed_fpgemm(X, ids, h, Y=Y, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            moqe.moqe_routed_fpgemm(X, ids, h, Y=Y, workspace=ws)
        out.append((Y, Y.clone()))
        graphs.append(g)
    for i in (0, 1, 2, 0, 2, 1, 1, 0, 0):
        out[i][0].fill_(float("nan"))
        graphs[i].replay()
        assert torch.equal(out[i][0], out[i][1])
        ws.fill_(255)
    for (X, ids, ex), f, (Y, _) in zip(cases, formats, out):
        _check(Y, X, ids, [w for _, w in ex], f)
    assert moqe.moqe_async_status() == moqe.OK


def test_an_expert_built_just_before_its_product():
    """Build, quantize and multiply in a row on one stream, many times: the product's weights are read before its rows are there."""
    g = np.random.default_rng(3)
    X = _bf16(g.standard_normal((9, 1024)))
    ids = torch.zeros(9, dtype=torch.int32, device="cuda")
    W = [_dev((g.standard_normal((512, 1024)) * 0.02).astype(np.float32)) for _ in range(4)]
    want = [moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(w, f)]) for w, f in zip(W, (MX, NV, BF, NV))]
    torch.cuda.synchronize()
    for _ in range(10):
        keep = []
        got = []
        for w, f in zip(W, (MX, NV, BF, NV)):
            keep.append(moqe.moqe_fp_quantize(w, f))
            got.append(moqe.moqe_routed_fpgemm(X, ids, [keep[-1]]))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_do_not_depend_on_their_company():
    """A row's output is the same bits in a small batch and in a large one, as long as nothing is split along k and both take the same
    kernel (a few rows of a small layer have one of their own, which shares a row's sum among fewer warps the more rows there are)."""
    for fmt in (MX, NV, BF):
        e, w = _expert(5, 2048, 512, fmt)
        X = _bf16(np.random.default_rng(6).standard_normal((3000, 512)))
        ids = torch.zeros(3000, dtype=torch.int32, device="cuda")
        Y = moqe.moqe_routed_fpgemm(X, ids, [e])
        for rows in (slice(5, 45), slice(100, 230), slice(0, 700)):
            assert torch.equal(moqe.moqe_routed_fpgemm(X[rows].contiguous(), ids[rows].contiguous(), [e]), Y[rows])


def test_random_routings_and_sizes():
    """Forty small calls of random sizes, formats and routings."""
    r = np.random.default_rng(99)
    for i in range(40):
        M, N, K = int(np.exp(r.uniform(0, 6.5))), 8 * int(r.integers(1, 80)), 8 * int(r.integers(1, 200))
        formats = [int(f) for f in r.integers(1, 4, int(r.integers(1, 6)))]
        X, ids, ex = _case(1000 + i, M, N, K, formats)
        Y = moqe.moqe_routed_fpgemm(X, ids, [e for e, _ in ex])
        _check(Y, X, ids, [w for _, w in ex], formats)
    assert moqe.moqe_async_status() == moqe.OK


@pytest.mark.parametrize("fmt", [MX, NV, BF])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_far_scales(fmt, M):
    """A power of two on the weights and one on the rows come out as their product, to the bit: nothing on the way leaves fp32's range
    as long as neither the sums nor the outputs do.  (One row takes a kernel of its own.)"""
    N, K = 4096, 1024
    g = np.random.default_rng(M)
    W, X = g.standard_normal((N, K)).astype(np.float32), g.standard_normal((M, K)).astype(np.float32)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    run = lambda w, x: moqe.moqe_routed_fpgemm(_bf16(x), ids, [moqe.moqe_fp_quantize(_dev(w), fmt)])
    Y = run(W, X).double()
    for a, b in ((100, -100), (-100, 100), (50, 40), (-30, -30)):
        assert torch.equal(run(np.ldexp(W, a), np.ldexp(X, b)).double(), Y * 2.0 ** (a + b)), (a, b)
    # sums of zeros under scales whose product is beyond fp32
    W[:, ::2] = 0
    X[:, 1::2] = 0
    assert bool((run(np.ldexp(W, 100), np.ldexp(X, 100)) == 0).all())


def test_an_imported_outer_scale_meets_small_rows():
    """The channel's scale goes to the sum first: its product with a small row's alone would be below fp32's normal numbers."""
    N, K = 256, 512
    g = np.random.default_rng(9)
    e0 = moqe.moqe_fp_quantize(_dev(g.standard_normal((N, K)).astype(np.float32)), NV)
    codes, scales, _, _ = moqe.moqe_fp_expert_export(e0)
    outer = (1 + g.random(N)).astype(np.float32)
    X = g.standard_normal((200, K)).astype(np.float32)
    for M in (1, 200):
        ids = torch.zeros(M, dtype=torch.int32, device="cuda")
        run = lambda a, b: moqe.moqe_routed_fpgemm(_bf16(np.ldexp(X[:M], b)), ids, [moqe.moqe_fp_expert_import(NV, codes, scales, _dev(np.ldexp(outer, a)))])
        assert torch.equal(run(30, -114).double(), run(0, 0).double() * 2.0 ** -84)
        assert torch.equal(run(-40, -60).double(), run(0, 0).double() * 2.0 ** -100)


def test_products_beyond_the_schedule_are_refused():
    """(before a pointer is looked at)"""
    import ctypes as C
    L, p = moqe.lib(), 0x10000
    e = moqe.moqe_fp_quantize(torch.zeros(65536, 4096, device="cuda"), BF)
    arr = (C.c_void_p * 1)(e.handle)
    for M in (2 ** 31 - 1, 2 ** 30 + 1, 2 ** 24):
        assert L.moqe_routed_fpgemm_workspace(M, arr, 1) == 0
        assert L.moqe_routed_fpgemm(p, p, M, arr, 1, p, p, 2 ** 62, None) == moqe.ERR_UNSUPPORTED
        assert L.moqe_routed_fpgemm_sorted(p, p, p, M, arr, 1, p, p, 2 ** 62, None) == moqe.ERR_UNSUPPORTED
    assert L.moqe_routed_fpgemm_workspace(2 ** 20, arr, 1) > 0


def test_a_workspace_for_many_rows_serves_fewer():
    for formats in ([NV], [MX, BF], [NV] * 31 + [BF]):
        for N in (128, 512, 11008):
            ex = [moqe.moqe_fp_quantize(torch.zeros(N, 256, device="cuda"), f) for f in formats]
            sizes = [moqe.moqe_routed_fpgemm_workspace(M, ex) for M in sorted([*range(1, 300), *range(300, 20000, 37), 9344, 9345, 9472, 9473])]
            assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("M,K", [(1100, 8200), (300, 32768), (300, 32776), (20000, 456), (9100, 1000)])
def test_many_rows_with_infinities_and_rows_of_nobody(M, K):
    """Rows that a ring in shared memory takes, on both sides of its limits: every format in turn, blocks that are NaN, zeros."""
    N, formats = 136, [NV, MX, BF, NV]
    g = np.random.default_rng(M)
    ex = [_expert(e, N, K, f) for e, f in enumerate(formats)]
    x = g.standard_normal((M, K)).astype(np.float32)
    x[5::97] = 0
    x[7::101] *= 1e-38
    X = _bf16(x)
    ids = _dev(g.integers(-1, 5, M).astype(np.int32))
    handles = [e for e, _ in ex]
    Y = moqe.moqe_routed_fpgemm(X, ids, handles)
    moqe.moqe_async_status()
    _check(Y, X, ids, [w for _, w in ex], formats)
    bad = torch.arange(3, M, 50, device="cuda")
    X[bad, torch.randint(0, K, bad.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))] = float("inf")
    Z = moqe.moqe_routed_fpgemm(X, ids, handles)
    moqe.moqe_async_status()
    good = torch.ones(M, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.equal(Z[good], Y[good])
    hit = bad[(ids[bad] >= 0) & (ids[bad] < 4)]
    four = hit[ids[hit] != 2]
    assert bool(Z[four].isnan().all()) and not bool(Z[hit].isfinite().any())


def test_many_rows_captured_with_inputs_that_change():
    """The rows' ring, the schedule and a sort in one graph, replayed with other rows and another routing; X from a 16-byte boundary only."""
    M, N, K = 2304, 264, 4104
    g = np.random.default_rng(21)
    ex = [_expert(e, N, K, f) for e, f in enumerate([NV, BF, MX])]
    handles = [e for e, _ in ex]
    X = torch.zeros(M * K + 8, dtype=torch.bfloat16, device="cuda")[8:].view(M, K)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    Y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, handles))
    moqe.moqe_routed_fpgemm(X, ids, handles, Y=Y, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moqe.moqe_routed_fpgemm(X, ids, handles, Y=Y, workspace=ws)
    for _ in range(4):
        X.copy_(_bf16(g.standard_normal((M, K))))
        ids.copy_(_dev(g.integers(0, 3, M).astype(np.int32)))
        Y.fill_(float("nan"))
        graph.replay()
        _check(Y, X, ids, [w for _, w in ex], [NV, BF, MX])
    assert moqe.moqe_async_status() == moqe.OK


@pytest.mark.parametrize("M", [130, 2500])
def test_an_expert_built_just_before_a_larger_product(M):
    N, K = 1032, 4096
    g = np.random.default_rng(M)
    X = _bf16(g.standard_normal((M, K)))
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    formats = (MX, NV, BF, NV)
    W = [_dev((g.standard_normal((N, K)) * 0.02).astype(np.float32)) for _ in formats]
    ws = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, [moqe.moqe_fp_quantize(W[0], BF)]) + moqe.moqe_routed_fpgemm_workspace(M, [moqe.moqe_fp_quantize(W[1], NV)]))
    want = [moqe.moqe_routed_fpgemm(X, ids, [moqe.moqe_fp_quantize(w, f)]) for w, f in zip(W, formats)]
    torch.cuda.synchronize()
    for _ in range(6):
        keep = [moqe.moqe_fp_quantize(W[0], MX)]
        got = []
        for w, f in zip(W, formats):
            keep.append(moqe.moqe_fp_quantize(w, f))
            got.append(moqe.moqe_routed_fpgemm(X, ids, [keep[-1]], workspace=ws))
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert moqe.moqe_async_status() == moqe.OK
