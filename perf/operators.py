"""The floating-point experts' operators as cases that can be timed and compared.

A case is one of three kinds:

  rows    : activations quantized to a microscaled 4-bit format, row by row: what a row's product with such an expert sees.
  expert  : one expert built from full-precision weights and exported for storage.
  product : one routed linear layer for a sorted batch.  Rows of an expert in a 4-bit format are quantized to that format in the
            call; rows of a bf16 expert stay as they are.

Formats: "mxfp4" (blocks of 32, power-of-two scales), "nvfp4" (blocks of 16, e4m3 scales, a power-of-two scale for each row) and
"bf16" (the unquantized model as an expert).

The plain forms are elementary torch operations in 32 bits.  Codes and scales are fixed by the formats' definitions: every
quotient that is rounded is either exact in 32 bits or never so near to a border that its own rounding would matter.
"""
import math

import torch

own = False

BLOCK = {"mxfp4": 32, "nvfp4": 16}
# how the rows of a batch spread over the experts, most loaded first
MIXES = {"even": None, "skewed": (0.7, 0.2, 0.1), "one": (1.0,)}
# (N, K) of the layers of a LLaMA-7B-shaped and a Qwen2.5-7B-shaped block
LAYERS = ((4096, 4096), (11008, 4096), (4096, 11008), (3584, 3584), (512, 3584), (18944, 3584), (3584, 18944))
LARGEST = 16384 * 11008 * 4096


def listed():
    return [
        # a decode step's rows on their way into a 4-bit layer: the smallest call
        {"name": "rows_mx_16x4096", "kind": "rows", "format": "mxfp4", "M": 16, "K": 4096},
        # uneven prompts of odd length, whose last blocks are short
        {"name": "rows_nv_1001x3592", "kind": "rows", "format": "nvfp4", "M": 1001, "K": 3592},
        # full-length prompts before the widest layer
        {"name": "rows_mx_16384x11008", "kind": "rows", "format": "mxfp4", "M": 16384, "K": 11008},
        # building a model's experts, one layer at a time: a wide layer, and grouped-query attention's narrow one
        {"name": "expert_nv_11008x4096", "kind": "expert", "format": "nvfp4", "N": 11008, "K": 4096},
        {"name": "expert_mx_512x3584", "kind": "expert", "format": "mxfp4", "N": 512, "K": 3584},
        # one user's generation, a token at a time
        {"name": "token_llama_1", "kind": "product", "M": 1, "N": 4096, "K": 11008, "experts": "mxfp4 nvfp4", "mix": "one"},
        # a small server's decode step over all three formats
        {"name": "decode_llama_16", "kind": "product", "M": 16, "N": 11008, "K": 4096, "experts": "mxfp4 nvfp4 bf16", "mix": "even"},
        # a busy server's decode step
        {"name": "decode_qwen_96", "kind": "product", "M": 96, "N": 18944, "K": 3584, "experts": "mxfp4 nvfp4", "mix": "even"},
        # a ragged batch on a layer of odd sizes
        {"name": "ragged_777", "kind": "product", "M": 777, "N": 1000, "K": 2056, "experts": "nvfp4 bf16 mxfp4", "mix": "skewed"},
        # prompts beside decoding sequences, four experts
        {"name": "mixed_qwen_4160", "kind": "product", "M": 4160, "N": 3584, "K": 18944, "experts": "mxfp4 nvfp4 nvfp4 bf16", "mix": "even"},
        # the unquantized model's share of a batch of prompts
        {"name": "prompts_bf16_8192", "kind": "product", "M": 8192, "N": 4096, "K": 4096, "experts": "bf16 bf16", "mix": "skewed"},
        # full-length prompts, most of them easy ones
        {"name": "prefill_llama_16384", "kind": "product", "M": 16384, "N": 11008, "K": 4096, "experts": "mxfp4 nvfp4 mxfp4", "mix": "skewed"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rows", "expert", "product", "product", "product"))
    if kind == "rows":
        return {"kind": kind, "format": rng.choice(("mxfp4", "nvfp4")), "M": _log(rng, 1, 16384), "K": 8 * _log(rng, 4, 1376)}
    if kind == "expert":
        N, K = rng.choice((rng.choice(LAYERS), (8 * _log(rng, 8, 1376), 8 * _log(rng, 8, 512))))
        return {"kind": kind, "format": rng.choice(("mxfp4", "nvfp4")), "N": N, "K": K}
    N, K = rng.choice((rng.choice(LAYERS), (8 * _log(rng, 8, 1376), 8 * _log(rng, 8, 1376))))
    M = min(_log(rng, 1, 16384), LARGEST // (N * K))
    experts = rng.choice(("mxfp4", "nvfp4 mxfp4", "mxfp4 nvfp4 bf16", "bf16 bf16", "nvfp4 nvfp4 mxfp4 mxfp4", "bf16 mxfp4 nvfp4 mxfp4 nvfp4"))
    return {"kind": kind, "M": M, "N": N, "K": K, "experts": experts, "mix": rng.choice(("even", "even", "skewed", "one"))}


# ---- the formats, in 32 bits ---------------------------------------------------------------------------------------
def _blocks(x, size):
    """[R][K] -> [R][blocks][size], the last block filled up with zeros."""
    short = -x.shape[1] % size
    if short:
        x = torch.cat((x, x.new_zeros(x.shape[0], short)), 1)
    return x.view(x.shape[0], -1, size)


def _floor_log2(a):
    return torch.frexp(a)[1] - 1


def _pow2(e):
    """2^e in fp32, exactly, for whole -149 <= e <= 127."""
    return torch.where(e >= -126, (e + 127) << 23, 1 << torch.clamp(e + 149, 0, 22)).to(torch.int32).view(torch.float32)


def _magnitude(q):
    """Index of the e2m1 number nearest to q >= 0, ties to the even index."""
    return ((q > 0.25).to(torch.uint8) + (q >= 0.75) + (q > 1.25) + (q >= 1.75) + (q > 2.5) + (q >= 3.5) + (q > 5.0)).to(torch.uint8)


def _e4m3(v):
    """Nearest e4m3 number to 0 <= v <= 448, ties to even: (byte, value)."""
    e = torch.clamp(_floor_log2(torch.clamp(v, min=2.0 ** -9)), min=-6)
    n = torch.round(v * _pow2(3 - e)).to(torch.int32)                            # 0..16 eighths of 2^e
    return (n + (e + 6) * 8).to(torch.uint8), n.float() * _pow2(e - 3)


def _encode(x, fmt):
    """fp32 [R][K] (finite) -> codes uint8 [R][blocks][size] (one a byte), scale bytes [R][blocks], row scales [R], scale values."""
    b = _blocks(x, BLOCK[fmt])
    amax = b.abs().amax(2)
    if fmt == "mxfp4":
        e = torch.where(amax > 0, torch.clamp(_floor_log2(amax) - 2, min=-127), -127)
        byte, outer, s = (e + 127).to(torch.uint8), None, _pow2(e)
        q = b.abs() * _pow2(-e)[:, :, None]
    else:
        top = amax.amax(1)
        r = torch.where(top > 0, torch.clamp(_floor_log2(top) - 10, min=-126), 0)
        outer = _pow2(r)
        byte, s = _e4m3(amax * _pow2(-r)[:, None] / 6.0)
        q = b.abs() * _pow2(-r)[:, None, None] / torch.where(s > 0, s, 1.0)[:, :, None]
        q = torch.where(s[:, :, None] > 0, q, 0.0)
    return _magnitude(q) + (torch.signbit(b).to(torch.uint8) << 3), byte, outer, s


def _numbers(codes):
    """What e2m1 codes stand for."""
    m, sign = codes & 7, 1.0 - 2.0 * (codes >> 3).float()
    mag = torch.where(m < 2, m.float() * 0.5, (1.0 + 0.5 * (m & 1).float()) * _pow2((m >> 1).int() - 1))
    return mag * sign


def _as_float8(byte, fmt):
    return byte.view(torch.float8_e8m0fnu if fmt == "mxfp4" else torch.float8_e4m3fn)


def _values(x, fmt):
    """The fp32 values that x is rounded to, and its scales."""
    codes, byte, outer, s = _encode(x, fmt)
    v = _numbers(codes) * s[:, :, None]
    v = v.reshape(x.shape[0], -1)[:, :x.shape[1]]
    return (v if outer is None else v * outer[:, None]), byte, outer


def _pack(codes, K):
    c = codes.reshape(codes.shape[0], -1)[:, :K]
    return (c[:, 0::2] | (c[:, 1::2] << 4)).contiguous()


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), 2).reshape(packed.shape[0], -1)


def _scale_values(byte, fmt):
    if fmt == "mxfp4":
        return _pow2(byte.int() - 127)
    e = (byte >> 3).int()
    return ((byte & 7).float() + 8.0 * (e > 0)) * _pow2(torch.clamp(e, min=1) - 10)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _acts(g, M, K):
    """Activations of a transformer: normal, a few channels far larger than the rest, and a padding row of zeros now and then."""
    x = torch.randn((M, K), device="cuda", generator=g)
    x *= torch.where(torch.rand((K,), device="cuda", generator=g) < 0.004, 20.0, 1.0)
    x *= (torch.rand((M, 1), device="cuda", generator=g) >= 0.003) | (torch.arange(M, device="cuda")[:, None] == 0)
    return x.to(torch.bfloat16)


def _weights(g, N, K):
    return torch.randn((N, K), device="cuda", generator=g).mul_(0.02)


def _counts(case):
    """How many of the rows go to each expert."""
    M, E = case["M"], len(case["experts"].split())
    p = list(MIXES[case["mix"]] or (1.0 / E,) * E)[:E]
    p += [0.0] * (E - len(p))
    n = [int(M * x / sum(p) + 1e-9) for x in p]
    n[0] += M - sum(n)
    return n


def _stored(W, fmt):
    """An expert as a checkpoint holds it."""
    if fmt == "bf16":
        return {"format": fmt, "values": W.to(torch.bfloat16)}
    codes, byte, outer, _ = _encode(W, fmt)
    return {"format": fmt, "codes": _pack(codes, W.shape[1]), "scales": byte, "outer": outer}


def prepare(case, seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    if case["kind"] == "rows":
        return {"kind": "rows", "format": case["format"], "X": _acts(g, case["M"], case["K"])}
    if case["kind"] == "expert":
        return {"kind": "expert", "format": case["format"], "W": _weights(g, case["N"], case["K"])}
    M, N, K = case["M"], case["N"], case["K"]
    stored = [_stored(_weights(g, N, K), f) for f in case["experts"].split()]
    counts = _counts(case)
    ids = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), torch.tensor(counts, device="cuda"))
    ids = ids[torch.randperm(M, device="cuda", generator=g)]
    offsets = [sum(counts[:e]) for e in range(len(counts) + 1)]
    s = {"kind": "product", "X": _acts(g, M, K), "stored": stored, "N": N, "counts": counts,
         "perm": torch.argsort(ids, stable=True).to(torch.int32), "offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda")}
    if own:
        import paper_2508_09204_b200 as moqe
        s["experts"] = [moqe.moqe_fp_expert_import(_format(x["format"]), codes=x.get("codes"), scales=x.get("scales"),
                                                   outer=x.get("outer"), values=x.get("values")) for x in stored]
        s["Y"] = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        s["workspace"] = moqe.alloc_workspace(moqe.moqe_routed_fpgemm_workspace(M, s["experts"]))
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def _format(fmt):
    import paper_2508_09204_b200 as moqe
    return {"mxfp4": moqe.FP_MXFP4, "nvfp4": moqe.FP_NVFP4, "bf16": moqe.FP_BF16}[fmt]


def _answer(values, byte, outer, fmt):
    return {"values": values, "scales": _as_float8(byte, fmt), "outer": outer}


def _run_own(s):
    import paper_2508_09204_b200 as moqe
    if s["kind"] == "rows":
        _, byte, outer, values = moqe.moqe_fp4_quantize_rows(s["X"], _format(s["format"]), values=True)
        return _answer(values, byte, outer, s["format"])
    if s["kind"] == "expert":
        _, byte, outer, values = moqe.moqe_fp_expert_export(moqe.moqe_fp_quantize(s["W"], _format(s["format"])), values=True)
        return _answer(values, byte, outer, s["format"])
    return moqe.moqe_routed_fpgemm_sorted(s["X"], s["perm"], s["offsets"], s["experts"], s["Y"], s["workspace"])


def _expert_values(x):
    """The fp32 weights of a stored expert."""
    if x["format"] == "bf16":
        return x["values"].float()
    v = _blocks(_numbers(_unpack(x["codes"])), BLOCK[x["format"]]) * _scale_values(x["scales"], x["format"])[:, :, None]
    v = v.reshape(v.shape[0], -1)[:, :2 * x["codes"].shape[1]]
    return v if x["outer"] is None else v * x["outer"][:, None]


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "rows":
        v, byte, outer = _values(s["X"].float(), s["format"])
        return _answer(v.to(torch.bfloat16), byte, outer, s["format"])
    if s["kind"] == "expert":
        v, byte, outer = _values(s["W"], s["format"])
        return _answer(v.to(torch.bfloat16), byte, outer, s["format"])
    Y = torch.empty((s["X"].shape[0], s["N"]), dtype=torch.bfloat16, device=s["X"].device)
    for rows, x in zip(torch.split(s["perm"].long(), s["counts"]), s["stored"]):
        if rows.numel():
            a = s["X"][rows].float()
            a = a if x["format"] == "bf16" else _values(a, x["format"])[0]
            Y[rows] = (a @ _expert_values(x).t()).to(torch.bfloat16)
    return Y


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest(q, grid):
    """Index into the ascending list `grid` of the number nearest to q >= 0; of two equally near, the even one."""
    t = torch.tensor(grid, dtype=torch.float64, device=q.device)
    i = torch.clamp(torch.searchsorted(t, q.contiguous(), right=True) - 1, 0, len(grid) - 2)
    below, above = q - t[i], t[i + 1] - q
    return i + ((above < below) | ((above == below) & (i % 2 == 1))).long()


def _power(e):
    return ((e + 1023) << 52).view(torch.float64)


def _exponent(a):
    """floor(log2 a) of positive numbers that are normal in 64 bits."""
    return (a.contiguous().view(torch.int64) >> 52) - 1023


def _defined(x, fmt):
    """Scales and values of a matrix, block by block, as the formats define them."""
    x = x.double()
    size = BLOCK[fmt]
    values, scales = torch.zeros_like(x), []
    outer = None
    if fmt == "nvfp4":
        top = x.abs().max(1).values
        outer = torch.where(top > 0, _power(torch.clamp(_exponent(top) - 10, min=-126)), 1.0)
        e4m3 = [i * 2.0 ** -9 for i in range(8)] + [(8 + i) * 2.0 ** (e - 3) for e in range(-6, 9) for i in range(8)][:119]
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    for k in range(0, x.shape[1], size):
        part = x[:, k:k + size]
        amax = part.abs().max(1).values
        if fmt == "mxfp4":
            s = whole = _power(torch.clamp(_exponent(amax) - 2, min=-127))
        else:
            s = torch.tensor(e4m3, dtype=torch.float64, device=x.device)[_nearest(amax / outer / 6.0, e4m3)]
            whole = s * outer
        q = torch.where(whole > 0, part.abs().t() / torch.where(whole > 0, whole, 1.0), 0.0).t()
        values[:, k:k + size] = grid[_nearest(q, _GRID)] * whole[:, None] * torch.where(torch.signbit(part), -1.0, 1.0)
        scales.append(s)
    return values, torch.stack(scales, 1), outer


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] != "product":
        x = s["X"] if s["kind"] == "rows" else s["W"]
        values, scales, outer = _defined(x, s["format"])
        return {"values": values, "scales": scales, "outer": outer}
    grid = torch.tensor(_GRID + tuple(-v for v in _GRID), dtype=torch.float64, device="cuda")
    Y = torch.zeros((case["M"], case["N"]), dtype=torch.float64, device="cuda")
    order, at = s["perm"].long(), 0
    for n, x in zip(s["counts"], s["stored"]):
        rows, at = order[at:at + n], at + n
        if n == 0:
            continue
        if x["format"] == "bf16":
            Y[rows] = s["X"][rows].double() @ x["values"].double().t()
            continue
        W = torch.empty((case["N"], case["K"]), dtype=torch.float64, device="cuda")
        W[:, 0::2], W[:, 1::2] = grid[(x["codes"] & 15).long()], grid[(x["codes"] >> 4).long()]
        scales = _as_float8(x["scales"], x["format"]).to(torch.float64)
        W *= torch.repeat_interleave(scales, BLOCK[x["format"]], 1)[:, :case["K"]]
        if x["outer"] is not None:
            W *= x["outer"].double()[:, None]
        Y[rows] = _defined(s["X"][rows], x["format"])[0] @ W.t()
    return Y


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def _bytes(R, K, fmt):
    """Codes and scales of a matrix."""
    if fmt == "bf16":
        return 2 * R * K
    return R * K // 2 + R * -(-K // BLOCK[fmt]) + (4 * R if fmt == "nvfp4" else 0)


def work(case):
    if case["kind"] == "rows":
        M, K = case["M"], case["K"]
        return {"bytes": 2 * M * K + _bytes(M, K, case["format"]) + 2 * M * K, "flops": 0}
    if case["kind"] == "expert":
        N, K = case["N"], case["K"]
        return {"bytes": 4 * N * K + 2 * _bytes(N, K, case["format"]) + 2 * N * K, "flops": 0}
    M, N, K = case["M"], case["N"], case["K"]
    weights = sum(_bytes(N, K, f) for f, n in zip(case["experts"].split(), _counts(case)) if n)
    return {"bytes": weights + 2 * M * K + 2 * M * N, "flops": 2 * M * N * K}
