"""Operators between the int8 products of a transformer block, as cases that can be prepared, run and checked one by one.

What an inference program does around int8 layers, in its plain form (``own`` false: elementary torch operations in 32 bits)
or through this library's entry points (``own`` true):

* ``norm``         the residual's addition and a root-mean-square norm, both results in 16 bits; 1 .. 8192 tokens of 64 .. 16384
                   values, odd widths and rows inside of larger ones among them, with a residual or without.
* ``norm_linear``  the same norm with its result in int8 and a scale per token, and the int8 layer that takes it (how a program has the
                   int8 form); 1 .. 8192 tokens, widths 64 .. 8192.
* ``add``          an int8 linear layer with bias, activation and the residual's addition behind it: a block's output projections;
                   M 1 .. 8192, N and K 64 .. 16384 (odd widths and row-major weights: M up to 2048, N and K up to 4096).
* ``gated``        both projections of a gated feed-forward block with the activation and the product of the two, from 16-bit
                   activations or from int8 ones with their scales (what the norm leaves); the same range.

The quantisation rule: for a token's values, rounded to 16 bits, with the largest magnitude a, the scale is a / 127 and the integers
are 127 x / a, rounded to nearest, halves away from zero; a row of zeros has the scale zero.  The protection scheme of the products is
the library's own choice; the sticky fault flag comes back with the result.
"""
import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------------------------ #
# the cases
# ------------------------------------------------------------------------------------------------------------------ #
def listed():
    return [
        # decoding one token: latency
        {"name": "norm_1x4096", "kind": "norm", "dtype": "bf16", "M": 1, "K": 4096, "pad": 0, "residual": True},
        # a width that fills no 16-byte chunk, rows inside of larger ones, no residual yet: a first block's norm
        {"name": "norm_1001x2047_strided", "kind": "norm", "dtype": "f16", "M": 1001, "K": 2047, "pad": 130, "residual": False},
        # prompts: bytes
        {"name": "norm_8192x8192", "kind": "norm", "dtype": "bf16", "M": 8192, "K": 8192, "pad": 0, "residual": True},
        # decoding a batch: norm, and the projection of queries, keys and values
        {"name": "norm_linear_64x6144x4096", "kind": "norm_linear", "dtype": "bf16", "M": 64, "N": 6144, "K": 4096, "residual": True},
        # decoding one token: the feed-forward block's way back to the residual stream
        {"name": "add_1x4096x12288", "kind": "add", "dtype": "bf16", "M": 1, "N": 4096, "K": 12288, "layout": "nk", "bias": False, "act": "none"},
        # a short prompt's output projection
        {"name": "add_256x4096x4096", "kind": "add", "dtype": "f16", "M": 256, "N": 4096, "K": 4096, "layout": "nk", "bias": True, "act": "none"},
        # sizes that fill no tile and no 16-byte chunk, weights kept row-major (in x out)
        {"name": "add_333x1000x2047_kn", "kind": "add", "dtype": "f16", "M": 333, "N": 1000, "K": 2047, "layout": "kn", "bias": True, "act": "gelu"},
        # prompts: compute bound
        {"name": "add_4096x4096x12288", "kind": "add", "dtype": "bf16", "M": 4096, "N": 4096, "K": 12288, "layout": "nk", "bias": False, "act": "none"},
        # decoding one token: the block's largest weights, read once
        {"name": "gated_1x12288x4096", "kind": "gated", "dtype": "bf16", "M": 1, "N": 12288, "K": 4096, "layout": "nk", "bias": False, "act": "silu", "input": "x"},
        # decoding a batch, behind the norm's int8 output
        {"name": "gated_64x8192x8192_i8", "kind": "gated", "dtype": "f16", "M": 64, "N": 8192, "K": 8192, "layout": "nk", "bias": False, "act": "silu", "input": "i8"},
        # odd sizes, biases, the other activation, row-major weights
        {"name": "gated_511x1000x2047_kn", "kind": "gated", "dtype": "f16", "M": 511, "N": 1000, "K": 2047, "layout": "kn", "bias": True, "act": "gelu_tanh", "input": "x"},
        # prompts: compute bound, the largest product of the benchmark
        {"name": "gated_8192x8192x4096", "kind": "gated", "dtype": "bf16", "M": 8192, "N": 8192, "K": 4096, "layout": "nk", "bias": False, "act": "silu", "input": "x"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_linear", "add", "add", "gated", "gated"])
    dtype = rng.choice(["f16", "bf16"])
    odd = rng.random() < 0.3
    if kind == "norm":
        M, K = _log_int(rng, 1, 8192), _log_int(rng, 64, 16384)
        if not odd:
            K = -(-K // 64) * 64
        return {"kind": kind, "dtype": dtype, "M": min(M, 2 ** 26 // K), "K": K, "pad": rng.choice([0, 0, 8, rng.randint(1, 300)]),
                "residual": rng.random() < 0.8}
    if kind == "norm_linear":
        K = _log_int(rng, 64, 8192)
        return {"kind": kind, "dtype": dtype, "M": _log_int(rng, 1, 8192), "N": -(-_log_int(rng, 64, 8192) // 64) * 64, "K": K if odd else -(-K // 128) * 128,
                "residual": rng.random() < 0.8}
    layout = rng.choice(["nk", "nk", "nk", "nk", "kn"])
    small = odd or layout == "kn"
    top = 4096 if small else 16384
    M, N, K = _log_int(rng, 1, 2048 if small else 8192), _log_int(rng, 64, top), _log_int(rng, 64, top)
    if not odd:   # most layers have widths of whole tiles; the rows are whatever the batch is
        N, K = -(-N // 64) * 64, -(-K // 128) * 128
    pair = 2 if kind == "gated" else 1
    case = {"kind": kind, "dtype": dtype, "M": max(1, min(M, 2 ** 39 // (pair * N * K))), "N": N, "K": K, "layout": layout, "bias": rng.random() < 0.4}
    if kind == "add":
        return case | {"act": rng.choice(["none", "none", "none", "relu", "silu", "gelu", "gelu_tanh"])}
    return case | {"act": rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu", "none"]), "input": rng.choice(["x", "i8"])}


# ------------------------------------------------------------------------------------------------------------------ #
# inputs, and what a program keeps
# ------------------------------------------------------------------------------------------------------------------ #
class State:
    pass


def _quantised(x):
    """(integers as floats, scales) of the groups along the last axis."""
    amax = x.abs().amax(-1, keepdim=True)
    y = torch.where(amax > 0, x * 127 / amax, torch.zeros_like(x))
    return torch.sign(y) * torch.floor(y.abs() + 0.5), (amax / 127).squeeze(-1)


def _activations(M, K, gen, spread=1.0):
    x = spread * torch.randn(M, K, device=DEV, generator=gen)
    x[:, ::61] *= 8.0          # some channels of a model's activations are much larger than the others
    return x


def _layer(s, case, gen):
    """int8 weights with a scale per output channel; of a gated block, each gate channel's before its up channel's."""
    N, K = case["N"] * (2 if case["kind"] == "gated" else 1), case["K"]
    layout = case.get("layout", "nk")
    w, s.w_scale = _quantised(torch.randn(N, K, device=DEV, generator=gen) / math.sqrt(K))
    w = w.to(torch.int8)
    s.w = w.t().contiguous() if layout == "kn" else w
    s.bias = 0.1 * torch.randn(N, device=DEV, generator=gen) if case.get("bias") else None
    s.flag = torch.zeros(1, device=DEV, dtype=torch.int32)
    if own:
        from paper_2104_09455_amd import binding as B
        M = case["M"]
        s.layout = B.B_KN if layout == "kn" else B.B_NK
        s.act = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU, "gelu_tanh": B.ACT_GELU_TANH}[case.get("act", "none")]
        s.out = torch.empty(M, case["N"], device=DEV, dtype=TORCH[case["dtype"]])
        # offline weight checksums, for where the scheme is the global one
        rn = B.abft_region_shape(M, N, K, B.I8, layout == "nk" and K % 16 == 0)[1]
        s.beta = torch.empty(B.abft_beta_bytes(K, N, rn), device=DEV, dtype=torch.uint8)
        B.abft_weight_checksum(K, N, s.w, s.w.stride(0), s.layout, B.I8, s.beta, rn)
        s.ws_bytes = B.abft_linear_scaled_workspace_bytes(M, N, K, B.AUTO)
        s.ws = torch.empty(s.ws_bytes, device=DEV, dtype=torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s, M, K, dtype = State(), case["M"], case["K"], TORCH[case["dtype"]]
    s.case = case
    pad = case.get("pad", 0)
    s.x = _activations(M, K + pad, gen).to(dtype)[:, :K]
    if own:
        from paper_2104_09455_amd import binding as B
        s.dt = {"f16": B.F16, "bf16": B.BF16}[case["dtype"]]
    if case["kind"] in ("norm", "norm_linear"):
        s.r = _activations(M, K + pad, gen, 4.0).to(dtype)[:, :K] if case["residual"] else None
        s.weight = 1.0 + 0.2 * torch.randn(K, device=DEV, generator=gen)
        if own:
            s.sum = torch.empty(M, K, device=DEV, dtype=dtype) if case["residual"] else None
            if case["kind"] == "norm":
                s.y = torch.empty(M, K, device=DEV, dtype=dtype)
            else:
                s.q = torch.empty(M, -(-K // 16) * 16, device=DEV, dtype=torch.int8)   # (rows of whole chunks)
                s.scale = torch.empty(M, device=DEV)
    if case["kind"] == "add":
        s.r = _activations(M, case["N"], gen, 4.0).to(dtype)
    if case.get("input") == "i8":
        q, s.x_scale = _quantised(s.x.float())
        s.x = q.to(torch.int8)
    if case["kind"] != "norm":
        _layer(s, case, gen)
    return s


# ------------------------------------------------------------------------------------------------------------------ #
# one pass
# ------------------------------------------------------------------------------------------------------------------ #
def _activated(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))   # (1 + tanh a) / 2 = 1 / (1 + exp(-2 a))
    return z


def _product(s, q, x_scale):
    w = s.w.float() if s.case.get("layout") == "kn" else s.w.float().t()
    y = torch.matmul(q, w) * x_scale[:, None] * s.w_scale
    return y if s.bias is None else y + s.bias


def _norm(s):
    """(the sum with the residual, the normed rows), both in the type of the activations."""
    total = s.x if s.r is None else (s.x.float() + s.r.float()).to(s.x.dtype)
    z = total.float()
    return total, (z * torch.rsqrt((z * z).mean(-1, keepdim=True) + EPS) * s.weight).to(s.x.dtype)


def _plain(s):
    case = s.case
    kind, dtype = case["kind"], TORCH[case["dtype"]]
    if kind in ("norm", "norm_linear"):
        total, y = _norm(s)
        out = {} if s.r is None else {"sum": total}
        if kind == "norm":
            return out | {"y": y}
        return out | {"out": _product(s, *_quantised(y.float())).to(dtype), "flag": s.flag}
    q, x_scale = (s.x.float(), s.x_scale) if case.get("input") == "i8" else _quantised(s.x.float())
    z = _product(s, q, x_scale)
    if kind == "add":
        y = s.r.float() + _activated(z, case["act"])
    else:
        y = _activated(z[:, 0::2], case["act"]) * z[:, 1::2]
    return {"out": y.to(dtype), "flag": s.flag}


def run(state):
    s, case = state, state.case
    if not own:
        return _plain(s)
    from paper_2104_09455_amd import binding as B
    kind, M, K = case["kind"], case["M"], case["K"]
    if kind == "norm":
        B.abft_rms_norm(M, K, s.x, s.x.stride(0), s.dt, s.weight, EPS, residual=s.r, ldr=s.r.stride(0) if s.r is not None else 0,
                        total=s.sum, ldt=K, Y=s.y, ldy=K)
        return {"y": s.y} if s.r is None else {"sum": s.sum, "y": s.y}
    N = case["N"]
    checks = dict(beta=s.beta, workspace=s.ws, workspace_bytes=s.ws_bytes, fault_flag=s.flag)
    if kind == "norm_linear":
        B.abft_rms_norm(M, K, s.x, s.x.stride(0), s.dt, s.weight, EPS, residual=s.r, ldr=s.r.stride(0) if s.r is not None else 0,
                        total=s.sum, ldt=K, Q=s.q, ldq=s.q.stride(0), scale=s.scale)
        B.abft_gemm_scaled(M, N, K, s.q, s.q.stride(0), s.scale, s.w, s.w.stride(0), s.layout, s.w_scale, s.bias, s.act, s.out, N, s.dt, B.AUTO, **checks)
        out = {"out": s.out, "flag": s.flag}
        return out if s.r is None else out | {"sum": s.sum}
    if kind == "add":
        B.abft_linear_scaled_add(M, N, K, s.x, s.x.stride(0), s.dt, s.w, s.w.stride(0), s.layout, s.w_scale, s.bias, s.act, s.r, s.r.stride(0),
                                 s.out, N, B.AUTO, **checks)
    elif case["input"] == "i8":
        B.abft_gemm_gated(M, N, K, s.x, s.x.stride(0), s.x_scale, s.w, s.w.stride(0), s.layout, s.w_scale, s.bias, s.act, s.out, N, s.dt, B.AUTO, **checks)
    else:
        B.abft_linear_gated(M, N, K, s.x, s.x.stride(0), s.dt, s.w, s.w.stride(0), s.layout, s.w_scale, s.bias, s.act, s.out, N, B.AUTO, **checks)
    return {"out": s.out, "flag": s.flag}


# ------------------------------------------------------------------------------------------------------------------ #
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------ #
def work(case):
    M, K, kind = case["M"], case["K"], case["kind"]
    if kind == "norm":
        return {"bytes": 2 * M * K * (4 if case["residual"] else 2) + 4 * K, "flops": 6 * M * K}
    N = case["N"]
    if kind == "norm_linear":
        return {"bytes": 2 * M * K * (3 if case["residual"] else 1) + 4 * K + N * K + 2 * M * N + 4 * N, "flops": 2 * M * N * K}
    cols = 2 * N if kind == "gated" else N
    moved = (M * K + 4 * M if case.get("input") == "i8" else 2 * M * K) + cols * K + 4 * cols * (2 if case["bias"] else 1) + 2 * M * N
    return {"bytes": moved + (2 * M * N if kind == "add" else 0), "flops": 2 * M * cols * K}


# ------------------------------------------------------------------------------------------------------------------ #
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------ #
def _exact_integers(x):
    """The quantisation rule: rows of integers and their scales."""
    top = x.abs().max(dim=1).values
    ratio = x * 127 / torch.where(top == 0, torch.ones_like(top), top)[:, None]
    return torch.where(ratio < 0, torch.ceil(ratio - 0.5), torch.floor(ratio + 0.5)), top / 127


def _exact_act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "silu":
        return z * torch.special.expit(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))) / 2
    return z


def exact(case, seed):
    s = prepare(case, seed)
    kind, dtype, out = case["kind"], TORCH[case["dtype"]], {}
    x = s.x.double()
    if kind in ("norm", "norm_linear"):
        if case["residual"]:
            x = x + s.r.double()
            out["sum"] = x
            x = x.to(dtype).double()      # the norm is that of the sum as it is stored
        length = torch.sqrt(x.pow(2).sum(dim=1) / case["K"] + EPS)
        x = x / length[:, None] * s.weight.double()[None, :]
        if kind == "norm":
            return out | {"y": x}
        x = x.to(dtype).double()          # the rule quantises values of 16 bits
    ints, scale = (x, s.x_scale.double()) if case.get("input") == "i8" else _exact_integers(x)
    w = s.w.double().t() if case.get("layout") == "kn" else s.w.double()         # channels x K
    z = (ints @ w.t()) * scale[:, None] * s.w_scale.double()[None, :]
    if s.bias is not None:
        z += s.bias.double()
    if kind == "gated":
        z = z.reshape(case["M"], case["N"], 2)
        z = _exact_act(z[:, :, 0], case["act"]) * z[:, :, 1]
    elif kind == "add":
        z = _exact_act(z, case["act"]) + s.r.double()
    return out | {"out": z, "flag": torch.zeros(1, device=DEV, dtype=torch.int32)}
