"""Operators of quantised language-model inference, as cases that can be prepared, run and checked one by one.

What an inference program does around an 8-bit model, in its plain form (``own`` false: elementary torch operations in 32
bits) or through this library's entry points (``own`` true):

* ``linear``     a linear layer of 16-bit activations and int8 weights: the activations are quantised per token, the
                 int8 product is scaled per token and channel, a bias is added, ReLU may follow; M 1 .. 8192, N and K 64 ..
                 8192 (odd widths and row-major weights: M up to 2048, N and K up to 4096).  The protection scheme is the
                 library's own choice; the sticky fault flag comes back with the result.
* ``cache``      keys and values of new tokens written to a paged cache and read back: int8 with a scale for each
                 token and head, or in the type of the activations; 1 .. 16384 tokens of 1 .. 64 sequences, 1 .. 16 heads of 16
                 .. 128, pages of 16 .. 256 tokens.
* ``attention``  a chunk of new tokens of every sequence over that cache: one token (decoding), whole prompts, and
                 batches of both; 1 .. 64 sequences, 1 .. 8192 new tokens, up to 32768 in the cache, 1 .. 16 query heads for
                 each of 1 .. 8 heads of the cache, causal, with a window or without.

The quantisation rule of all of them: for a group of values (a token's activations, a token's key of one head) with the
largest magnitude a, the scale is a / 127 and the integers are 127 x / a, rounded to nearest, halves away from zero; a
group of zeros has the scale zero.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------------ #
# the cases
# ------------------------------------------------------------------------------------------------------------------ #
def _text(lengths):
    """New tokens (q) and tokens in the cache with them (kv) of every sequence are one text of numbers."""
    return " ".join(str(n) for n in lengths)


def _lengths(case):
    return [int(n) for n in case["q"].split()], [int(n) for n in case["kv"].split()]


def listed():
    return [
        # decoding one token: a 4096-wide layer's weights are all there is to read
        {"name": "linear_1x4096x4096", "kind": "linear", "dtype": "bf16", "M": 1, "N": 4096, "K": 4096, "layout": "nk", "bias": False, "relu": False},
        # a batch of tokens in decoding, or a short prompt, through the same layer
        {"name": "linear_256x4096x4096", "kind": "linear", "dtype": "f16", "M": 256, "N": 4096, "K": 4096, "layout": "nk", "bias": True, "relu": True},
        # sizes that fill no tile and no 16-byte chunk, weights kept row-major (in x out)
        {"name": "linear_511x1000x2047_kn", "kind": "linear", "dtype": "f16", "M": 511, "N": 1000, "K": 2047, "layout": "kn", "bias": True, "relu": False},
        # prompts, compute bound: the largest product of the benchmark
        {"name": "linear_8192x8192x8192", "kind": "linear", "dtype": "bf16", "M": 8192, "N": 8192, "K": 8192, "layout": "nk", "bias": True, "relu": False},
        # a decoding step's keys and values: one token of each of 64 sequences
        {"name": "cache_64_tokens", "kind": "cache", "dtype": "bf16", "cache": "i8", "seqs": 64, "tokens": 64, "heads": 8, "dim": 128, "page": 16},
        # a prompt's: bytes
        {"name": "cache_8192_tokens", "kind": "cache", "dtype": "f16", "cache": "i8", "seqs": 2, "tokens": 8192, "heads": 8, "dim": 128, "page": 64},
        # decoding a single sequence: few rows, a long axis
        {"name": "attention_decode_1x16384", "kind": "attention", "dtype": "bf16", "cache": "i8", "q": "1", "kv": "16384", "heads": 8, "group": 4,
         "dim": 128, "page": 16, "causal": True, "window": 0},
        # decoding a batch of ragged lengths from the quantised cache: its bytes
        {"name": "attention_decode_64", "kind": "attention", "dtype": "bf16", "cache": "i8", "q": _text([1] * 64), "kv": _text(129 * i + 17 for i in range(64)),
         "heads": 8, "group": 4, "dim": 128, "page": 16, "causal": True, "window": 0},
        # the same from a 16-bit cache, as many query heads as heads of the cache
        {"name": "attention_decode_16_heads", "kind": "attention", "dtype": "f16", "cache": "f16", "q": _text([1] * 16), "kv": _text(251 * i + 33 for i in range(16)),
         "heads": 16, "group": 1, "dim": 64, "page": 64, "causal": True, "window": 0},
        # chunks of long prompts beside single tokens, as a server batches them
        {"name": "attention_mixed", "kind": "attention", "dtype": "f16", "cache": "i8", "q": "1 509 1 1 1024 1 37 1", "kv": "3001 4605 17 8000 1024 900 37 1",
         "heads": 4, "group": 7, "dim": 128, "page": 32, "causal": True, "window": 0},
        # a chunk over a long context with a window, heads that are no power of two wide
        {"name": "attention_window", "kind": "attention", "dtype": "bf16", "cache": "bf16", "q": "2048", "kv": "12000", "heads": 8, "group": 4,
         "dim": 80, "page": 48, "causal": True, "window": 1000},
        # a whole prompt: compute bound
        {"name": "attention_prompt_8192", "kind": "attention", "dtype": "bf16", "cache": "bf16", "q": "8192", "kv": "8192", "heads": 8, "group": 4,
         "dim": 128, "page": 64, "causal": True, "window": 0},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "cache", "attention", "attention", "attention"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "linear":
        layout = rng.choice(["nk", "nk", "nk", "nk", "kn"])
        odd = rng.random() < 0.3
        top = 8192 if layout == "nk" and not odd else 4096
        M, N, K = _log_int(rng, 1, top if top == 8192 else 2048), _log_int(rng, 64, top), _log_int(rng, 64, top)
        if not odd:  # most layers have widths of whole tiles; the rows are whatever the batch is
            N, K = -(-N // 64) * 64, -(-K // 128) * 128
        return {"kind": kind, "dtype": dtype, "M": M, "N": N, "K": K, "layout": layout, "bias": rng.random() < 0.5, "relu": rng.random() < 0.3}
    dim = rng.choice([64, 128, 128, 16 * rng.randint(1, 8)])
    page = rng.choice([16, 32, 64, 16 * rng.randint(1, 16)])
    cache = rng.choice(["i8", "i8", dtype])
    if kind == "cache":
        seqs = _log_int(rng, 1, 64)
        heads = rng.choice([1, 2, 4, 8, rng.randint(1, 16)])
        return {"kind": kind, "dtype": dtype, "cache": cache, "seqs": seqs, "tokens": _log_int(rng, seqs, 16384), "heads": heads, "dim": dim, "page": page}
    heads, group = rng.choice([1, 2, 4, 8, rng.randint(1, 8)]), rng.choice([1, 4, 8, rng.randint(1, 16)])
    what = rng.choice(["decode", "decode", "chunk", "mixed"])
    if what == "decode":
        seqs, top = _log_int(rng, 1, 64), 32768
        top = min(top, max(64, 400000 // seqs))
        q, kv = [1] * seqs, [_log_int(rng, 1, top) for _ in range(seqs)]
    else:
        seqs = _log_int(rng, 1, 8)
        # (as many products of a query and a key, over all heads, as the whole prompt has at most)
        left = 2 ** 30 // (heads * group * seqs)
        q, kv = [], []
        for _ in range(seqs):
            n = 1 if what == "mixed" and rng.random() < 0.5 else _log_int(rng, 1, 8192)
            n = max(1, min(n, int(math.sqrt(left))))
            q.append(n)
            kv.append(n + min(_log_int(rng, 1, 32768) - 1, max(0, left // n - n)))
    return {"kind": kind, "dtype": dtype, "cache": cache, "q": _text(q), "kv": _text(kv), "heads": heads, "group": group, "dim": dim, "page": page,
            "causal": rng.random() < 0.8, "window": _log_int(rng, 1, 8192) if rng.random() < 0.2 else 0}


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


def _prepare_linear(case, gen):
    s, M, N, K = State(), case["M"], case["N"], case["K"]
    s.x = torch.randn(M, K, device=DEV, generator=gen)
    s.x[:, ::61] *= 8.0          # some channels of a model's activations are much larger than the others
    s.x = s.x.to(TORCH[case["dtype"]])
    w, s.w_scale = _quantised(0.02 * torch.randn(N, K, device=DEV, generator=gen))
    w = w.to(torch.int8)
    s.w = w.t().contiguous() if case["layout"] == "kn" else w
    s.bias = 0.1 * torch.randn(N, device=DEV, generator=gen) if case["bias"] else None
    if own:
        from paper_2104_09455_amd import binding as B
        s.dt = {"f16": B.F16, "bf16": B.BF16}[case["dtype"]]
        s.layout = B.B_KN if case["layout"] == "kn" else B.B_NK
        s.act = B.ACT_RELU if case["relu"] else B.ACT_NONE
        s.out = torch.empty(M, N, device=DEV, dtype=s.x.dtype)
        s.flag = torch.zeros(1, device=DEV, dtype=torch.int32)
        # offline weight checksums, for where the scheme is the global one
        rn = B.abft_region_shape(M, N, K, B.I8, case["layout"] == "nk" and K % 16 == 0)[1]
        s.beta = torch.empty(B.abft_beta_bytes(K, N, rn), device=DEV, dtype=torch.uint8)
        B.abft_weight_checksum(K, N, s.w, s.w.stride(0), s.layout, B.I8, s.beta, rn)
        s.ws_bytes = B.abft_linear_scaled_workspace_bytes(M, N, K, B.AUTO)
        s.ws = torch.empty(s.ws_bytes, device=DEV, dtype=torch.uint8)
    else:
        s.flag = torch.zeros(1, device=DEV, dtype=torch.int32)
    return s


def _paged(kv, page, rng):
    """(pages, block table as rows of page numbers): the pages of every sequence lie anywhere."""
    need = [-(-n // page) for n in kv]
    pages = sum(need) + 3
    order, at, table = rng.permutation(pages), 0, np.zeros((len(kv), max(max(need), 1)), np.int32)
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return pages, table


def _handle(B, s, case):
    kinds = {"f16": B.F16, "bf16": B.BF16, "i8": B.I8}
    s.dt = kinds[case["dtype"]]
    s.cache = B.kv_cache(s.k, s.v, s.k_scale, s.v_scale, kinds[case["cache"]], s.pages, case["page"], case["heads"], case["dim"])


def _prepare_cache(case, gen, rng):
    s, heads, dim, page = State(), case["heads"], case["dim"], case["page"]
    cuts = np.sort(rng.choice(np.arange(1, case["tokens"]), case["seqs"] - 1, replace=False)) if case["seqs"] > 1 else np.zeros(0, int)
    lens = np.diff(np.concatenate([[0], cuts, [case["tokens"]]])).astype(int)
    before = rng.integers(0, 1000, case["seqs"])       # tokens that the sequences already have
    s.pages, table = _paged([int(b + n) for b, n in zip(before, lens)], page, rng)
    slots = []
    for i in range(case["seqs"]):
        t = np.arange(before[i], before[i] + lens[i])
        slots.append(table[i, t // page].astype(np.int64) * page + t % page)
    s.slots = torch.from_numpy(np.concatenate(slots)).to(DEV)
    T, n = case["tokens"], heads * dim
    s.qkv = torch.randn(T, 6 * n, device=DEV, generator=gen).to(TORCH[case["dtype"]])   # the product that makes them
    s.new_k, s.new_v = s.qkv[:, 4 * n:5 * n], s.qkv[:, 5 * n:]
    kind = torch.int8 if case["cache"] == "i8" else TORCH[case["cache"]]
    s.k = torch.zeros(s.pages, heads, page, dim, device=DEV, dtype=kind)
    s.v = torch.zeros_like(s.k)
    s.k_scale = s.v_scale = None
    if case["cache"] == "i8":
        s.k_scale = torch.zeros(s.pages, heads, page, device=DEV)
        s.v_scale = torch.zeros(s.pages, heads, page, device=DEV)
    if own:
        from paper_2104_09455_amd import binding as B
        _handle(B, s, case)
        s.back_k = torch.empty(T, heads, dim, device=DEV, dtype=s.qkv.dtype)
        s.back_v = torch.empty_like(s.back_k)
    return s


def _prepare_attention(case, gen, rng):
    s, heads, dim, page = State(), case["heads"], case["dim"], case["page"]
    s.nq, s.nk = _lengths(case)
    s.pages, table = _paged(s.nk, page, rng)
    s.table = torch.from_numpy(table).to(DEV)
    n = len(s.nq)
    s.q_start = torch.from_numpy(np.concatenate([[0], np.cumsum(s.nq)]).astype(np.int32)).to(DEV)
    s.kv_len = torch.tensor(s.nk, dtype=torch.int32, device=DEV)
    T, hq = sum(s.nq), heads * case["group"]
    s.qkv = torch.randn(T, (hq + 2 * heads) * dim, device=DEV, generator=gen).to(TORCH[case["dtype"]])
    s.q = s.qkv[:, :hq * dim]
    s.k_scale = s.v_scale = None
    if case["cache"] == "i8":
        s.k, s.k_scale = _quantised(torch.randn(s.pages, heads, page, dim, device=DEV, generator=gen))
        s.v, s.v_scale = _quantised(torch.randn(s.pages, heads, page, dim, device=DEV, generator=gen))
        s.k, s.v = s.k.to(torch.int8), s.v.to(torch.int8)
    else:
        s.k = torch.randn(s.pages, heads, page, dim, device=DEV, generator=gen).to(TORCH[case["cache"]])
        s.v = torch.randn(s.pages, heads, page, dim, device=DEV, generator=gen).to(TORCH[case["cache"]])
    s.scale = 1.0 / math.sqrt(dim)
    if own:
        from paper_2104_09455_amd import binding as B
        _handle(B, s, case)
        s.out = torch.empty(T, hq, dim, device=DEV, dtype=s.qkv.dtype)
        s.n, s.total, s.max_q, s.max_kv, s.hq = n, T, max(s.nq), max(s.nk), hq
        s.ws_bytes = B.abft_attention_workspace_bytes(s.cache, s.n, s.total, s.max_q, s.max_kv, hq, s.dt)
        s.ws = torch.zeros(s.ws_bytes, device=DEV, dtype=torch.uint8)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = np.random.Generator(np.random.PCG64(seed))
    if case["kind"] == "linear":
        s = _prepare_linear(case, gen)
    elif case["kind"] == "cache":
        s = _prepare_cache(case, gen, rng)
    else:
        s = _prepare_attention(case, gen, rng)
    s.case = case
    return s


# ------------------------------------------------------------------------------------------------------------------ #
# one pass
# ------------------------------------------------------------------------------------------------------------------ #
def _linear(s):
    case = s.case
    q, x_scale = _quantised(s.x.float())
    w = s.w.float() if case["layout"] == "kn" else s.w.float().t()
    y = torch.matmul(q, w) * x_scale[:, None] * s.w_scale
    if s.bias is not None:
        y = y + s.bias
    if case["relu"]:
        y = torch.clamp(y, min=0)
    return {"out": y.to(s.x.dtype), "flag": s.flag}


def _cache(s):
    case = s.case
    page, off = s.slots // case["page"], s.slots % case["page"]
    back = {}
    for name, new, values, scales in (("k", s.new_k, s.k, s.k_scale), ("v", s.new_v, s.v, s.v_scale)):
        new = new.reshape(-1, case["heads"], case["dim"])
        if scales is None:
            values[page, :, off] = new
            back[name] = values[page, :, off]
        else:
            q, scale = _quantised(new.float())
            values[page, :, off] = q.to(torch.int8)
            scales[page, :, off] = scale
            back[name] = (values[page, :, off].float() * scales[page, :, off][..., None]).to(new.dtype)
    return back


def _attention(s, wide=torch.float32):
    """The softmax of each head's products over what the row may see, times the values; rows that see nothing are zero."""
    case = s.case
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    out = torch.zeros(sum(s.nq), heads * group, dim, device=DEV, dtype=wide)
    at = 0
    for i, (nq, nk) in enumerate(zip(s.nq, s.nk)):
        t = torch.arange(nk, device=DEV)
        rows, off = s.table[i][t // page].long(), t % page
        k, v = s.k[rows, :, off].to(wide), s.v[rows, :, off].to(wide)               # tokens x heads x dim
        if s.k_scale is not None:
            k, v = k * s.k_scale[rows, :, off][..., None], v * s.v_scale[rows, :, off][..., None]
        q = s.q[at:at + nq].reshape(nq, heads, group, dim).to(wide)
        mask = None
        if case["causal"] or case["window"]:
            pos = (nk - nq) + torch.arange(nq, device=DEV)[:, None]
            mask = (t[None] <= pos) if case["causal"] else torch.ones(nq, nk, dtype=torch.bool, device=DEV)
            if case["window"]:
                mask = mask & (t[None] > pos - case["window"])
            mask = mask[:, None]
        for h in range(heads):
            logits = torch.matmul(q[:, h].reshape(nq * group, dim), k[:, h].t().contiguous()).reshape(nq, group, nk) * s.scale
            if mask is not None:
                logits = logits.masked_fill(~mask, -math.inf)
            top = logits.amax(-1, keepdim=True)
            p = torch.exp(logits - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            total = p.sum(-1, keepdim=True)
            p = p / torch.where(total > 0, total, torch.ones_like(total))
            o = torch.matmul(p.reshape(nq * group, nk), v[:, h].contiguous())
            out[at:at + nq, h * group:(h + 1) * group] = o.reshape(nq, group, dim)
        at += nq
    return out


def run(state):
    s, case = state, state.case
    kind = case["kind"]
    if not own:
        if kind == "linear":
            return _linear(s)
        if kind == "cache":
            return _cache(s)
        return {"out": _attention(s).to(s.qkv.dtype)}
    from paper_2104_09455_amd import binding as B
    if kind == "linear":
        B.abft_linear_scaled(case["M"], case["N"], case["K"], s.x, s.x.stride(0), s.dt, s.w, s.w.stride(0), s.layout, s.w_scale, s.bias, s.act,
                             s.out, s.out.stride(0), B.AUTO, beta=s.beta, workspace=s.ws, workspace_bytes=s.ws_bytes, fault_flag=s.flag)
        return {"out": s.out, "flag": s.flag}
    if kind == "cache":
        stride = s.qkv.stride(0)
        B.abft_kv_write(s.cache, case["tokens"], s.slots, s.new_k, stride, s.new_v, stride, s.dt)
        B.abft_kv_read(s.cache, case["tokens"], s.slots, s.back_k, s.back_k.stride(0), s.back_v, s.back_v.stride(0), s.dt)
        return {"k": s.back_k, "v": s.back_v}
    B.abft_attention(s.cache, s.n, s.q_start, s.kv_len, s.table, s.table.stride(0), s.total, s.max_q, s.max_kv, s.q, s.q.stride(0), s.hq, s.dt,
                     s.scale, case["causal"], case["window"], s.out, s.out.stride(0), workspace=s.ws, workspace_bytes=s.ws_bytes)
    return {"out": s.out}


# ------------------------------------------------------------------------------------------------------------------ #
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------ #
def _pairs(nq, nk, causal, window):
    """Products of a query and a key that the masks leave."""
    pos = np.arange(nk - nq, nk, dtype=np.int64)
    hi = np.minimum(pos, nk - 1) if causal else np.full(nq, nk - 1, np.int64)
    lo = np.maximum(pos - window + 1, 0) if window else np.zeros(nq, np.int64)
    return int(np.maximum(hi - lo + 1, 0).sum()), int(lo.min()), int(hi.max())


def work(case):
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K + 2 * M * N + 4 * N * (2 if case["bias"] else 1), "flops": 2 * M * N * K}
    stored = case["dim"] + 4 if case["cache"] == "i8" else 2 * case["dim"]       # bytes of a token's key of one head
    if case["kind"] == "cache":
        n = 2 * case["tokens"] * case["heads"]
        return {"bytes": n * (2 * case["dim"] + 2 * stored + 2 * case["dim"]) + 8 * case["tokens"], "flops": 4 * n * case["dim"]}
    hq, flops, keys = case["heads"] * case["group"], 0, 0
    for nq, nk in zip(*_lengths(case)):
        pairs, lo, hi = _pairs(nq, nk, case["causal"], case["window"])
        flops += 4 * case["dim"] * hq * pairs
        keys += hi - lo + 1
    return {"bytes": 2 * keys * case["heads"] * stored + 4 * sum(_lengths(case)[0]) * hq * case["dim"], "flops": flops}


# ------------------------------------------------------------------------------------------------------------------ #
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------ #
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        top = s.x.double().abs().max(dim=1).values
        safe = torch.where(top == 0, torch.ones_like(top), top)[:, None]
        ratio = s.x.double() * 127 / safe
        ints = torch.where(ratio < 0, torch.ceil(ratio - 0.5), torch.floor(ratio + 0.5))
        w = s.w.double() * (s.w_scale.double()[None, :] if case["layout"] == "kn" else s.w_scale.double()[:, None])
        if case["layout"] == "nk":
            w = w.t()
        y = (ints * (top / 127)[:, None]) @ w
        if s.bias is not None:
            y += s.bias.double()
        if case["relu"]:
            y = torch.where(y < 0, torch.zeros_like(y), y)
        return {"out": y, "flag": torch.zeros(1, device=DEV, dtype=torch.int32)}
    if case["kind"] == "cache":
        back = {}
        for name, new in (("k", s.new_k), ("v", s.new_v)):
            x = new.double().reshape(case["tokens"], case["heads"], case["dim"])
            if case["cache"] == "i8":
                top = x.abs().max(dim=2, keepdim=True).values
                ratio = x * 127 / torch.where(top == 0, torch.ones_like(top), top)
                x = torch.where(ratio < 0, torch.ceil(ratio - 0.5), torch.floor(ratio + 0.5)) * (top / 127)
            back[name] = x
        return back
    # attention, key by page, all rows of a head at once in runs of rows
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    out, row0 = [], 0
    for i, (nq, nk) in enumerate(zip(s.nq, s.nk)):
        used = s.table[i, :-(-nk // page)].long()
        ks, vs = s.k[used].double(), s.v[used].double()                              # pages x heads x page x dim
        if s.k_scale is not None:
            ks, vs = ks * s.k_scale[used].double().unsqueeze(-1), vs * s.v_scale[used].double().unsqueeze(-1)
        ks, vs = (x.transpose(0, 1).reshape(heads, -1, dim)[:, :nk] for x in (ks, vs))
        rows = s.q[row0:row0 + nq].double().reshape(nq, heads * group, dim)
        got = torch.zeros(nq, heads * group, dim, device=DEV, dtype=torch.float64)
        key = torch.arange(nk, device=DEV)
        step = max(1, (1 << 26) // max(nk, 1))
        for h in range(heads * group):
            kh, vh = ks[h // group].contiguous(), vs[h // group].contiguous()
            for a in range(0, nq, step):
                b = min(nq, a + step)
                z = (rows[a:b, h].contiguous() @ kh.t().contiguous()) / math.sqrt(dim)
                place = torch.arange(nk - nq + a, nk - nq + b, device=DEV).unsqueeze(1)
                seen = torch.ones(b - a, nk, dtype=torch.bool, device=DEV)
                if case["causal"]:
                    seen &= key <= place
                if case["window"] > 0:
                    seen &= key > place - case["window"]
                any_seen = seen.any(dim=1, keepdim=True)
                z = torch.softmax(torch.where(seen, z, torch.full_like(z, -1e300)), dim=1) * any_seen
                got[a:b, h] = z @ vh
        out.append(got)
        row0 += nq
    return {"out": torch.cat(out)}
