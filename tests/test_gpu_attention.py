"""Attention over the paged cache against its definition in 64 bits.

Bound of an element.  Its weights are rounded to the type of the queries (u: 2^-11 or 2^-8 of a weight; below that type's
smallest normal, absolutely: 2^-25 of the largest weight in fp16), after an exponential whose argument carries the rounding
of dim fp32 additions, dim 2^-24 scale sum |q k|, and a few more of the argument itself; the sums over keys run in fp32 with
at most that many roundings again, and the result is rounded once.  With p_j the exact weights, A = sum p_j |v_j|:
    |error| <= (u + 2 e) A + u |o| + small,   e = 2^-24 (dim + keys / 16 + 64) (1 + max_j scale sum |q k_j|),
    small = 2^-25 sum_j |v_j| max_j p_j (t_j) for fp16 weights (t: an int8 value's scale), and the output's smallest step."""
import math

import numpy as np
import pytest
import torch

from paper_2104_09455_amd import binding as B
from test_gpu_linear_scaled import DEV, TYPES

pytestmark = pytest.mark.gpu


class Case:
    """A batch of sequences over a cache whose other places, and unused table entries, hold what must not matter."""

    def __init__(self, q, kv, heads, group, dim, page, dtype, cache, seed=0, causal=True, window=0, extra_pages=3, scale=None, poison=True):
        self.q, self.kv, self.heads, self.group, self.dim, self.page = q, kv, heads, group, dim, page
        self.dt, self.t, self.u, self.tiny = TYPES[dtype]
        self.i8, self.causal, self.window = cache == "i8", causal, window
        self.scale = scale or 1 / math.sqrt(dim)
        g = torch.Generator(device=DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in kv]
        self.pages = sum(need) + extra_pages
        order = rng.permutation(self.pages)
        self.width = max(max(need), 1) + 2
        table = rng.choice([-7, 1 << 30, 0, -(1 << 31)], (len(q), self.width)).astype(np.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        self.table_host = table
        self.table = torch.from_numpy(table).to(DEV)
        shape = (self.pages, heads, page, dim)
        ones = self.pages, heads, page
        bad = float("nan") if poison else 0.0
        if self.i8:
            self.k = torch.randint(-127, 128, shape, device=DEV, generator=g, dtype=torch.int8)
            self.v = torch.randint(-127, 128, shape, device=DEV, generator=g, dtype=torch.int8)
            self.ks = 0.02 * 2.0 ** (4 * torch.rand(ones, device=DEV, generator=g) - 3)
            self.vs = 0.02 * 2.0 ** (4 * torch.rand(ones, device=DEV, generator=g) - 2)
        else:
            self.k = torch.randn(shape, device=DEV, generator=g).to(self.t)
            self.v = torch.randn(shape, device=DEV, generator=g).to(self.t)
            self.ks = self.vs = None
        used = torch.zeros(ones, dtype=torch.bool, device=DEV)
        for i, n in enumerate(kv):
            t = torch.arange(n, device=DEV)
            used[self.table[i][t // page].long(), :, t % page] = True
        if poison:
            for x in ((self.ks, self.vs) if self.i8 else (self.k, self.v)):
                x[~used] = bad
        self.total, self.hq = sum(q), heads * group
        self.ldq = self.hq * dim + 24
        self.Q = torch.full((max(self.total, 1), self.ldq), float("nan"), dtype=self.t, device=DEV)
        self.Q[:self.total, :self.hq * dim] = torch.randn(self.total, self.hq * dim, device=DEV, generator=g).to(self.t)
        self.q_start = torch.from_numpy(np.concatenate([[0], np.cumsum(q)]).astype(np.int32)).to(DEV)
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device=DEV)
        self.handle = B.kv_cache(self.k, self.v, self.ks, self.vs, B.I8 if self.i8 else self.dt, self.pages, page, heads, dim)

    def run(self, max_q=None, max_kv=None, stream=None):
        max_q, max_kv = max(self.q) if max_q is None else max_q, max(self.kv) if max_kv is None else max_kv
        ldo = self.hq * self.dim + 4
        out = torch.full((self.total + 1, ldo), 7.0, dtype=self.t, device=DEV)
        n = B.abft_attention_workspace_bytes(self.handle, len(self.q), self.total, max_q, max_kv, self.hq, self.dt)
        ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)   # (NaN)
        ws[:4096] = 0
        torch.cuda.synchronize()
        B.abft_attention(self.handle, len(self.q), self.q_start, self.kv_len, self.table, self.width, self.total, max_q, max_kv, self.Q, self.ldq,
                         self.hq, self.dt, self.scale, self.causal, self.window, out, ldo, workspace=ws if n else None, workspace_bytes=n, stream=stream)
        torch.cuda.synchronize()
        assert not ws[:4096].any()
        assert (out[:, self.hq * self.dim:] == 7.0).all() and (out[self.total] == 7.0).all()
        return out[:self.total, :self.hq * self.dim].reshape(self.total, self.hq, self.dim)

    def want(self, i, h):
        """(rows, bounds) of sequence i and head h in 64 bits."""
        nq, nk, D = self.q[i], self.kv[i], self.dim
        t = torch.arange(nk, device=DEV)
        at, off = self.table[i][t // self.page].long(), t % self.page
        kh = h // self.group
        k, v = self.k[at, kh, off].double(), self.v[at, kh, off].double()
        step = torch.ones(nk, device=DEV, dtype=torch.float64)
        if self.i8:
            step = self.vs[at, kh, off].double()
            k = k * self.ks[at, kh, off].double()[:, None]
            v = v * step[:, None]
        r0 = int(sum(self.q[:i]))
        q = self.Q[r0:r0 + nq, h * D:(h + 1) * D].double()
        pos = nk - nq + torch.arange(nq, device=DEV)[:, None]
        seen = torch.ones(nq, nk, dtype=torch.bool, device=DEV)
        if self.causal:
            seen &= t[None] <= pos
        if self.window:
            seen &= t[None] > pos - self.window
        some = seen.any(1, keepdim=True)
        z = (q @ k.t().contiguous()) * self.scale
        z = torch.where(seen, z, torch.full_like(z, -math.inf))
        top = torch.where(some, z.amax(1, keepdim=True) if nk else torch.zeros(nq, 1, device=DEV, dtype=torch.float64), torch.zeros(1, device=DEV, dtype=torch.float64))
        w = torch.where(seen, torch.exp(z - top), torch.zeros_like(z))
        p = w / torch.where(some, w.sum(1, keepdim=True), torch.ones_like(top))
        # (what is not seen counts as nothing, whatever it holds)
        out = torch.zeros(nq, D, device=DEV, dtype=torch.float64)
        clean = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
        out = p @ clean
        for j in (~torch.isfinite(v)).any(1).nonzero().flatten().tolist():
            rows = seen[:, j]
            out[rows] += torch.where(torch.isfinite(v[j]), torch.zeros_like(v[j]), p[rows, j][:, None] * v[j])
        A = p @ clean.abs()
        mag = self.scale * (q.abs() @ k.abs().t().contiguous())
        mag = torch.where(seen, mag, torch.zeros_like(mag)).amax(1, keepdim=True) if nk else torch.zeros_like(top)
        e = 2.0 ** -24 * (D + nk / 16 + 64) * (1 + mag)
        small = torch.zeros(nq, 1, device=DEV, dtype=torch.float64)
        if self.t == torch.float16 and nk:
            # (the integers of int8 values, or the values)
            raw = self.v[at, kh, off].double() if self.i8 else clean
            small = 2.0 ** -25 * (seen.double() @ raw.abs()) * (p * step).amax(1, keepdim=True)
        return out, (self.u + 2 * e) * A + self.u * out.abs() + small + self.tiny

    def check(self, got):
        for i in range(len(self.q)):
            r0 = int(sum(self.q[:i]))
            for h in range(self.hq):
                out, bound = self.want(i, h)
                g = got[r0:r0 + self.q[i], h].double()
                nan = torch.isnan(out)
                assert torch.equal(torch.isnan(g), nan), (i, h)
                inf = torch.isinf(out)
                assert torch.equal(g[inf], out[inf]), (i, h)
                ok = ~(nan | inf)
                err = (g - out).abs()[ok]
                assert (err <= bound[ok]).all(), (i, h, float((err / bound[ok]).max()))


def both(dtype):
    return [(dtype, "i8"), (dtype, "same")]


TYPES_AND_CACHES = both("f16") + both("bf16")


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
@pytest.mark.parametrize("kv,heads,group,dim,page", [
    ([1], 1, 1, 16, 16), ([2, 31, 32, 33], 2, 4, 64, 16), ([127, 128, 129, 0, 1], 3, 5, 48, 32), ([500, 17, 1000], 2, 16, 128, 48),
    ([5000], 1, 8, 128, 16), ([3, 9000, 0, 256, 257, 511, 512, 513], 2, 4, 80, 64), ([70] * 100, 1, 1, 32, 256), ([700, 20], 2, 17, 64, 16)])
def test_single_tokens(kv, heads, group, dim, page, dtype, cache):
    print(f"case single kv={kv[:8]} heads={heads}x{group} dim={dim} page={page} {dtype} {cache}", flush=True)
    for window in (0, 1, 100):
        c = Case([1] * len(kv), kv, heads, group, dim, page, dtype, cache, seed=sum(kv), window=window)
        c.check(c.run())


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
@pytest.mark.parametrize("q,kv,heads,group,dim,page", [
    ([2], [2], 1, 1, 16, 16), ([5, 64], [5, 64], 2, 3, 64, 16), ([33, 1, 7], [33, 90, 200], 1, 4, 128, 32), ([128], [700], 2, 1, 112, 48),
    ([3, 0, 1, 0, 40], [9, 5, 6, 0, 41], 2, 8, 96, 64), ([10, 1, 6], [4, 0, 1], 1, 2, 32, 16), ([300], [300], 1, 7, 80, 256), ([2, 2, 2], [4000, 1, 65], 1, 4, 128, 16),
    ([9, 1], [6000, 6100], 2, 2, 64, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 37), (False, 64)])
def test_chunks(q, kv, heads, group, dim, page, causal, window, dtype, cache):
    print(f"case chunk q={q} kv={kv} heads={heads}x{group} dim={dim} page={page} causal={causal} window={window} {dtype} {cache}", flush=True)
    c = Case(q, kv, heads, group, dim, page, dtype, cache, seed=sum(kv) + 1, causal=causal, window=window)
    c.check(c.run())


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q,kv", [([10, 1, 6], [4, 0, 1]), ([300], [170]), ([1, 200, 1], [90, 900, 2])])
def test_windows_as_large_as_they_can_be(q, kv, causal, window, dtype, cache):
    """They hide nothing, also where a sequence has more new tokens than the cache holds."""
    print(f"case window={window} q={q} kv={kv} causal={causal} {dtype} {cache}", flush=True)
    c = Case(q, kv, 2, 2, 64, 16, dtype, cache, seed=sum(kv), causal=causal, window=window)
    c.check(c.run())


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
def test_many_sequences(dtype, cache):
    """More sequences than a wavefront has lanes, single tokens and chunks among them, and bounds that are larger than needed."""
    rng = np.random.default_rng(7)
    q = [int(n) for n in rng.choice([0, 1, 1, 1, 2, 9, 40], 150)]
    kv = [int(n + rng.integers(0, 90)) if n else 0 for n in q]
    c = Case(q, kv, 2, 2, 64, 16, dtype, cache, seed=5)
    got = c.run()
    c.check(got)
    c.check(c.run(max_q=min(sum(q), 100), max_kv=(c.width * 16)))


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
@pytest.mark.parametrize("what", ["v", "k", "both"])
def test_values_that_are_not_finite_where_they_are_not_seen(what, dtype, cache):
    """Infinities and NaN in keys and values that some rows of a tile see and others do not: only those rows show them."""
    for causal, window in ((True, 0), (True, 20), (False, 50)):
        c = Case([70, 1, 5], [150, 40, 66], 2, 2, 64, 16, dtype, cache, seed=11, causal=causal, window=window)
        for i, places in enumerate(([0, 81, 100, 149], [3], [62, 65])):
            for n, j in enumerate(places):
                page, off = int(c.table_host[i, j // 16]), j % 16
                bad = [float("inf"), float("nan"), -float("inf")][n % 3]
                if c.i8:
                    if what != "k":
                        c.vs[page, 1, off] = float("nan")
                    if what != "v":
                        c.ks[page, 0, off] = float("nan")
                else:
                    if what != "k":
                        c.v[page, 1, off, 5 + n] = bad
                    if what != "v":
                        c.k[page, 0, off, 2 * n] = float("nan")
        if c.i8:
            # (a scale that is NaN makes all of the key's values NaN)
            got = c.run()
            for i in range(3):
                r0 = sum(c.q[:i])
                for h in range(c.hq):
                    out, _ = c.want(i, h)
                    assert torch.equal(torch.isnan(got[r0:r0 + c.q[i], h].double()).all(1), torch.isnan(out).all(1)), (i, h)
                    assert torch.equal(torch.isnan(got[r0:r0 + c.q[i], h].double()).any(1), torch.isnan(out).any(1)), (i, h)
        else:
            c.check(c.run())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scales_of_very_different_size(dtype):
    """int8 values whose scales differ by 2^20, and keys whose products are large: weights stay in range, and the rows of
    zero scales are what they are."""
    c = Case([1, 30], [300, 200], 2, 3, 64, 32, dtype, "i8", seed=2)
    g = torch.Generator(device=DEV).manual_seed(1)
    c.vs *= 2.0 ** torch.randint(-20, 1, c.vs.shape, device=DEV, generator=g)
    c.ks *= 3
    page, off = int(c.table_host[0, 1]), 7
    c.vs[page, :, off], c.ks[page, :, off] = 0.0, 0.0
    c.v[page, :, off], c.k[page, :, off] = 0, 0
    c.check(c.run())


def test_results_do_not_depend_on_the_stream_or_the_run():
    c = Case([1, 100, 1], [3000, 900, 10], 2, 4, 128, 16, "bf16", "i8", seed=4)
    first = c.run()
    side = torch.cuda.Stream()
    for _ in range(3):
        again = c.run(stream=side)
        assert torch.equal(first.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("cache", ["i8", "same"])
def test_offsets_beyond_32_bits(cache):
    """A cache whose last pages lie more than 2^32 bytes from its first."""
    heads, dim, page = 8, 128, 64
    per_page = heads * dim * page * (1 if cache == "i8" else 2)
    pages = (1 << 32) // per_page + 40
    k = torch.empty(pages, heads, page, dim, dtype=torch.int8 if cache == "i8" else torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    c = Case([1, 80], [200, 300], heads, 1, dim, page, "bf16", cache, seed=8)
    shift = pages - c.pages
    k[shift:], v[shift:] = c.k, c.v
    ks = vs = None
    if cache == "i8":
        ks, vs = (torch.empty(pages, heads, page, device=DEV) for _ in range(2))
        ks[shift:], vs[shift:] = c.ks, c.vs
    want = c.run()
    c.handle = B.kv_cache(k, v, ks, vs, B.I8 if cache == "i8" else B.BF16, pages, page, heads, dim)
    c.table = torch.where((c.table >= 0) & (c.table < c.pages), c.table + shift, c.table)
    got = c.run()
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))
    # and the cache's own way there
    x = torch.randn(5, heads * dim, device=DEV).to(torch.bfloat16)
    slots = torch.tensor([pages * page - 1 - i for i in range(5)], device=DEV)
    B.abft_kv_write(c.handle, 5, slots, x, heads * dim, x, heads * dim, B.BF16)
    a, b = torch.empty_like(x), torch.empty_like(x)
    B.abft_kv_read(c.handle, 5, slots, a, heads * dim, b, heads * dim, B.BF16)
    torch.cuda.synchronize()
    top = x.view(5, heads, dim).abs().amax(-1, keepdim=True).double()
    assert ((a.view(5, heads, dim).double() - x.view(5, heads, dim).double()).abs() <= top / 127 / 2 + 2.0 ** -8 * top).all()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_nothing_to_do():
    c = Case([1], [5], 1, 1, 16, 16, "f16", "i8")
    B.abft_attention(c.handle, 1, None, None, None, 1, 0, 0, 5, None, 16, 1, B.F16, 1.0, True, 0, None, 16)


def test_attention_in_a_graph():
    """One captured launch sequence over changing lengths, with the program's own work between the replays."""
    c = Case([1] * 6, [900, 3, 2000, 64, 65, 1], 2, 4, 64, 16, "f16", "i8", seed=6, poison=False)
    out = torch.empty(c.total, c.hq, c.dim, dtype=c.t, device=DEV)
    n = B.abft_attention_workspace_bytes(c.handle, 6, 6, 1, 2000, c.hq, c.dt)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)

    def call():
        B.abft_attention(c.handle, 6, c.q_start, c.kv_len, c.table, c.width, 6, 1, 2000, c.Q, c.ldq, c.hq, c.dt, c.scale, True, 0, out, c.hq * c.dim,
                         workspace=ws, workspace_bytes=n)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        c.kv_len.copy_(torch.tensor([900 - 200 * step, 3, 2000 - step, 64 - step, 65, step], dtype=torch.int32))
        c.kv = c.kv_len.tolist()
        c.Q.normal_()
        call()
        torch.cuda.synchronize()
        want = out.clone()
        c.check(want)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("dtype,cache", both("bf16") + both("f16"))
@pytest.mark.parametrize("q,kv,heads,group,dim,window", [
    ([16], [20000], 2, 4, 128, 0),                          # one row tile of which half is empty, dozens of pieces
    ([70, 3], [9000, 7777], 1, 8, 64, 0),                   # several row tiles, each with many
    ([33, 1, 2], [12001, 12001, 40], 2, 3, 80, 0),          # beside single tokens
    ([16], [30000], 3, 4, 96, 9000),                        # and in a window
    ([2] * 112, [64] * 111 + [20000], 9, 1, 64, 0),         # more counters wanted than there are
])
def test_many_pieces(q, kv, heads, group, dim, window, dtype, cache):
    c = Case(q, kv, heads, group, dim, 64, dtype, cache, seed=11, window=window)
    got = c.run()
    c.check(got)
    # (whoever comes last joins the pieces: always in the same order)
    for _ in range(3):
        assert torch.equal(c.run(), got)


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
@pytest.mark.parametrize("rows", [1, 60000])
def test_many_small_weights(rows, dtype, cache):
    """A million keys of e^-18 (less than 2^-25) of the largest weight each: together 1.6 %, which must not get lost, also where
    one wavefront goes through all of them (as many rows as fill the chip without dividing the keys).

    Bound, as above but with the roundings of the sums and those of an exponent, which have different sizes, apart:
    e = 2^-24 (keys / 16 + (dim + 64) (1 + max_j scale sum |q k_j|)); and fp16 weights 2^7 above the largest's, small = 2^-32 sum |v_j|."""
    dt, t, u, tiny = TYPES[dtype]
    n, dim, page = 1 << 20, 16, 4096
    g = torch.Generator(device=DEV).manual_seed(3)
    k = torch.zeros(n // page, 1, page, dim, device=DEV)
    k[..., 0] = -6
    k[5, 0, 77, 0] = 0     # the one key of weight 1
    v = torch.randint(64, 128, k.shape, device=DEV, generator=g).float()
    ks = vs = None
    if cache == "i8":
        ks, vs = (torch.full(k.shape[:3], step, device=DEV) for step in (1.0, 1 / 128))
        k, v = k.to(torch.int8), v.to(torch.int8)
    else:
        k, v = k.to(t), (v / 128).to(t)
    q = torch.zeros(rows, dim, dtype=t, device=DEV)
    q[:, 0] = 3
    out = torch.empty(rows, dim, dtype=t, device=DEV)
    table = torch.arange(n // page, dtype=torch.int32, device=DEV)
    q_start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    kv_len = torch.tensor([n], dtype=torch.int32, device=DEV)
    handle = B.kv_cache(k, v, ks, vs, B.I8 if cache == "i8" else dt, n // page, page, 1, dim)
    size = B.abft_attention_workspace_bytes(handle, 1, rows, rows, n, 1, dt)
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    B.abft_attention(handle, 1, q_start, kv_len, table, n // page, rows, rows, n, q, dim, 1, dt, 1.0, False, 0, out, dim, workspace=ws, workspace_bytes=size)
    torch.cuda.synchronize()
    values = v.double().reshape(n, dim) * (1 / 128 if cache == "i8" else 1)
    w = torch.exp(3 * k.double().reshape(n, dim)[:, 0])
    want = (w @ values) / w.sum()
    e = 2.0 ** -24 * (n / 16 + (dim + 64) * 19)
    small = 2.0 ** -32 * values.sum(0) if dtype == "f16" else torch.zeros_like(want)
    err = (out.double() - want).abs()
    bound = (2 * u + 2 * e) * want + small + tiny
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("dtype,cache", TYPES_AND_CACHES)
@pytest.mark.parametrize("q,kv,heads,group,dim", [
    ([1] * 127 + [40], [30] * 127 + [9000], 8, 1, 64), ([1] * 150 + [16, 300, 0, 2], [17] * 150 + [7000, 900, 5, 3000], 8, 2, 32), ([33] + [1] * 22, [8000] + [100] * 22, 32, 1, 64),
    ([2] * 140, [1500] * 140, 8, 1, 16)])
def test_pieces_beside_many_sequences(q, kv, heads, group, dim, dtype, cache):
    """Chunks whose keys are divided beside more sequences than there are counters for, were each a row tile; and row tiles beyond the counters."""
    c = Case(q, kv, heads, group, dim, 64, dtype, cache, seed=12)
    got = c.run()
    c.check(got)
    assert torch.equal(c.run(), got)
