"""int8 layers with a residual behind them, and gated pairs of projections, against their definitions in 64 bits.

Bounds.  A value z of the product (its sum exact, by definition of int8 products here) takes three roundings to fp32, as in the scaled
product: dz = 2^-22 (|scaled| + |z|).  An activation function has a slope of at most 1.13 and an error of its own: with
below(z) = |act(-|z|)|, what it keeps of the side it cuts, an exponential whose argument of at most z^2 + 8 is rounded a few times, a
reciprocal and, for GELU, a polynomial good to 5e-7: below (z^2 + 8) 2^-21 + |act| 2^-22, and nothing below 2^-100 counts.  The addition, or the
product of the two, is one more rounding to fp32 (2^-23 of its operands), and then half a unit in the last place of the output type."""
import ctypes

import pytest
import torch

from paper_2104_09455_amd import binding as B
from test_gpu_linear_scaled import DEV, TYPES, Product, hard_rows, quantised, run_quantize

pytestmark = pytest.mark.gpu
ACTS = [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU, B.ACT_GELU, B.ACT_GELU_TANH]


def activated(z, act):
    if act != B.ACT_NONE:   # (minus infinity's limit, which the formulas do not give)
        z = torch.where(z == -float("inf"), torch.zeros_like(z), z)
    if act == B.ACT_RELU:
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == B.ACT_SILU:
        return z * torch.special.expit(z)
    if act == B.ACT_GELU:
        return z * torch.special.ndtr(z)
    if act == B.ACT_GELU_TANH:
        return z * torch.special.expit(2 * (2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3))
    return z


def act_error(z, dz, act):
    z = torch.where(torch.isfinite(z), z, torch.zeros_like(z))   # (infinities go to themselves or to 0)
    own = activated(-z.abs(), act).abs() * (z * z + 8) * 2.0 ** -21 if act > B.ACT_RELU else 0
    return 1.13 * dz + own + activated(z, act).abs() * 2.0 ** -22


class Block(Product):
    """A product whose values go on: to a residual (kind "add"), or as pairs of columns (kind "gated", N columns of C)."""

    def __init__(self, kind, M, N, K, dtype, layout, seed, pad=0, offset=0, bias=True):
        self.kind, self.cols = kind, N
        super().__init__(M, 2 * N if kind == "gated" else N, K, dtype, layout, seed, pad, offset, bias)
        g = torch.Generator().manual_seed(seed + 1)
        self.ldc, self.ldr = N + pad, N + 2 * pad
        self.C = torch.full((M, self.ldc), 55.0, dtype=self.t, device=DEV)
        self.R = torch.full((M, self.ldr), float("nan"), dtype=self.t, device=DEV)
        self.R[:, :N] = (8 * torch.randn(M, N, generator=g)).to(self.t).to(DEV)

    def workspace(self, mode, linear=False):
        if linear:
            n = B.abft_linear_scaled_workspace_bytes(self.M, self.N, self.K, mode)
        else:
            n = B.abft_workspace_bytes(self.M, self.N, self.K, B.I8, B.abft_scaled_select(self.M, self.N, self.K, self.aligned) if mode == B.AUTO else mode)
        return (torch.full((n,), 201, dtype=torch.uint8, device=DEV) if n else None), n

    def checksums(self, aligned=None):
        rn = B.abft_region_shape(self.M, self.N, self.K, B.I8, self.aligned if aligned is None else aligned)[1]
        beta = torch.empty(B.abft_beta_bytes(self.K, self.N, rn), dtype=torch.uint8, device=DEV)
        B.abft_weight_checksum(self.K, self.N, self.Bm, self.ldb, self.layout, B.I8, beta, rn)
        return beta

    def run(self, mode, act=B.ACT_NONE, report=False, inject=None, with_beta=False, in_place=False):
        self.C.fill_(55.0)
        self.flag.zero_()
        self.rep.zero_()
        ws, n = self.workspace(mode)
        more = dict(beta=self.checksums() if with_beta else None, workspace=ws, workspace_bytes=n, fault_flag=self.flag,
                    report=self.rep if report else None, inject=inject)
        a = (self.M, self.cols, self.K, self.A, self.lda, self.rs, self.Bm, self.ldb, self.layout, self.cs, self.bias, act)
        if self.kind == "add":
            if in_place:
                self.C[:, :self.cols] = self.R[:, :self.cols]
            B.abft_gemm_scaled_add(*a, *((self.C, self.ldc) if in_place else (self.R, self.ldr)), self.C, self.ldc, self.dt, mode, **more)
        else:
            B.abft_gemm_gated(*a, self.C, self.ldc, self.dt, mode, **more)
        torch.cuda.synchronize()
        assert (self.C[:, self.cols:] == 55.0).all()
        return self.C[:, :self.cols], int(self.flag.item())

    def linear(self, x, mode, act, with_beta=False, stream=None):
        ws, n = self.workspace(mode, linear=True)
        out = torch.full((self.M, self.cols + 1), 7.0, dtype=self.t, device=DEV)
        more = dict(beta=self.checksums(self.K % 16 == 0 and self.layout == B.B_NK and self.aligned) if with_beta else None, workspace=ws, workspace_bytes=n, fault_flag=self.flag, stream=stream)
        a = (self.M, self.cols, self.K, x, x.stride(0), self.dt, self.Bm, self.ldb, self.layout, self.cs, self.bias, act)
        torch.cuda.synchronize()
        if self.kind == "add":
            B.abft_linear_scaled_add(*a, self.R, self.ldr, out, self.cols + 1, mode, **more)
        else:
            B.abft_linear_gated(*a, out, self.cols + 1, mode, **more)
        torch.cuda.synchronize()
        assert (out[:, self.cols:] == 7.0).all() and int(self.flag.item()) == 0
        return out[:, :self.cols]

    def definition(self, act):
        """(values, bounds) in 64 bits."""
        sums = self.a.to(DEV).double() @ self.b.to(DEV).double().t().contiguous()
        scaled = sums * self.rs.double()[:, None]
        # (the sum times its row's scale is a float: from 2^128 on, less half a step, infinite)
        scaled = torch.where(scaled.abs() >= 2.0 ** 128 * (1 - 2.0 ** -25), torch.sign(scaled) * float("inf"), scaled) * self.cs.double()
        z = scaled if self.bias is None else scaled + self.bias.double()
        dz = 2.0 ** -22 * (scaled.abs() + z.abs())
        dz = torch.where(torch.isfinite(z), dz, torch.zeros_like(dz))   # (infinite is infinite)
        if self.kind == "add":
            y, r = activated(z, act), self.R[:, :self.cols].double()
            want, err = y + r, act_error(z, dz, act) + 2.0 ** -23 * (y.abs() + r.abs())
        else:
            g, u, dg, du = z[:, 0::2], z[:, 1::2], dz[:, 0::2], dz[:, 1::2]
            y = activated(g, act)
            want = y * u
            err = act_error(g, dg, act) * (u.abs() + du) + y.abs() * du + 2.0 ** -23 * want.abs() + 2.0 ** -100 * u.abs()
        return want, self.u * want.abs() * (1 + 2.0 ** -8) + self.tiny + err * (1 + self.u) + 2.0 ** -100

    def check(self, got, act=B.ACT_NONE):
        want, bound = self.definition(act)
        beyond = ~torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.double()[beyond].nan_to_num(7.0), want[beyond].nan_to_num(7.0))
        got, want, bound = got[~beyond], want[~beyond], bound[~beyond]
        # (half a step of the type, u times the power of two below its largest value, beyond that value begins infinity)
        top = torch.finfo(self.t).max
        edge = top + self.u * 2.0 ** int(torch.tensor(top).double().log2().floor())
        infinite = torch.isinf(got)
        assert (want.abs() + bound >= edge)[infinite].all() and (torch.sign(want) == torch.sign(got.double()))[infinite].all()
        assert (want.abs() - bound <= edge)[~infinite].all()
        err = (got.double() - want).abs()[~infinite]
        assert (err <= bound[~infinite]).all(), float((err / bound[~infinite]).max())


# every tile of the aligned and of the generic kernels, ragged and whole: few rows, latency-bound, one round, many tiles
SHAPES = [(1, 1, 1), (1, 16, 16), (5, 3, 7), (16, 64, 128), (16, 100, 33), (1, 4096, 256), (13, 9000, 64), (17, 100, 96), (33, 129, 257), (64, 64, 64), (100, 33, 1024),
          (128, 256, 640), (300, 1000, 257), (512, 520, 512), (1000, 700, 128), (2048, 65, 256), (1536, 1100, 512), (1152, 4096, 1024), (3000, 2100, 256), (4096, 3300, 256)]


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("mode", [B.NONE, B.GLOBAL, B.THREAD])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products(M, N, K, dtype, mode, kind):
    for i, (layout, pad, offset) in enumerate(((B.B_NK, 0, 0), (B.B_KN, 0, 0), (B.B_NK, 5, 1))):
        if layout == B.B_KN and M * N > 2_000_000:
            continue
        act = ACTS[(M + N + K + mode + i) % 5]
        print(f"case {kind} {M}x{N}x{K} {dtype} mode={mode} layout={layout} pad={pad} act={act}", flush=True)
        p = Block(kind, M, N, K, dtype, layout, seed=M + N + K, pad=pad, offset=offset, bias=(M + K) % 2 == 0)
        got, flag = p.run(mode, act, with_beta=(M % 2 == 0))
        assert flag == 0
        p.check(got, act)
        first = got.clone()
        if mode != B.NONE:
            again, flag = p.run(mode, act, report=True)
            assert flag == 0 and torch.equal(first, again)
        if kind == "add":
            again, flag = p.run(mode, act, in_place=True)
            assert flag == 0 and torch.equal(first, again)


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,K", [(3, 200, 64), (16, 500, 100), (96, 200, 128), (300, 512, 384), (1152, 1024, 1024), (1200, 900, 130)])
def test_activation_functions(M, N, K, act, kind):
    """Values from far below zero to far above it, through every kernel's epilogue."""
    for dtype in ("f16", "bf16"):
        p = Block(kind, M, N, K, dtype, B.B_NK, seed=act + M)
        p.rs *= torch.logspace(-3, 1, M, device=DEV)
        got, flag = p.run(B.THREAD, act)
        assert flag == 0
        p.check(got, act)


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("mode", [B.GLOBAL, B.THREAD])
@pytest.mark.parametrize("M,N,K", [(4, 500, 256), (16, 40, 100), (70, 90, 512), (300, 260, 512), (1200, 1300, 512), (3000, 2100, 256)])
def test_planted_faults_are_flagged(M, N, K, mode, kind):
    """One flipped bit of one int32 sum: the flag goes up, and no other element changes."""
    for pad in (0, 3):
        p = Block(kind, M, N, K, "bf16", B.B_NK, seed=3, pad=pad)
        clean, flag = p.run(mode, B.ACT_SILU)
        clean = clean.clone()
        assert flag == 0
        for row, col, bit in ((0, 0, 3), (M - 1, p.N - 1, 30), (M // 2, p.N // 3, 17)):
            print(f"case planted {kind} {M}x{N}x{K} mode={mode} pad={pad} at {row},{col} bit {bit}", flush=True)
            bad, flag = p.run(mode, B.ACT_SILU, inject=B.Fault(row, col, bit, -1))
            assert flag == 1
            differs = bad.contiguous().view(torch.int16) != clean.contiguous().view(torch.int16)
            differs[row, col // 2 if kind == "gated" else col] = False
            assert not differs.any()


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("mode", [B.NONE, B.GLOBAL, B.THREAD, B.AUTO])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K,layout", [(1, 96, 64, B.B_NK), (1, 33, 7, B.B_KN), (1, 1, 17, B.B_NK), (2, 40, 130, B.B_NK), (3, 100, 1001, B.B_NK), (4, 2048, 8192, B.B_NK), (4, 50, 8193, B.B_NK),
                                          (1, 70, 32768, B.B_NK), (3, 16, 10000, B.B_NK), (1, 6000, 4096, B.B_NK), (5, 64, 256, B.B_NK), (16, 512, 4100, B.B_NK), (9, 4096, 2048, B.B_NK),
                                          (64, 5000, 512, B.B_NK), (130, 200, 300, B.B_NK), (600, 1030, 512, B.B_NK), (600, 103, 512, B.B_KN)])
def test_linear_layer_is_its_two_steps(M, N, K, layout, dtype, mode, kind):
    """Bit for bit what the quantisation and the product of its integers give, on a stream of its own."""
    act = ACTS[(M + N) % 5]
    print(f"case linear {kind} {M}x{N}x{K} {dtype} mode={mode} layout={layout} act={act}", flush=True)
    p = Block(kind, M, N, K, dtype, layout, seed=K)
    x = torch.zeros(M, K + 2, dtype=p.t, device=DEV)
    x[:, :K] = hard_rows(M, K, p.t, seed=K)
    x[:, K:] = float("nan")
    ldq = -(-K // 16) * 16
    q, scale = run_quantize(x, K, ldq)
    p.bufs.append(torch.zeros(M, ldq, dtype=torch.int8, device=DEV))
    p.bufs[-1][:, :K] = q
    p.A, p.lda, p.rs = p.bufs[-1].data_ptr(), ldq, scale
    want, flag = p.run(mode, act)
    assert flag == 0
    side = torch.cuda.Stream()
    got = p.linear(x, mode, act, with_beta=M % 2 == 0, stream=side)
    assert torch.equal(got.contiguous().view(torch.int16), want.contiguous().view(torch.int16))


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("M,N,K", [(2, 100, 64), (40, 70, 64), (300, 512, 256), (1200, 1030, 256)])
def test_nan_stays_and_touches_nothing_else(M, N, K, kind):
    """A row whose scale is NaN, a column whose bias is NaN, a residual's NaN and infinity: through every activation function."""
    for act in ACTS:
        p = Block(kind, M, N, K, "f16", B.B_NK, seed=9)
        plain, _ = p.run(B.THREAD, act)
        plain = plain.clone()
        p.rs[M // 2], p.bias[p.N // 2] = float("nan"), float("nan")
        nan = torch.zeros(M, N, dtype=torch.bool, device=DEV)
        nan[M // 2] = True
        nan[:, p.N // 2 // (2 if kind == "gated" else 1)] = True
        if kind == "add":
            p.R[0, 1], p.R[M - 1, 0] = float("nan"), float("inf")
            nan[0, 1] = True
        got, flag = p.run(B.THREAD, act)
        assert flag == 0 and torch.equal(torch.isnan(got), nan)
        if kind == "add":
            if not nan[M - 1, 0]:   # (two rows: the row whose scale is NaN)
                assert got[M - 1, 0] == float("inf")
            nan[M - 1, 0] = True
        assert torch.equal(got[~nan], plain[~nan])


@pytest.mark.parametrize("kind", ["add", "gated"])
def test_infinite_values(kind):
    """Scales that overflow: -infinity is activated to 0, +infinity stays."""
    for act in ACTS[1:]:
        for M in (2, 100):
            p = Block(kind, M, 64, 64, "bf16", B.B_NK, seed=1)
            p.bias.zero_()
            p.bias[0::2], p.bias[1::2] = -float("inf"), (float("inf") if kind == "add" else 1.0)
            p.R[:, :64] = 2.0
            got, _ = p.run(B.NONE, act)
            if kind == "add":
                assert (got[:, 0::2] == 2.0).all() and (got[:, 1::2] == float("inf")).all()
            else:
                assert (got == 0).all()


@pytest.mark.parametrize("kind", ["add", "gated"])
def test_layers_in_a_graph(kind):
    for M, N, K in ((2, 256, 384), (24, 256, 384), (300, 700, 512)):
        p = Block(kind, M, N, K, "bf16", B.B_NK, seed=5)
        ws, n = p.workspace(B.AUTO, linear=True)
        x = hard_rows(M, K, p.t, seed=0)
        out = torch.empty(M, N, dtype=p.t, device=DEV)

        def call():
            a = (M, N, K, x, K, p.dt, p.Bm, p.ldb, B.B_NK, p.cs, p.bias, B.ACT_SILU)
            if kind == "add":
                B.abft_linear_scaled_add(*a, p.R, p.ldr, out, N, B.AUTO, workspace=ws, workspace_bytes=n, fault_flag=p.flag)
            else:
                B.abft_linear_gated(*a, out, N, B.AUTO, workspace=ws, workspace_bytes=n, fault_flag=p.flag)

        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for seed in range(1, 4):
            x.copy_(hard_rows(M, K, p.t, seed=seed))
            call()
            torch.cuda.synchronize()
            want = out.clone()
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and int(p.flag.item()) == 0


def test_a_block_as_it_is_used():
    """norm -> int8 -> gated projections -> down projection onto the residual stream -> norm, for a prompt and for single tokens; each step
    bit for bit the plain steps' chain, and in all as near to 64 bits as 16-bit steps are."""
    for M, dtype in ((1, "bf16"), (4, "f16"), (70, "bf16"), (600, "f16")):
        dt, t, u, _ = TYPES[dtype]
        W, F = 512, 1000
        g = torch.Generator().manual_seed(M)
        stream = (2 * torch.randn(M, W, generator=g)).to(t).to(DEV)
        branch = torch.randn(M, W, generator=g).to(t).to(DEV)
        weight = (1 + 0.1 * torch.randn(W, generator=g)).to(DEV)
        up = torch.randint(-127, 128, (2 * F, W), generator=g, dtype=torch.int8).to(DEV)
        down = torch.randint(-127, 128, (W, F), generator=g, dtype=torch.int8).to(DEV)
        up_scale, down_scale = torch.full((2 * F,), 0.02 / W ** 0.5, device=DEV), torch.full((W,), 0.02 / F ** 0.5, device=DEV)
        flag = torch.zeros(1, dtype=torch.int32, device=DEV)
        n = max(B.abft_linear_scaled_workspace_bytes(M, 2 * F, W, B.AUTO), B.abft_linear_scaled_workspace_bytes(M, W, F, B.AUTO))
        ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        more = dict(workspace=ws, workspace_bytes=n, fault_flag=flag)
        q, scale = torch.empty(M, W, dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
        h, y = torch.empty(M, F, dtype=t, device=DEV), torch.empty(M, W, dtype=t, device=DEV)
        s = stream.clone()
        B.abft_rms_norm(M, W, branch, W, dt, weight, 1e-5, residual=s, ldr=W, total=s, ldt=W, Q=q, ldq=W, scale=scale)
        B.abft_gemm_gated(M, F, W, q, W, scale, up, W, B.B_NK, up_scale, None, B.ACT_SILU, h, F, dt, B.AUTO, **more)
        B.abft_linear_scaled_add(M, W, F, h, F, dt, down, F, B.B_NK, down_scale, None, B.ACT_NONE, s, W, s, W, B.AUTO, **more)
        B.abft_rms_norm(M, W, s, W, dt, weight, 1e-5, Y=y, ldy=W)
        torch.cuda.synchronize()
        assert int(flag.item()) == 0
        # the chain in 64 bits, rounded to 16 where the stream and the block's middle are held so
        first = (stream.double() + branch.double()).to(t).double()
        normed = (first / torch.sqrt(first.pow(2).mean(1, keepdim=True) + 1e-5) * weight.double()).to(t)
        ints, sc = quantised(normed)
        z = (ints @ up.double().t().contiguous()) * sc.double()[:, None] * up_scale.double()
        mid = (z[:, 0::2] * torch.special.expit(z[:, 0::2]) * z[:, 1::2]).to(t)
        ints, sc = quantised(mid)
        last = first + (ints @ down.double().t().contiguous()) * sc.double()[:, None] * down_scale.double()
        want = last / torch.sqrt(last.pow(2).mean(1, keepdim=True) + 1e-5) * weight.double()
        # an element of the middle that rounds the other way moves an integer by one: each of them by one half step of the largest
        # magnitude over 127, independent of each other
        off = (s.double() - last).norm() / last.norm()
        assert off < 2 * u, float(off)
        assert (y.double() - want).norm() / want.norm() < 4 * u


# (activations kept in registers: an eighth of k of one to sixteen k tiles a wavefront, k ends inside of a tile and leaves wavefronts without one,
# columns by the sixteen and by the four, one run of them a workgroup and several, rows quantised by the workgroups and before)
RESIDENT = [(1, 1, 528), (2, 40, 640), (16, 17, 1024), (3, 700, 1040), (9, 4096, 1408), (1, 12288, 2048), (5, 5000, 3008), (16, 4300, 4096), (1, 8576, 4112), (4, 5120, 5120),
            (8, 333, 6144), (7, 6000, 7040), (1, 4480, 8192), (4, 4096, 9216), (12, 260, 10240), (4, 4096, 12288), (1, 100, 14000), (2, 700, 16384), (16, 2050, 16384)]
# (a few columns of a long k loop run on the tilings: both sides of that, with the widest runs of k)
RESIDENT += [(12, 2560, 10240), (3, 2559, 10240), (1, 3600, 14000), (5, 3500, 14000), (16, 2047, 8192), (16, 2049, 8192), (2, 4098, 16384), (4, 4100, 16384), (11, 4096, 16384)]


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", RESIDENT)
def test_few_rows_of_large_weights(M, N, K, dtype, kind):
    act = ACTS[(M + N) % 5]
    print(f"case few {kind} {M}x{N}x{K} {dtype} act={act}", flush=True)
    p = Block(kind, M, N, K, dtype, B.B_NK, seed=K + M, bias=M % 2 == 0)
    p.cs *= 0.3
    x = torch.zeros(M, K + 3, dtype=p.t, device=DEV)
    x[:, :K] = hard_rows(M, K, p.t, seed=K)
    x[:, K:] = float("nan")
    got = p.linear(x, B.AUTO, act)
    q, scale = quantised(x[:, :K])
    p.a, p.rs = q.to(torch.int8).cpu(), scale
    p.check(got, act)
    # the same from integers, at any address, in every scheme
    p.lda = K + 5
    p.bufs.append(torch.full((M, p.lda), 99, dtype=torch.int8, device=DEV))
    p.bufs[-1][:, :K] = q.to(torch.int8)
    p.A = p.bufs[-1].data_ptr()
    for mode in (B.NONE, B.THREAD, B.AUTO):
        again, flag = p.run(mode, act, in_place=(kind == "add" and mode == B.THREAD))
        assert flag == 0 and torch.equal(again.contiguous().view(torch.int16), got.contiguous().view(torch.int16))
    # a report and the global scheme run on the tilings: the same bits
    for mode, report in ((B.THREAD, True), (B.GLOBAL, False)):
        again, flag = p.run(mode, act, report=report)
        assert flag == 0 and torch.equal(again.contiguous().view(torch.int16), got.contiguous().view(torch.int16))
    clean = got.contiguous().view(torch.int16).clone()
    for row, col, bit, after in ((0, 0, 4, -1), (M - 1, p.N - 1, 28, -2), (M // 2, p.N // 2, 9, -1)):
        bad, flag = p.run(B.THREAD, act, inject=B.Fault(row, col, bit, after))
        assert flag == 1
        differs = bad.contiguous().view(torch.int16) != clean
        differs[row, col // 2 if kind == "gated" else col] = False
        assert not differs.any()


def test_few_rows_whose_values_are_not_finite():
    """A row with an infinity or a NaN among rows quantised by the workgroups: NaN, the flag stays down, other rows are untouched."""
    for M, N, K in ((1, 100, 4096), (4, 700, 8192), (9, 50, 1040), (16, 64, 2048)):
        p = Block("gated", M, N, K, "bf16", B.B_NK, seed=2)
        x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).to(p.t).to(DEV)
        plain = p.linear(x, B.THREAD, B.ACT_SILU).clone()
        x[M // 2, K - 1] = float("inf")
        x[M - 1, 0] = float("nan")
        got = p.linear(x, B.THREAD, B.ACT_SILU)
        bad = torch.zeros(M, dtype=torch.bool, device=DEV)
        bad[[M // 2, M - 1]] = True
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], plain[~bad])


# (one launch that quantises and multiplies: k tiles for one to eight wavefronts, ends of k inside of a chunk, columns that end inside of four, rows
# and weights at every alignment, both orders; 256 tiles of 32 x 64 and one more)
@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(5, 2, 16), (1, 30, 17), (33, 65, 100), (12, 66, 128), (64, 3, 129), (31, 254, 500), (100, 130, 755), (7, 1000, 1000), (257, 70, 1023), (300, 200, 1024),
                                   (2048, 127, 64), (2050, 256, 200)])
def test_small_layers_in_one_launch(M, N, K, dtype, kind):
    act = ACTS[(M + K) % 5]
    for layout, pad, offset in ((B.B_NK, 0, 0), (B.B_KN, 0, 0), (B.B_NK, 3, 1), (B.B_KN, 5, 3), (B.B_NK, 2, 2)):
        print(f"case joint {kind} {M}x{N}x{K} {dtype} layout={layout} pad={pad} act={act}", flush=True)
        p = Block(kind, M, N, K, dtype, layout, seed=K + M, pad=pad, offset=offset, bias=M % 2 == 0)
        p.cs *= 0.3
        x = torch.zeros(M, K + 3, dtype=p.t, device=DEV)
        x[:, :K] = hard_rows(M, K, p.t, seed=K)
        x[:, K:] = float("nan")
        got = p.linear(x, B.AUTO, act).clone()
        q, scale = quantised(x[:, :K])
        p.a, p.rs = q.to(torch.int8).cpu(), scale
        p.check(got, act)
        assert torch.equal(bits16(p.linear(x, B.NONE, act)), bits16(got))
        # the global scheme runs on the tilings: the same bits
        assert torch.equal(bits16(p.linear(x, B.GLOBAL, act)), bits16(got))
        ws, n = p.workspace(B.THREAD, linear=True)
        for row, col, bit, after in ((0, 0, 4, -1), (M - 1, p.N - 1, 28, -2), (M // 2, p.N // 2, 9, -1)):
            out = torch.empty(M, N, dtype=p.t, device=DEV)
            p.flag.zero_()
            a = (M, N, K, x, x.stride(0), p.dt, p.Bm, p.ldb, layout, p.cs, p.bias, act)
            more = dict(workspace=ws, workspace_bytes=n, fault_flag=p.flag, inject=B.Fault(row, col, bit, after))
            if kind == "add":
                B.abft_linear_scaled_add(*a, p.R, p.ldr, out, N, B.THREAD, **more)
            else:
                B.abft_linear_gated(*a, out, N, B.THREAD, **more)
            torch.cuda.synchronize()
            assert int(p.flag.item()) == 1
            p.flag.zero_()
            differs = bits16(out) != bits16(got)
            differs[row, col // 2 if kind == "gated" else col] = False
            assert not differs.any()


def bits16(x):
    return x.contiguous().view(torch.int16)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 8200), (5, 12288), (300, 16384), (3, 16385)])
def test_long_rows_are_quantised_exactly(M, K, dtype):
    """The rows of down projections: held in registers up to 16384 values, beyond that read twice."""
    _, t, _, _ = TYPES[dtype]
    x = hard_rows(M, K, t, seed=M + K)
    q, scale = run_quantize(x, K, K)
    want, want_scale = quantised(x)
    assert torch.equal(scale, want_scale) and torch.equal(q.double(), want)
