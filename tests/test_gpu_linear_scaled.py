"""Per-token quantisation, the scaled int8 product and the two in one call, against their definitions in 64 bits.

Bounds.  The integers have to be equal and the scales equal to the last bit: 127 x is exact and the quotient is either
an exact half or at least 2^-19 of itself away from one (see quantize.h).  An element of the product takes the integer
sum (equal, by definition of int8 products here) through three roundings to fp32 (2^-24 each: to float, times the row's
scale, the fused step) and one to the output type (half a unit in the last place: 2^-11 or 2^-8 of the value, or half the
smallest subnormal)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2104_09455_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": (B.F16, torch.float16, 2.0 ** -11, 2.0 ** -25), "bf16": (B.BF16, torch.bfloat16, 2.0 ** -8, 2.0 ** -134)}
GUARD = 77   # bytes around outputs that have to stay as they are


def quantised(x):
    """(integers, scales as floats) of the rows of a 16-bit tensor, in 64 bits; rows with anything not finite: zeros, NaN."""
    d = x.double()
    top = d.abs().amax(1)
    finite = torch.isfinite(d).all(1)
    safe = torch.where((top > 0) & finite, top, torch.ones_like(top))[:, None]
    ratio = torch.where(finite[:, None], d, torch.zeros_like(d)) * 127 / safe
    q = torch.where(ratio < 0, torch.ceil(ratio - 0.5), torch.floor(ratio + 0.5))
    return q, (torch.where(finite, top, torch.full_like(top, float("nan"))) / 127).float()


def run_quantize(x, K, ldq, offset=0):
    """The library's quantisation of the first K columns of a tensor whose rows may be longer."""
    dt = B.F16 if x.dtype == torch.float16 else B.BF16
    M = x.shape[0]
    q = torch.full((offset + M * ldq + 64,), GUARD, dtype=torch.int8, device=DEV)
    scale = torch.full((M + 4,), -5.0, device=DEV)
    B.abft_quantize_rows(M, K, x, x.stride(0), dt, q.data_ptr() + offset, ldq, scale)
    torch.cuda.synchronize()
    body = q[offset:offset + M * ldq].view(M, ldq)
    assert (body[:, K:] == GUARD).all() and (q[:offset] == GUARD).all() and (q[offset + M * ldq:] == GUARD).all()
    assert (scale[M:] == -5.0).all()
    return body[:, :K], scale[:M]


def hard_rows(M, K, dtype, seed):
    """Rows of normal values of very different size, and in turn rows of zeros, of one value only, of exact halves (the
    largest magnitude a multiple of 127: every 127 x / a is a multiple of a half or so), of subnormals, and of the type's
    largest value."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g).double() * 2.0 ** torch.randint(-8, 9, (M, 1), generator=g).double()
    for m in range(M):
        if m % 7 == 1:
            x[m] = 0
        elif m % 7 == 2:
            x[m] = torch.where(torch.rand(K, generator=g) < 0.5, -1.5, 1.5).double()
        elif m % 7 == 3:
            x[m] = torch.randint(-254, 255, (K,), generator=g).double() / 2
            x[m, 0] = 127.0
        elif m % 7 == 4:
            x[m] *= 2.0 ** (-22 if dtype == torch.float16 else -130)
        elif m % 7 == 5:
            x[m, K // 2] = -torch.finfo(dtype).max
    return x.to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 5), (9, 8), (5, 77), (13, 512), (7, 513), (5, 2048), (1030, 2000), (8, 2049), (3, 8192), (9, 8193), (2, 20011)])
def test_quantised_rows_are_exact(M, K, dtype):
    _, t, _, _ = TYPES[dtype]
    for pad, offset in ((0, 0), (3, 1)):
        print(f"case quantize {M}x{K} {dtype} pad={pad}", flush=True)
        x = torch.zeros(M, K + pad, dtype=t, device=DEV)
        x[:, :K] = hard_rows(M, K, t, seed=M + K)
        x[:, K:] = float("nan")   # behind the rows' ends
        q, scale = run_quantize(x, K, K + pad, offset)
        want, want_scale = quantised(x[:, :K])
        assert torch.equal(scale, want_scale)
        assert torch.equal(q.double(), want)


@pytest.mark.parametrize("K", [1, 9])
def test_more_rows_than_a_launch_holds(K):
    """2^26 rows, four a workgroup: more than 2^32 threads."""
    M = (1 << 26) + 5
    x = torch.zeros(M, K, dtype=torch.float16, device=DEV)
    places = [0, 1, (1 << 23) - 1, 1 << 23, (1 << 25) - 1, 1 << 25, M - 6, M - 1]
    x[places] = torch.randn(len(places), K, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.float16)
    q = torch.full((M, K), GUARD, dtype=torch.int8, device=DEV)
    scale = torch.full((M,), -5.0, device=DEV)
    B.abft_quantize_rows(M, K, x, K, B.F16, q, K, scale)
    torch.cuda.synchronize()
    want, want_scale = quantised(x[places])
    assert torch.equal(q[places].double(), want) and torch.equal(scale[places], want_scale)
    assert int((scale != 0).sum()) == len(places) and int((q != 0).any(1).sum()) == len(places)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_that_are_not_finite_have_scale_nan(dtype):
    _, t, _, _ = TYPES[dtype]
    x = hard_rows(6, 300, t, seed=1)
    x[0, 3], x[2, 299], x[4, 0] = float("inf"), float("nan"), -float("inf")
    q, scale = run_quantize(x, 300, 300)
    want, want_scale = quantised(x)
    assert torch.equal(torch.isnan(scale), torch.isnan(want_scale)) and torch.isnan(scale[[0, 2, 4]]).all()
    assert torch.equal(q.double(), want) and (q[[0, 2, 4]] == 0).all()


class Product:
    """Operands of a scaled product on the device, at chosen paddings and offsets."""

    def __init__(self, M, N, K, dtype, layout, seed, pad=0, offset=0, bias=True):
        g = torch.Generator().manual_seed(seed)
        self.M, self.N, self.K, self.layout, self.pad = M, N, K, layout, pad
        self.dt, self.t, self.u, self.tiny = TYPES[dtype]
        self.a = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8)
        self.b = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int8)
        self.rs = (torch.rand(M, generator=g) * 0.05 + 1e-4).to(DEV)
        self.cs = (torch.rand(N, generator=g) * 0.01 + 1e-5).to(DEV)
        self.bias = (torch.randn(N, generator=g) * 3).to(DEV) if bias else None
        self.lda, self.ldb, self.ldc = K + pad, (K if layout == B.B_NK else N) + pad, N + pad
        self.bufs = []

        def place(x, ld):
            buf = torch.full((offset + x.shape[0] * ld,), 99, dtype=torch.int8)
            buf[offset:].view(x.shape[0], ld)[:, :x.shape[1]] = x
            self.bufs.append(buf.to(DEV))
            return self.bufs[-1].data_ptr() + offset

        self.A = place(self.a, self.lda)
        self.Bm = place(self.b if layout == B.B_NK else self.b.t().contiguous(), self.ldb)
        self.aligned = offset == 0 and pad % 16 == 0 and K % 16 == 0 and layout == B.B_NK
        self.C = torch.full((M, self.ldc), 55.0, dtype=self.t, device=DEV)
        self.flag = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.rep = torch.zeros(ctypes.sizeof(B.Report), dtype=torch.uint8, device=DEV)

    def run(self, mode, act=B.ACT_NONE, report=False, inject=None, with_beta=False):
        self.C.fill_(55.0)
        self.flag.zero_()
        self.rep.zero_()
        n = B.abft_workspace_bytes(self.M, self.N, self.K, B.I8, B.abft_scaled_select(self.M, self.N, self.K, self.aligned) if mode == B.AUTO else mode)
        ws = torch.full((n,), 201, dtype=torch.uint8, device=DEV) if n else None
        beta = None
        if with_beta:
            rn = B.abft_region_shape(self.M, self.N, self.K, B.I8, self.aligned)[1]
            beta = torch.empty(B.abft_beta_bytes(self.K, self.N, rn), dtype=torch.uint8, device=DEV)
            B.abft_weight_checksum(self.K, self.N, self.Bm, self.ldb, self.layout, B.I8, beta, rn)
        B.abft_gemm_scaled(self.M, self.N, self.K, self.A, self.lda, self.rs, self.Bm, self.ldb, self.layout, self.cs, self.bias, act,
                           self.C, self.ldc, self.dt, mode, beta=beta, workspace=ws, workspace_bytes=n, fault_flag=self.flag,
                           report=self.rep if report else None, inject=inject)
        torch.cuda.synchronize()
        assert (self.C[:, self.N:] == 55.0).all()
        return self.C[:, :self.N], int(self.flag.item())

    def check(self, got, act=B.ACT_NONE):
        sums = self.a.to(DEV).double() @ self.b.to(DEV).double().t().contiguous()
        scaled = sums * self.rs.double()[:, None] * self.cs.double()
        want = scaled if self.bias is None else scaled + self.bias.double()
        if act == B.ACT_RELU:
            want = want.clamp(min=0)
        bound = self.u * want.abs() + self.tiny + 2.0 ** -22 * (scaled.abs() + want.abs())
        err = (got.double() - want).abs()
        assert (err <= bound).all(), float((err / bound).max())


# every tile of the aligned and of the generic kernels, ragged and whole: few rows, latency-bound, one round, many tiles
SHAPES = [(1, 1, 1), (1, 16, 16), (5, 3, 7), (16, 64, 128), (16, 100, 33), (1, 4096, 256), (13, 9000, 64), (17, 100, 96), (33, 129, 257), (64, 64, 64), (100, 33, 1024),
          (128, 256, 640), (300, 1000, 257), (512, 520, 512), (1000, 700, 128), (2048, 65, 256), (1536, 1100, 512), (1152, 4096, 1024), (3000, 2100, 256),
          (4096, 3300, 256)]


@pytest.mark.parametrize("mode", [B.NONE, B.GLOBAL, B.THREAD])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_scaled_product(M, N, K, dtype, mode):
    for layout, pad, offset in ((B.B_NK, 0, 0), (B.B_KN, 0, 0), (B.B_NK, 5, 1)):
        if layout == B.B_KN and M * N > 2_000_000:
            continue
        print(f"case scaled {M}x{N}x{K} {dtype} mode={mode} layout={layout} pad={pad}", flush=True)
        p = Product(M, N, K, dtype, layout, seed=M + N + K, pad=pad, offset=offset, bias=(M + K) % 2 == 0)
        act = B.ACT_RELU if N % 2 else B.ACT_NONE
        got, flag = p.run(mode, act, with_beta=(M % 2 == 0))
        assert flag == 0
        p.check(got, act)
        if mode != B.NONE:
            first = got.clone()
            again, flag = p.run(mode, act, report=True)
            assert flag == 0 and torch.equal(first, again)


@pytest.mark.parametrize("mode", [B.GLOBAL, B.THREAD])
@pytest.mark.parametrize("M,N,K", [(4, 500, 256), (16, 40, 100), (70, 90, 512), (300, 260, 512), (1200, 1300, 512), (3000, 2100, 256)])
def test_planted_faults_are_flagged(M, N, K, mode):
    """One flipped bit of one int32 sum: the flag goes up, and no other element changes."""
    for pad in (0, 3):
        p = Product(M, N, K, "bf16", B.B_NK, seed=3, pad=pad)
        clean, flag = p.run(mode)
        clean = clean.clone()
        assert flag == 0
        for row, col, bit in ((0, 0, 3), (M - 1, N - 1, 30), (M // 2, N // 3, 17)):
            print(f"case planted {M}x{N}x{K} mode={mode} pad={pad} at {row},{col} bit {bit}", flush=True)
            bad, flag = p.run(mode, inject=B.Fault(row, col, bit, -1))
            assert flag == 1
            differs = bad != clean
            differs[row, col] = False
            assert not differs.any()


def test_scales_that_are_nan_or_zero():
    """A row of zeros leaves the bias, a row whose scale is NaN is NaN, and neither touches another row."""
    p = Product(40, 70, 64, "f16", B.B_NK, seed=9)
    p.rs[3], p.rs[7] = 0.0, float("nan")
    got, flag = p.run(B.THREAD)
    assert flag == 0
    assert torch.equal(got[3].double(), p.bias.to(torch.float16).double())
    assert torch.isnan(got[7]).all()
    assert torch.isfinite(got[[i for i in range(40) if i != 7]]).all()


# (every store of C: the few rows' kernel, skinny, streaming, direct-to-LDS and generic tiles, whole and cut)
@pytest.mark.parametrize("mode", [B.NONE, B.GLOBAL, B.THREAD])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K,layout", [(1, 96, 64, B.B_NK), (2, 40, 130, B.B_KN), (4, 4096, 256, B.B_NK), (9, 200, 256, B.B_NK), (64, 64, 64, B.B_NK), (100, 33, 1024, B.B_NK),
                                      (130, 200, 300, B.B_NK), (70, 65, 33, B.B_KN), (512, 520, 512, B.B_NK), (1000, 700, 128, B.B_NK), (1152, 4096, 1024, B.B_NK), (3000, 2100, 257, B.B_NK)])
def test_relu_keeps_what_is_not_a_number(M, N, K, layout, dtype, mode):
    """Rows that hold an infinity or a NaN, and columns whose scale or bias is NaN, are NaN behind the activation function too;
    everything else is what it makes of the layer's values.  (The sums of such a row are zeros: no check sees it.)"""
    print(f"case relu {M}x{N}x{K} {dtype} mode={mode} layout={layout}", flush=True)
    p = Product(M, N, K, dtype, layout, seed=M)
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).to(p.t).to(DEV)
    bad = sorted({0, M // 2, M - 1} - ({0} if 1 < M < 4 else set()))
    for i, m in enumerate(bad):
        x[m, (7 * m + 3) % K] = [float("inf"), float("nan"), -float("inf")][(i + M) % 3]
    p.cs[N // 2], p.bias[N - 1] = float("nan"), float("nan")
    n = B.abft_linear_scaled_workspace_bytes(M, N, K, mode)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    outs = []
    for act in (B.ACT_NONE, B.ACT_RELU):
        outs.append(torch.full((M, N), 7.0, dtype=p.t, device=DEV))
        B.abft_linear_scaled(M, N, K, x, K, p.dt, p.Bm, p.ldb, layout, p.cs, p.bias, act, outs[-1], N, mode, workspace=ws, workspace_bytes=n, fault_flag=p.flag)
    torch.cuda.synchronize()
    plain, got = outs
    rows = torch.zeros(M, dtype=torch.bool, device=DEV)
    rows[bad] = True
    columns = torch.zeros(N, dtype=torch.bool, device=DEV)
    columns[[N // 2, N - 1]] = True
    assert torch.equal(torch.isnan(plain), rows[:, None] | columns)
    assert torch.equal(torch.isnan(got), torch.isnan(plain))
    number = ~torch.isnan(plain)
    assert torch.equal(got[number], plain[number].clamp(min=0))


@pytest.mark.parametrize("mode", [B.NONE, B.GLOBAL, B.THREAD, B.AUTO])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K,layout", [(1, 96, 64, B.B_NK), (1, 33, 7, B.B_KN), (1, 1, 17, B.B_NK), (2, 40, 130, B.B_NK), (3, 100, 1001, B.B_NK), (4, 4096, 8192, B.B_NK), (4, 50, 8193, B.B_NK), (1, 70, 32768, B.B_NK),
                                      (3, 16, 10000, B.B_NK), (5, 64, 256, B.B_NK), (16, 512, 4100, B.B_NK), (9, 4096, 2048, B.B_NK), (130, 200, 300, B.B_NK), (600, 1030, 512, B.B_NK)])
def test_linear_layer_is_its_two_steps(M, N, K, layout, dtype, mode):
    """Bit for bit what the quantisation and the scaled product give, on a stream of its own."""
    p = Product(M, N, K, dtype, layout, seed=K)
    x = torch.zeros(M, K + 2, dtype=p.t, device=DEV)
    x[:, :K] = hard_rows(M, K, p.t, seed=K)
    x[:, K:] = float("nan")
    ldq = -(-K // 16) * 16
    q, scale = run_quantize(x, K, ldq)
    p.bufs.append(torch.zeros(M, ldq, dtype=torch.int8, device=DEV))
    p.bufs[-1][:, :K] = q
    p.A, p.lda, p.rs = p.bufs[-1].data_ptr(), ldq, scale
    want, flag = p.run(mode)
    assert flag == 0
    n = B.abft_linear_scaled_workspace_bytes(M, N, K, mode)
    ws = torch.full((n,), 131, dtype=torch.uint8, device=DEV)
    out = torch.full((M, N), 7.0, dtype=p.t, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.abft_linear_scaled(M, N, K, x, x.stride(0), p.dt, p.Bm, p.ldb, layout, p.cs, p.bias, B.ACT_NONE, out, N, mode, workspace=ws,
                             workspace_bytes=n, fault_flag=p.flag)
    side.synchronize()
    assert int(p.flag.item()) == 0
    assert torch.equal(out.view(torch.int16), want.contiguous().view(torch.int16))


# (one launch: rows of one, two and four chunks a thread; wavefronts with few k tiles, with many, and, at 4225 and 5119, both in a workgroup)
@pytest.mark.parametrize("mode", [B.NONE, B.THREAD])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(4, 512, 4096), (3, 100, 4095), (2, 512, 8192), (2, 70, 4225), (1, 70, 4225), (1, 512, 16384), (1, 70, 8209), (1, 64, 8320),
                                   (2, 33, 5119), (1, 33, 16383)])
def test_few_rows_of_long_products(M, N, K, dtype, mode):
    """The sums from the quantisation's definition, in 64 bits, and bit for bit the two calls' results."""
    print(f"case few {M}x{N}x{K} {dtype} mode={mode}", flush=True)
    p = Product(M, N, K, dtype, B.B_NK, seed=K + M)
    x = torch.zeros(M, K + 3, dtype=p.t, device=DEV)
    x[:, :K] = hard_rows(M, K, p.t, seed=K)
    x[:, K:] = float("nan")
    n = B.abft_linear_scaled_workspace_bytes(M, N, K, mode)
    ws = torch.full((n,), 131, dtype=torch.uint8, device=DEV)
    out = torch.full((M, N), 7.0, dtype=p.t, device=DEV)
    B.abft_linear_scaled(M, N, K, x, K + 3, p.dt, p.Bm, p.ldb, B.B_NK, p.cs, p.bias, B.ACT_NONE, out, N, mode, workspace=ws, workspace_bytes=n,
                         fault_flag=p.flag)
    torch.cuda.synchronize()
    assert int(p.flag.item()) == 0
    q, scale = quantised(x[:, :K])
    p.a, p.rs = q.to(torch.int8).cpu(), scale
    p.check(out)
    ldq = -(-K // 16) * 16
    p.bufs.append(torch.zeros(M, ldq, dtype=torch.int8, device=DEV))
    p.bufs[-1][:, :K] = q.to(torch.int8)
    p.A, p.lda = p.bufs[-1].data_ptr(), ldq
    want, flag = p.run(mode)
    assert flag == 0 and torch.equal(out.view(torch.int16), want.contiguous().view(torch.int16))


@pytest.mark.parametrize("M", [1, 4])
def test_few_rows_with_a_report_or_a_planted_fault(M):
    """Calls that cannot take the few rows' kernel give its results, and see a fault."""
    p = Product(M, 200, 520, "f16", B.B_NK, seed=M)
    x = hard_rows(M, 520, p.t, seed=2)
    n = B.abft_linear_scaled_workspace_bytes(M, 200, 520, B.THREAD)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    outs = []
    for report, inject in ((None, None), (p.rep, None), (None, B.Fault(M - 1, 77, 20, -1))):
        out = torch.empty(M, 200, dtype=p.t, device=DEV)
        p.flag.zero_()
        B.abft_linear_scaled(M, 200, 520, x, 520, p.dt, p.Bm, p.ldb, B.B_NK, p.cs, p.bias, B.ACT_NONE, out, 200, B.THREAD, workspace=ws, workspace_bytes=n,
                             fault_flag=p.flag, report=report, inject=inject)
        torch.cuda.synchronize()
        assert int(p.flag.item()) == (1 if inject else 0)
        outs.append(out.view(torch.int16).clone())
    assert torch.equal(outs[0], outs[1])
    differs = outs[0] != outs[2]
    differs[M - 1, 77] = False
    assert not differs.any()


@pytest.mark.parametrize("M", [1, 4, 9, 200])
def test_events_around_the_product(M):
    """The measurement hook records both events in every form of the call: behind what the stream held when it was made."""
    N, K = 300, 512
    p = Product(M, N, K, "f16", B.B_NK, seed=M)
    x = hard_rows(M, K, p.t, seed=1)
    n = B.abft_linear_scaled_workspace_bytes(M, N, K, B.THREAD)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    start, stop, made = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    start.record()
    stop.record()
    torch.zeros(1 << 24, device=DEV).sin_()   # (time goes by on the stream)
    made.record()
    B.abft_set_kernel_events(start.cuda_event, stop.cuda_event)
    try:
        B.abft_linear_scaled(M, N, K, x, K, p.dt, p.Bm, p.ldb, B.B_NK, p.cs, p.bias, B.ACT_NONE, p.C, p.ldc, B.THREAD, workspace=ws, workspace_bytes=n,
                             fault_flag=p.flag)
    finally:
        B.abft_set_kernel_events(None, None)
    torch.cuda.synchronize()
    assert made.elapsed_time(start) >= 0 and start.elapsed_time(stop) > 0


def test_linear_layer_in_a_graph():
    M, N, K = 24, 256, 384
    p = Product(M, N, K, "bf16", B.B_NK, seed=5)
    n = B.abft_linear_scaled_workspace_bytes(M, N, K, B.AUTO)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    x = hard_rows(M, K, p.t, seed=0)
    out = torch.empty(M, N, dtype=p.t, device=DEV)

    def call():
        B.abft_linear_scaled(M, N, K, x, K, p.dt, p.Bm, p.ldb, B.B_NK, p.cs, p.bias, B.ACT_NONE, out, N, B.AUTO, workspace=ws,
                             workspace_bytes=n, fault_flag=p.flag)

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
