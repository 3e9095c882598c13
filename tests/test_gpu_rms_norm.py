"""Root-mean-square norm of rows against its definition in 64 bits.

Bounds.  The sum with the residual is one fp32 addition rounded to 16 bits, and has to be equal.  A normed value takes the rounding to
16 bits (half a unit in the last place, or half the smallest subnormal) and the fp32 steps before it: the mean of squares is a sum of
n = K / 64 or fewer squares in a thread, a tree of eight additions, a division and eps, so off by at most (n + 12) 2^-24 of itself, its
root by half of that; root, reciprocal and three products add 2^-24 to 2^-23 each.  Integers and scales are those of the quantisation
of the 16-bit result, bit for bit."""
import pytest
import torch

from paper_2104_09455_amd import binding as B
from test_gpu_linear_scaled import GUARD, TYPES, hard_rows, run_quantize

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


def bits(x):
    return x.contiguous().view(torch.int16)


class Rows:
    """Rows on the device, `pad` elements longer than K and `offset` elements off their buffer's start, NaN all around."""

    def __init__(self, x, pad=0, offset=0):
        M, self.K = x.shape
        self.ld = self.K + pad
        self.buf = torch.full((offset + M * self.ld + 8,), float("nan"), dtype=x.dtype, device=DEV)
        self.view = self.buf[offset:offset + M * self.ld].view(M, self.ld)
        self.view[:, :self.K] = x.to(DEV)
        self.ptr = self.buf.data_ptr() + 2 * offset

    @property
    def rows(self):
        return self.view[:, :self.K]

    def clean(self):
        outside = torch.ones_like(self.buf, dtype=torch.bool)
        n = self.view.numel()
        at = (self.ptr - self.buf.data_ptr()) // 2
        outside[at:at + n].view(self.view.shape)[:, :self.K] = False
        return bool(torch.isnan(self.buf[outside]).all())


def definition(s, weight, eps):
    d = s.double()
    y = d / torch.sqrt(d.pow(2).mean(1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32)))
    return y if weight is None else y * weight.double()


def check(got, s, weight, dtype, eps=EPS):
    _, t, u, tiny = TYPES[dtype]
    want = definition(s, weight, eps)
    K = s.shape[1]
    over = want.abs() >= torch.finfo(t).max * (1 - u)    # (rounds to the largest value or infinity)
    bound = want.abs() * (u + ((K / 64 + 12) / 2 + 12) * 2.0 ** -24) + tiny
    assert torch.isfinite(got[~over]).all()
    err = (got.double() - want).abs()[~over]
    assert (err <= bound[~over]).all(), float((err / bound[~over]).max())


def run(x, dtype, K, residual=None, weight=None, eps=EPS, total=None, y=True, q=False, pad=0, offset=0, stream=None):
    """(sum or None, y or None, (integers, scales) or None) of a call whose outputs have what surrounds them looked at."""
    dt, t, _, _ = TYPES[dtype]
    M = x.rows.shape[0]
    out = Rows(torch.zeros(M, K, dtype=t), pad, offset) if y else None
    ldq = K + pad
    ints = torch.full((offset + M * ldq + 64,), GUARD, dtype=torch.int8, device=DEV) if q else None
    scale = torch.full((M + 4,), -5.0, device=DEV) if q else None
    B.abft_rms_norm(M, K, x.ptr, x.ld, dt, weight, eps, residual=residual.ptr if residual else None, ldr=residual.ld if residual else 0,
                    total=total.ptr if total else None, ldt=total.ld if total else 0, Y=out.ptr if y else None, ldy=out.ld if y else 0,
                    Q=ints.data_ptr() + offset if q else None, ldq=ldq if q else 0, scale=scale, stream=stream)
    torch.cuda.synchronize()
    for rows in (x, residual, total, out):
        assert rows is None or rows.clean()
    if not q:
        return out.rows if y else None, None
    body = ints[offset:offset + M * ldq].view(M, ldq)
    assert (body[:, K:] == GUARD).all() and (ints[:offset] == GUARD).all() and (ints[offset + M * ldq:] == GUARD).all()
    assert (scale[M:] == -5.0).all()
    return out.rows if y else None, (body[:, :K], scale[:M])


# a wavefront and a workgroup a row, one, four and eight chunks a thread, rows gone over again; ends inside of chunks
SHAPES = [(1, 1), (3, 5), (9, 8), (5, 77), (13, 512), (7, 513), (5, 2048), (1030, 2000), (1025, 2048), (8, 2049), (3, 8192), (9, 8193), (2, 16384), (3, 16391), (2, 20011),
          (2048, 2050), (2500, 4096), (1030, 4500), (1025, 8191)]   # (rows in turn)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm(M, K, dtype):
    _, t, _, _ = TYPES[dtype]
    g = torch.Generator().manual_seed(M + K)
    weight = (1 + 0.3 * torch.randn(K, generator=g)).to(DEV)
    for pad, offset, with_residual, with_weight in ((0, 0, True, True), (3, 1, True, False), (8, 0, False, True)):
        print(f"case norm {M}x{K} {dtype} pad={pad} residual={with_residual}", flush=True)
        x = Rows(hard_rows(M, K, t, seed=M + K).cpu(), pad, offset)
        r = Rows((4 * torch.randn(M, K, generator=g)).to(t), pad, offset) if with_residual else None
        w = weight if with_weight else None
        s = (x.rows.float() + r.rows.float()).to(t) if r else x.rows.clone()
        fine = torch.isfinite(s).all(1)   # (the sum may pass the type's range)
        total = Rows(torch.zeros(M, K, dtype=t), pad, offset) if r else None
        y, (ints, scale) = run(x, dtype, K, r, w, total=total, q=True, pad=pad, offset=offset)
        if r:
            assert torch.equal(bits(total.rows), bits(s))
        check(y[fine], s[fine], w, dtype)
        want, want_scale = run_quantize(y.contiguous(), K, K)
        assert torch.equal(ints, want) and torch.equal(scale.view(torch.int32), want_scale.view(torch.int32))
        # one result by itself, and the sum in an operand's place
        only_y, _ = run(x, dtype, K, r, w, pad=pad, offset=offset)
        assert torch.equal(bits(only_y), bits(y))
        if r:
            keep = x.rows.clone()
            _, (only_q, only_scale) = run(x, dtype, K, r, w, total=r, y=False, q=True, pad=pad, offset=offset)
            assert torch.equal(only_q, ints) and torch.equal(only_scale.view(torch.int32), scale.view(torch.int32))
            assert torch.equal(bits(r.rows), bits(s))
            r = Rows((s.float() * 0 + 1).nan_to_num(1.0).to(t), pad, offset)
            s = (keep.float() + r.rows.float()).to(t)
            y2, _ = run(x, dtype, K, r, w, total=x, pad=pad, offset=offset)
            fine = torch.isfinite(s).all(1)
            assert torch.equal(bits(x.rows), bits(s))
            check(y2[fine], s[fine], w, dtype)


@pytest.mark.parametrize("K", [40, 1000, 4096, 9000, 20000])
def test_rows_whose_squares_are_no_floats(K):
    g = torch.Generator().manual_seed(K)
    for size in (1e20, 1e30, 2e38):
        x = Rows((torch.rand(6, K, generator=g) * size).to(torch.bfloat16))
        y, (ints, scale) = run(x, "bf16", K, q=True)
        check(y, x.rows, None, "bf16")
        want, want_scale = run_quantize(y.contiguous(), K, K)
        assert torch.equal(ints, want) and torch.equal(scale, want_scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("K", [40, 1000, 4096, 9000, 20000])
def test_rows_of_zeros_and_rows_that_are_not_finite(K, dtype):
    """Zeros stay zeros with the scale 0; infinities and NaN give what the formula gives, and touch no other row."""
    _, t, _, _ = TYPES[dtype]
    x = torch.randn(7, K, generator=torch.Generator().manual_seed(K)).to(t)
    plain, _ = run(Rows(x), dtype, K)
    x[1] = 0
    x[3, K // 2], x[4, 0], x[5, K - 1] = float("inf"), float("nan"), -float("inf")
    y, (ints, scale) = run(Rows(x), dtype, K, q=True)
    assert (y[1] == 0).all() and (ints[1] == 0).all() and scale[1] == 0
    assert torch.isnan(y[4]).all()
    for m, k in ((3, K // 2), (5, K - 1)):
        nan = torch.isnan(y[m])
        assert nan[k] and int(nan.sum()) == 1 and (y[m][~nan] == 0).all()
    assert torch.isnan(scale[3:6]).all() and (ints[3:6] == 0).all()
    for m in (0, 2, 6):
        assert torch.equal(bits(y[m]), bits(plain[m]))


def test_eps_counts_where_rows_are_small():
    x = Rows(torch.full((4, 256), 2.0 ** -20, dtype=torch.bfloat16))
    for eps in (1e-30, 1e-12, 1.0, 1e30):
        y, _ = run(x, "bf16", 256, eps=eps)
        check(y, x.rows, None, "bf16", eps)


@pytest.mark.parametrize("M,K", [(3, 96), (5, 1000), (2, 8192), (2, 20000), (2048, 4096)])
def test_mean_and_eps_that_are_no_float_together(M, K):
    """The mean of squares and eps are floats, their sum is not; and eps beside a mean that is none counts."""
    g = torch.Generator().manual_seed(K)
    x = Rows(((torch.rand(M, K, generator=g) * 0.5 + 1.0) * 2.0 ** 63).to(torch.bfloat16))
    for eps in (3.4e38, 3e38, 1e38):
        y, _ = run(x, "bf16", K, eps=eps)
        check(y, x.rows, None, "bf16", eps)
    x = Rows(((torch.rand(M, K, generator=g) * 0.5 + 1.0) * 2.0 ** 65).to(torch.bfloat16))
    y, _ = run(x, "bf16", K, eps=3.4e38)
    check(y, x.rows, None, "bf16", 3.4e38)


def test_more_rows_than_a_launch_holds():
    """2^25 rows, four a workgroup."""
    M, K = (1 << 25) + 5, 3
    x = torch.zeros(M, K, dtype=torch.float16, device=DEV)
    places = [0, 1, (1 << 23) - 1, 1 << 23, (1 << 25) - 1, 1 << 25, M - 1]
    x[places] = torch.randn(len(places), K, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.float16)
    y = torch.full((M, K), 7.0, dtype=torch.float16, device=DEV)
    q = torch.full((M, K), GUARD, dtype=torch.int8, device=DEV)
    scale = torch.full((M,), -5.0, device=DEV)
    B.abft_rms_norm(M, K, x, K, B.F16, None, EPS, Y=y, ldy=K, Q=q, ldq=K, scale=scale)
    torch.cuda.synchronize()
    check(y[places], x[places], None, "f16")
    assert int((y != 0).any(1).sum()) == len(places) and int((q != 0).any(1).sum()) == len(places) and int((scale != 0).sum()) == len(places)


def test_two_streams_and_a_graph():
    """Calls at the same time, and recorded ones replayed on new rows, give what a call by itself gives."""
    M, K = 300, 4096
    g = torch.Generator().manual_seed(3)
    xs = [torch.randn(M, K, generator=g).to(torch.bfloat16).to(DEV) for _ in range(4)]
    w = (1 + 0.1 * torch.randn(K, generator=g)).to(DEV)

    def call(x, r, s, y, stream=None):
        B.abft_rms_norm(M, K, x, K, B.BF16, w, EPS, residual=r, ldr=K, total=s, ldt=K, Y=y, ldy=K, stream=stream)

    want = []
    for i in range(3):
        s, y = torch.empty_like(xs[0]), torch.empty_like(xs[0])
        call(xs[i], xs[3], s, y)
        want.append((s, y))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [(torch.zeros_like(xs[0]), torch.zeros_like(xs[0])) for _ in range(3)]
    torch.cuda.synchronize()
    for i, stream in enumerate(streams):
        call(xs[i], xs[3], *got[i], stream=stream)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(bits(p), bits(q)) for p, q in zip(a, b))
    x, s, y = xs[0].clone(), torch.empty_like(xs[0]), torch.empty_like(xs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(x, xs[3], s, y)
    for i in (0, 1, 2, 1):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(s), bits(want[i][0])) and torch.equal(bits(y), bits(want[i][1]))
