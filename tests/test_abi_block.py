"""CPU-only checks of what the norm, the residual's and the gated products refuse.  Every call here ends before anything is launched:
the pointers are numbers that are never followed."""
import pytest

from paper_2104_09455_amd import binding as B
from test_abi_quantised import COMMON, E_ENUM, E_LD, E_NULL, E_SHAPE, E_VALUE, E_WORKSPACE, P, _lib, refuses  # noqa: F401

# (activation functions: any of the five here)
COMMON = [(c, code) for c, code in COMMON if "act" not in c] + [(dict(act=5), E_ENUM), (dict(act=-1), E_ENUM)]
GEMM = [(dict(A=None), E_NULL), (dict(row_scale=None), E_NULL), (dict(lda=63), E_LD), (dict(out_dtype=B.I8), E_ENUM),
        (dict(K=131072, lda=131072, ldb=131072), E_SHAPE), (dict(mode=B.GLOBAL, workspace_bytes=255), E_WORKSPACE)]
LINEAR = [(dict(X=None), E_NULL), (dict(ldx=63), E_LD), (dict(dtype=B.I8), E_ENUM), (dict(workspace=None), E_WORKSPACE), (dict(workspace_bytes=255), E_WORKSPACE)]
ADD = [(dict(R=None), E_NULL), (dict(ldr=31), E_LD)]


def arguments(linear, change):
    a = dict(M=4, N=32, K=64, B=P, ldb=64, b_layout=B.B_NK, col_scale=P, bias=None, act=0, C=P, ldc=32, mode=B.THREAD, workspace=P,
             workspace_bytes=1 << 30, fault_flag=P)
    a.update(dict(X=P, ldx=64, dtype=B.F16) if linear else dict(A=P, lda=64, row_scale=P, out_dtype=B.BF16))
    if linear and change.get("K") == 131072:
        a["ldx"] = 131072
    if change.get("K") == 131072 and not linear:
        a["lda"] = 131072
    a.update(change)
    return a


@pytest.mark.parametrize("change,code", COMMON + GEMM + ADD)
def test_gemm_scaled_add(change, code):
    refuses(code, lambda: B.abft_gemm_scaled_add(stream=0, **{**dict(R=P, ldr=32), **arguments(False, change)}))


@pytest.mark.parametrize("change,code", COMMON + LINEAR + ADD)
def test_linear_scaled_add(change, code):
    refuses(code, lambda: B.abft_linear_scaled_add(stream=0, **{**dict(R=P, ldr=32), **arguments(True, change)}))


# (64 columns of weights for 32 of C: a fault may be in any of them)
GATED = [(c, code) for c, code in COMMON if "inject" not in c or c["inject"].col != 32] + [
    (dict(inject=B.Fault(0, 64, 0, -1)), -6), (dict(N=1 << 30), E_SHAPE), (dict(N=-1), E_SHAPE), (dict(b_layout=B.B_KN, ldb=63), E_LD)]


@pytest.mark.parametrize("change,code", GATED + GEMM)
def test_gemm_gated(change, code):
    refuses(code, lambda: B.abft_gemm_gated(stream=0, **arguments(False, change)))


@pytest.mark.parametrize("change,code", GATED + LINEAR)
def test_linear_gated(change, code):
    refuses(code, lambda: B.abft_linear_gated(stream=0, **arguments(True, change)))


def test_gated_workspace_is_that_of_twice_the_columns():
    M, N, K = 100, 600, 512
    need = B.abft_linear_scaled_workspace_bytes(M, 2 * N, K, B.GLOBAL)
    a = arguments(True, dict(M=M, N=N, K=K, ldx=K, ldb=K, ldc=N, mode=B.GLOBAL))
    refuses(E_WORKSPACE, lambda: B.abft_linear_gated(stream=0, **dict(a, workspace_bytes=need - 1)))


@pytest.mark.parametrize("change,code", [
    (dict(M=0), E_SHAPE), (dict(K=0), E_SHAPE), (dict(M=-3), E_SHAPE), (dict(X=None), E_NULL), (dict(ldx=63), E_LD), (dict(ldr=63), E_LD), (dict(ldt=63), E_LD),
    (dict(ldy=63), E_LD), (dict(ldq=63), E_LD), (dict(dtype=B.I8), E_ENUM), (dict(dtype=7), E_ENUM), (dict(residual=None), E_NULL),
    (dict(Y=None, Q=None, scale=None), E_NULL), (dict(scale=None), E_NULL), (dict(eps=0.0), E_VALUE), (dict(eps=-1.0), E_VALUE),
    (dict(eps=float("inf")), E_VALUE), (dict(eps=float("nan")), E_VALUE)])
def test_rms_norm(change, code):
    a = dict(M=4, K=64, X=P, ldx=64, dtype=B.F16, weight=P, eps=1e-5, residual=P, ldr=64, total=P, ldt=64, Y=P, ldy=64, Q=P, ldq=64, scale=P)
    a.update(change)
    refuses(code, lambda: B.abft_rms_norm(stream=0, **a))
