"""The compiled marshalling of the norm, the residual's and the gated products: what it hands on, and what it refuses before the
library is called.  No kernel is launched here (shapes are empty or refused)."""
import ctypes
import subprocess
import sys

import pytest
import torch

from paper_2104_09455_amd import binding as B

X = torch.zeros(16, 16)


def norm(**kw):
    a = dict(M=0, K=16, X=X, ldx=16, dtype=B.F16, weight=X, eps=1e-5, Y=X, ldy=16, stream=0)
    a.update(kw)
    B.abft_rms_norm(**a)


def linear_add(**kw):
    a = dict(M=0, N=16, K=16, X=X, ldx=16, dtype=B.F16, B=X, ldb=16, b_layout=B.B_NK, col_scale=X, bias=None, act=B.ACT_NONE, R=X, ldr=16,
             C=X, ldc=16, mode=B.NONE, workspace=X, workspace_bytes=1024, fault_flag=X, stream=0)
    a.update(kw)
    B.abft_linear_scaled_add(**a)


def test_every_entry_point_gets_each_argument_in_its_place(monkeypatch):
    """The five functions are bound to a callback of the C signature that notes what arrived; the arguments are all different."""
    i, q, p = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
    signatures = {
        "gemm_scaled_add": [i, i, i, p, q, p, p, q, i, p, p, i, p, q, p, q, i, i, p, p, ctypes.c_size_t, p, p, p, p],
        "linear_scaled_add": [i, i, i, p, q, i, p, q, i, p, p, i, p, q, p, q, i, p, p, ctypes.c_size_t, p, p, p, p],
        "gemm_gated": [i, i, i, p, q, p, p, q, i, p, p, i, p, q, i, i, p, p, ctypes.c_size_t, p, p, p, p],
        "linear_gated": [i, i, i, p, q, i, p, q, i, p, p, i, p, q, i, p, p, ctypes.c_size_t, p, p, p, p],
        "rms_norm": [i, i, p, q, i, p, ctypes.c_float, p, q, p, q, p, q, p, q, p, p],
    }
    m = B._compiled()
    got = []
    callbacks = [ctypes.CFUNCTYPE(i, *t)(lambda *a: got.append(a) or 7) for t in signatures.values()]
    L = B.lib()
    try:
        m.bind(*(ctypes.cast(c, p).value for c in callbacks))
        for name, types in signatures.items():
            fault = B.Fault()
            args, want = [], []
            for k, t in enumerate(types):
                if t is p and k == len(types) - 2 and name != "rms_norm":   # the fault descriptor, by its address
                    args.append(fault), want.append(ctypes.addressof(fault))
                elif t is p:
                    args.append(X[k % 16, k // 16:] if k % 3 else 10 ** 12 + k)
                    want.append(args[-1].data_ptr() if k % 3 else args[-1])
                elif t is i:
                    args.append(-5 - k), want.append(-5 - k)
                elif t is ctypes.c_float:
                    args.append(0.5), want.append(0.5)
                else:
                    args.append(2 ** 40 + k), want.append(2 ** 40 + k)
            assert getattr(m, name)(*args) == 7
            assert list(got.pop()) == want, name
            args = [None if t is p else v for t, v in zip(types, args)]
            getattr(m, name)(*args)
            assert [v for v, t in zip(got.pop(), types) if t is p] == [None] * types.count(p), name
    finally:
        m.bind(*(ctypes.cast(f, p).value for f in (L.abft_gemm_scaled_add, L.abft_linear_scaled_add, L.abft_gemm_gated, L.abft_linear_gated,
                                                   L.abft_rms_norm)))


@pytest.mark.parametrize("bad, error", [(dict(M=2 ** 31), OverflowError), (dict(K=-2 ** 31 - 1), OverflowError), (dict(ldx=2 ** 63), OverflowError),
                                        (dict(M=1.0), TypeError), (dict(eps="1"), TypeError), (dict(X=1.5), AttributeError),
                                        (dict(X=2 ** 64), OverflowError), (dict(M="1", X=1.5, eps="1"), TypeError)])
def test_values_that_are_no_argument_are_refused(bad, error):
    with pytest.raises(error):
        norm(**bad)


def test_the_librarys_refusals_come_back():
    with pytest.raises(B.AbftError) as e:
        norm(M=-1)
    assert e.value.code == -2   # a bad problem shape
    with pytest.raises(B.AbftError):
        linear_add(K=-1, inject=B.Fault())


@pytest.mark.parametrize("inject", [3, b"abc", "x", X])
def test_a_fault_descriptor_is_the_structure(inject):
    with pytest.raises((TypeError, BufferError)):
        linear_add(inject=inject)


def test_a_wrong_number_of_arguments_and_a_call_before_bind():
    m = B._compiled()
    for f in (m.gemm_scaled_add, m.linear_scaled_add, m.gemm_gated, m.linear_gated, m.rms_norm, m.bind):
        with pytest.raises(TypeError):
            f()
        with pytest.raises(TypeError):
            f(*[0] * 30)
    code = "from paper_2104_09455_amd import _marshal as m\ntry:\n    m.rms_norm(*[0] * 17)\nexcept RuntimeError:\n    print('refused')\n"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert r.stdout.strip() == "refused", r.stderr
