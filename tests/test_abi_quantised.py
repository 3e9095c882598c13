"""CPU-only checks of what the quantised entry points refuse.  Every call here ends before anything is launched: the pointers
are numbers that are never followed."""
import ctypes
import os

import pytest

from paper_2104_09455_amd import binding as B

P = 1 << 20            # stands for an aligned device address
E_NULL, E_SHAPE, E_LD, E_ENUM, E_WORKSPACE, E_INJECT, E_UNSUPPORTED, E_VALUE = -1, -2, -3, -4, -5, -6, -9, -10


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2104_09455_amd.build import build
        build()
    return B.lib()


def refuses(code, call):
    with pytest.raises(B.AbftError) as e:
        call()
    assert e.value.code == code
    assert "unknown error code" not in str(e.value)


def test_every_error_has_a_text():
    for code in range(-10, 0):
        assert "unknown error code" not in B.abft_strerror(code)


@pytest.mark.parametrize("change,code", [
    (dict(M=0), E_SHAPE), (dict(K=-1), E_SHAPE), (dict(X=None), E_NULL), (dict(Q=None), E_NULL), (dict(scale=None), E_NULL), (dict(ldx=63), E_LD),
    (dict(ldq=63), E_LD), (dict(dtype=B.I8), E_ENUM), (dict(dtype=9), E_ENUM)])
def test_quantize_rows(change, code):
    a = dict(M=4, K=64, X=P, ldx=64, dtype=B.F16, Q=P, ldq=64, scale=P)
    a.update(change)
    refuses(code, lambda: B.abft_quantize_rows(stream=0, **a))


COMMON = [
    (dict(M=0), E_SHAPE), (dict(N=0), E_SHAPE), (dict(K=0), E_SHAPE), (dict(K=131072, ldb=131072), E_SHAPE), (dict(B=None), E_NULL), (dict(C=None), E_NULL),
    (dict(col_scale=None), E_NULL), (dict(ldb=63), E_LD), (dict(ldc=31), E_LD), (dict(b_layout=2), E_ENUM), (dict(act=2), E_ENUM), (dict(mode=8), E_ENUM),
    (dict(mode=B.REPLICA), E_UNSUPPORTED), (dict(mode=B.THREAD_HALF), E_UNSUPPORTED), (dict(mode=B.TWOSIDED), E_UNSUPPORTED),
    (dict(mode=B.GLOBAL_WEIGHTED), E_UNSUPPORTED), (dict(fault_flag=None), E_NULL), (dict(mode=B.GLOBAL, workspace=None), E_WORKSPACE),
    (dict(mode=B.GLOBAL, workspace=P + 8), E_WORKSPACE), (dict(inject=B.Fault(4, 0, 0, -1)), E_INJECT), (dict(inject=B.Fault(0, 32, 0, -1)), E_INJECT),
    (dict(inject=B.Fault(0, 0, 32, -1)), E_INJECT), (dict(inject=B.Fault(0, 0, 1, 5)), E_INJECT)]


@pytest.mark.parametrize("change,code", COMMON + [(dict(A=None), E_NULL), (dict(row_scale=None), E_NULL), (dict(lda=63), E_LD), (dict(out_dtype=B.I8), E_ENUM),
                                                  (dict(K=131072, lda=131072, ldb=131072), E_SHAPE), (dict(mode=B.GLOBAL, workspace_bytes=255), E_WORKSPACE)])
def test_gemm_scaled(change, code):
    a = dict(M=4, N=32, K=64, A=P, lda=64, row_scale=P, B=P, ldb=64, b_layout=B.B_NK, col_scale=P, bias=None, act=0, C=P, ldc=32, out_dtype=B.BF16,
             mode=B.THREAD, workspace=P, workspace_bytes=1 << 30, fault_flag=P)
    a.update(change)
    refuses(code, lambda: B.abft_gemm_scaled(stream=0, **a))


@pytest.mark.parametrize("change,code", COMMON + [(dict(X=None), E_NULL), (dict(ldx=63), E_LD), (dict(dtype=B.I8), E_ENUM), (dict(workspace=None), E_WORKSPACE),
                                                  (dict(workspace_bytes=255), E_WORKSPACE), (dict(K=131072, ldx=131072, ldb=131072), E_SHAPE)])
def test_linear_scaled(change, code):
    if change.get("K") == 131072 and "ldx" not in change:
        change = dict(change, ldx=131072)
    a = dict(M=4, N=32, K=64, X=P, ldx=64, dtype=B.F16, B=P, ldb=64, b_layout=B.B_NK, col_scale=P, bias=None, act=0, C=P, ldc=32,
             mode=B.THREAD, workspace=P, workspace_bytes=1 << 30, fault_flag=P)
    a.update(change)
    refuses(code, lambda: B.abft_linear_scaled(stream=0, **a))


def test_linear_workspace():
    """Room for the quantised rows and their scales, and what the product wants beside."""
    for M, N, K in ((1, 8, 8), (33, 100, 1001), (512, 4096, 4096)):
        small = B.abft_linear_scaled_workspace_bytes(M, N, K, B.THREAD)
        assert small >= M * K + 4 * M
        assert B.abft_linear_scaled_workspace_bytes(M, N, K, B.GLOBAL) == small + B.abft_workspace_bytes(M, N, K, B.I8, B.GLOBAL)
    assert B.abft_linear_scaled_workspace_bytes(0, 8, 8, B.NONE) == 0


def test_scheme_of_scaled_products():
    """Aligned: the tiles of 32 x 32 against the compute units; else the rule of plain products."""
    assert B.abft_scaled_select(64, 4096, 4096) == B.THREAD
    assert B.abft_scaled_select(65, 4096, 4096) == B.GLOBAL
    assert B.abft_scaled_select(8192, 32, 64) == B.THREAD
    for M, N, K in ((500, 1000, 2047), (8192, 8192, 8191)):
        assert B.abft_scaled_select(M, N, K, aligned=False) == B.abft_select(M, N, K, B.I8)
    refuses(E_SHAPE, lambda: B.abft_scaled_select(0, 1, 1))


CACHE = dict(k=P, v=P, k_scale=P, v_scale=P, dtype=B.I8, pages=4, page_size=16, heads=2, head_dim=64)
BAD_CACHES = [(dict(k=None), E_NULL), (dict(v=None), E_NULL), (dict(k_scale=None), E_NULL), (dict(v_scale=None), E_NULL), (dict(k=P + 8), E_LD), (dict(v_scale=P + 4), E_LD),
              (dict(dtype=B.BF16), E_ENUM), (dict(dtype=5), E_ENUM), (dict(pages=0), E_SHAPE), (dict(heads=0), E_SHAPE), (dict(head_dim=24), E_SHAPE),
              (dict(head_dim=0), E_SHAPE), (dict(head_dim=144), E_SHAPE), (dict(page_size=0), E_VALUE), (dict(page_size=24), E_VALUE),
              (dict(page_size=8192), E_VALUE), (dict(pages=1 << 27), E_SHAPE)]


@pytest.mark.parametrize("move", ["write", "read"])
@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_bad_caches(change, code, move):
    cache = B.kv_cache(**dict(CACHE, **change))
    call = B.abft_kv_write if move == "write" else B.abft_kv_read
    refuses(code, lambda: call(cache, 3, P, P, 128, P, 128, B.F16, stream=0))


@pytest.mark.parametrize("move", ["write", "read"])
@pytest.mark.parametrize("change,code", [(dict(tokens=-1), E_SHAPE), (dict(slots=None), E_NULL), (dict(K=None), E_NULL), (dict(V=None), E_NULL), (dict(ldk=127), E_LD),
                                         (dict(ldv=127), E_LD), (dict(dtype=B.I8), E_ENUM)])
def test_bad_tokens(change, code, move):
    a = dict(tokens=3, slots=P, K=P, ldk=128, V=P, ldv=128, dtype=B.F16)
    a.update(change)
    call = B.abft_kv_write if move == "write" else B.abft_kv_read
    refuses(code, lambda: call(B.kv_cache(**CACHE), stream=0, **a))


def test_no_cache():
    assert B.lib().abft_kv_write(None, 1, P, P, 128, P, 128, B.F16, None) == E_NULL
    assert B.lib().abft_kv_read(ctypes.POINTER(B.KVCache)(), 1, P, P, 128, P, 128, B.F16, None) == E_NULL


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_attention_over_bad_caches(change, code):
    cache = B.kv_cache(**dict(CACHE, **change))
    refuses(code, lambda: B.abft_attention(cache, 2, P, P, P, 4, 5, 4, 60, P, 128, 2, B.F16, 0.1, True, 0, P, 128, workspace=P, workspace_bytes=1 << 40, stream=0))
    assert B.abft_attention_workspace_bytes(cache, 2, 5, 4, 60, 2, B.F16) == 0


@pytest.mark.parametrize("change,code", [
    (dict(n_seqs=0), E_SHAPE), (dict(total_q=-1), E_SHAPE), (dict(max_q=6), E_SHAPE), (dict(max_q=-1), E_SHAPE), (dict(max_kv=-1), E_SHAPE),
    (dict(max_kv=(1 << 24) + 1), E_SHAPE), (dict(q_heads=0), E_SHAPE), (dict(q_heads=3), E_SHAPE), (dict(q_start=None), E_NULL), (dict(kv_len=None), E_NULL),
    (dict(block_table=None), E_NULL), (dict(Q=None), E_NULL), (dict(O=None), E_NULL), (dict(dtype=B.I8), E_ENUM), (dict(scale=0.0), E_VALUE),
    (dict(scale=float("nan")), E_VALUE), (dict(scale=float("inf")), E_VALUE), (dict(scale=-1.0), E_VALUE), (dict(window=-1), E_VALUE), (dict(ldq=255), E_LD),
    (dict(ldo=255), E_LD), (dict(ldq=260), E_LD), (dict(ldo=258), E_LD), (dict(Q=P + 8), E_LD), (dict(O=P + 4), E_LD), (dict(ld_table=312), E_LD),
    (dict(workspace=None), E_WORKSPACE), (dict(workspace=P + 64), E_WORKSPACE), (dict(workspace_bytes=100), E_WORKSPACE)])
def test_attention(change, code):
    a = dict(n_seqs=2, q_start=P, kv_len=P, block_table=P, ld_table=313, total_q=5, max_q=4, max_kv=5000, Q=P, ldq=256, q_heads=4, dtype=B.BF16, scale=0.1, causal=True,
             window=0, O=P, ldo=256, workspace=P, workspace_bytes=1 << 40)
    a.update(change)
    refuses(code, lambda: B.abft_attention(B.kv_cache(**CACHE), stream=0, **a))


@pytest.mark.parametrize("change,code", [
    (dict(), E_WORKSPACE), (dict(n_seqs=1 << 17), E_SHAPE), (dict(n_seqs=1, total_q=(1 << 24) + 1, max_q=1 << 24), E_SHAPE),
    (dict(n_seqs=1 << 20, q_heads=1 << 30, total_q=1, max_q=1), E_SHAPE), (dict(n_seqs=(1 << 31) - 1, q_heads=(1 << 31) - 128, total_q=1, max_q=1, max_kv=1 << 24), E_SHAPE),
    (dict(n_seqs=1 << 17, total_q=1 << 17, max_q=1), E_WORKSPACE)])
def test_attention_larger_than_a_launch(change, code):
    """2^24 workgroups of row tiles and more are refused (the first and the last are just smaller, and end at the missing workspace)."""
    a = dict(n_seqs=(1 << 17) - 2100, q_start=P, kv_len=P, block_table=P, ld_table=8, total_q=(1 << 18) - 1, max_q=2, max_kv=100, Q=P, ldq=1 << 40, q_heads=128, dtype=B.BF16,
             scale=0.1, causal=True, window=0, O=P, ldo=1 << 40, workspace=None, workspace_bytes=0)
    a.update(change)
    cache = B.kv_cache(**dict(CACHE, heads=128, head_dim=16))
    refuses(code, lambda: B.abft_attention(cache, stream=0, **a))
    if code == E_SHAPE:
        assert B.abft_attention_workspace_bytes(cache, a["n_seqs"], a["total_q"], a["max_q"], a["max_kv"], a["q_heads"], a["dtype"]) == 0


def test_room_for_pieces_beside_many_single_tokens():
    """127 single tokens and a chunk of 512 over 32768 keys: its 16 row tiles of 8 heads have room for two pieces each at least, since single tokens
    are no row tiles; 8 prompts of 4096, whose row tiles fill the chip, have none."""
    cache = B.kv_cache(**dict(CACHE, heads=8, head_dim=128))
    piece = 128 * 128 * 4
    assert B.abft_attention_workspace_bytes(cache, 128, 639, 512, 32768, 32, B.F16) >= 2 * 16 * 8 * piece
    assert B.abft_attention_workspace_bytes(cache, 8, 8 * 4096, 4096, 4096, 32, B.F16) == 0


def test_stream_without_the_raw_handle(monkeypatch):
    """A torch that does not give the current stream's handle by itself: it is taken from the stream."""
    import types

    import torch
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=4660))
    assert B._stream(None) == 4660
    assert B._stream(7) == 7 and B._stream(0) is None
