"""The paged cache: what is written to it and read back, against the definition in 64 bits.

Integers and scales have to be equal (see quantize.h), other slots untouched.  Reading back multiplies an integer of at most
seven bits and a float (one rounding, 2^-24) and rounds to the output type."""
import numpy as np
import pytest
import torch

from paper_2104_09455_amd import binding as B
from test_gpu_linear_scaled import DEV, TYPES, hard_rows, quantised

pytestmark = pytest.mark.gpu


def make_cache(pages, heads, page, dim, kind, t):
    """A cache filled with marks."""
    k = torch.full((pages, heads, page, dim), 77, dtype=torch.int8 if kind == "i8" else t, device=DEV)
    v = k.clone()
    ks = torch.full((pages, heads, page), -3.0, device=DEV) if kind == "i8" else None
    vs = ks.clone() if kind == "i8" else None
    dt = {"i8": B.I8, torch.float16: B.F16, torch.bfloat16: B.BF16}[kind if kind == "i8" else t]
    return k, v, ks, vs, B.kv_cache(k, v, ks, vs, dt, pages, page, heads, dim)


@pytest.mark.parametrize("kind", ["i8", "same"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,heads,dim,page,offset", [(1, 1, 16, 16, 0), (1, 8, 128, 16, 0), (7, 3, 48, 48, 1), (33, 5, 64, 32, 0), (70, 2, 112, 256, 3),
                                                          (257, 4, 80, 16, 0), (1000, 8, 128, 64, 0)])
def test_written_and_read_back(tokens, heads, dim, page, offset, dtype, kind):
    dt, t, u, tiny = TYPES[dtype]
    print(f"case cache tokens={tokens} heads={heads} dim={dim} page={page} {dtype} {kind}", flush=True)
    g = torch.Generator().manual_seed(tokens)
    pages = -(-tokens // page) + 2
    n = heads * dim
    rows = hard_rows(2 * tokens * heads, dim, t, seed=tokens).view(tokens, 2 * n)
    wide = torch.zeros(tokens * (2 * n + 6) + offset, dtype=t, device=DEV)   # columns of a larger product, rows at any address
    new = wide[offset:].view(tokens, 2 * n + 6)
    new[:, 3:3 + 2 * n] = rows
    K, V = new[:, 3:3 + n], new[:, 3 + n:3 + 2 * n]
    slots = torch.randperm(pages * page, generator=g)[:tokens].to(DEV)
    passed = tokens // 3
    if passed:   # tokens without a place
        slots[:passed] = torch.tensor([-1, pages * page, 2 ** 40], device=DEV)[torch.arange(passed) % 3]
    k, v, ks, vs, cache = make_cache(pages, heads, page, dim, kind, t)
    B.abft_kv_write(cache, tokens, slots, K, new.stride(0), V, new.stride(0), dt)
    torch.cuda.synchronize()
    back_k = torch.full((tokens, n + 5), 9.0, dtype=t, device=DEV)
    back_v = torch.full((tokens, n + 5), 9.0, dtype=t, device=DEV)
    B.abft_kv_read(cache, tokens, slots, back_k, n + 5, back_v, n + 5, dt)
    torch.cuda.synchronize()
    at, off = slots[passed:] // page, slots[passed:] % page
    for given, stored, scales, back in ((K, k, ks, back_k), (V, v, vs, back_v)):
        x = given[passed:].reshape(-1, heads, dim)
        got = stored[at, :, off]
        if kind == "i8":
            q, s = quantised(x.reshape(-1, dim))
            assert torch.equal(got.reshape(-1, dim).double(), q)
            assert torch.equal(scales[at, :, off].reshape(-1), s)
            want = (q * s.double()[:, None]).view_as(x)
            err = (back[passed:, :n].reshape_as(x).double() - want).abs()
            assert (err <= (u + 2.0 ** -22) * want.abs() + tiny).all()
            scales[at, :, off] = -3.0
            assert (scales == -3.0).all()
        else:
            assert torch.equal(got.view(torch.int16), x.contiguous().view(torch.int16))
            assert torch.equal(back[passed:, :n].reshape_as(x).view(torch.int16), x.contiguous().view(torch.int16))
        stored[at, :, off] = 77
        assert (stored == 77).all()          # no other slot was written
        assert (back[:passed, :n] == 0).all() and (back[:, n:] == 9.0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_values_that_are_not_finite(dtype):
    """A key with an infinity or a NaN reads back as NaN, and its neighbours as ever; a 16-bit cache keeps it."""
    dt, t, _, _ = TYPES[dtype]
    x = hard_rows(12, 64, t, seed=3).view(4, 192)
    x[1, 70], x[2, 5] = float("nan"), float("inf")
    slots = torch.tensor([3, 17, 0, 31], device=DEV)
    for kind in ("i8", "same"):
        k, v, ks, vs, cache = make_cache(2, 3, 16, 64, kind, t)
        B.abft_kv_write(cache, 4, slots, x, 192, x, 192, dt)
        a, b = torch.empty_like(x), torch.empty_like(x)
        B.abft_kv_read(cache, 4, slots, a, 192, b, 192, dt)
        torch.cuda.synchronize()
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        if kind == "same":
            assert torch.equal(a.view(torch.int16), x.view(torch.int16))
        else:
            bad = torch.isnan(a).view(4, 3, 64).all(-1)
            assert torch.equal(bad, torch.tensor([[False] * 3, [False, True, False], [True, False, False], [False] * 3], device=DEV))
            assert torch.isfinite(a.view(4, 3, 64)[~bad]).all()


def test_no_tokens():
    _, _, _, _, cache = make_cache(1, 1, 16, 16, "i8", torch.float16)
    B.abft_kv_write(cache, 0, None, None, 16, None, 16, B.F16)
    B.abft_kv_read(cache, 0, None, None, 16, None, 16, B.F16)


def test_more_tokens_than_a_launch_holds():
    """2^24 tokens of 64 heads, most of them nowhere in the cache: more than 2^32 threads.  (Keys and values share their memory.)"""
    tokens, heads, dim, page = (1 << 24) + 3, 64, 16, 16
    row = heads * dim
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 40 GB")
    x = torch.zeros(tokens, row, dtype=torch.bfloat16, device=DEV)
    places = torch.tensor([0, (1 << 23) - 1, 1 << 23, tokens - 4, tokens - 1], device=DEV)
    x[places] = torch.randn(5, row, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.bfloat16)
    kept = x[places].clone()
    k = torch.full((1, heads, page, dim), 3.0, dtype=torch.bfloat16, device=DEV)
    cache = B.kv_cache(k, k, None, None, B.BF16, 1, page, heads, dim)
    slots = torch.full((tokens,), -1, dtype=torch.int64, device=DEV)
    at = torch.tensor([9, 2, 15, 4, 0], device=DEV)
    slots[places] = at
    B.abft_kv_write(cache, tokens, slots, x, row, x, row, B.BF16)
    torch.cuda.synchronize()
    stored = k[0].transpose(0, 1).reshape(page, row)
    assert torch.equal(stored[at], kept)
    assert int((stored != 3.0).any(1).sum()) == 5
    x.fill_(7.0)
    B.abft_kv_read(cache, tokens, slots, x, row, x, row, B.BF16)
    torch.cuda.synchronize()
    assert torch.equal(x[places], kept)
    assert int(x[:, ::dim].ne(0).any(1).sum()) == 5
