"""The example decoder: every call of a prompt and of the steps behind it against its definition in 64 bits, from the
inputs that the call had, and the recorded step against the calls.

(Not the whole network against one in 64 bits: a rounding to 16 bits that moves a value over an integer's border moves it by a whole
step, and from layer to layer such steps add up to the quantisation's own noise, in which a mistake would not show.)"""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

_spec = importlib.util.spec_from_file_location("int8_decoder", os.path.join(os.path.dirname(__file__), "..", "examples", "int8_decoder.py"))


@pytest.fixture(scope="module")
def example():
    module = importlib.util.module_from_spec(_spec)
    _spec.loader.exec_module(module)
    return module


def quantised(x):
    """(integers, scales) of groups along the last axis, the integers rounded to nearest."""
    top = x.abs().amax(-1, keepdim=True)
    y = torch.where(top > 0, x * 127 / torch.where(top > 0, top, torch.ones_like(top)), torch.zeros_like(x))
    return torch.sign(y) * torch.floor(y.abs() + 0.5), top / 127


def check_linear(layer, x, out):
    """The integers' sums are exact; scales and the one rounding to 16 bits (test_gpu_linear_scaled.py) are not."""
    u, tiny = {torch.float16: (2.0 ** -11, 2.0 ** -24), torch.bfloat16: (2.0 ** -8, 2.0 ** -133)}[out.dtype]
    q, scale = quantised(x.double())
    want = (q @ layer.w.double().t().contiguous()) * scale * layer.w_scale.double()   # (a sum of zero is zero)
    if layer.act:
        want = want.clamp(min=0)
    assert ((out.double() - want).abs() <= (u + 2.0 ** -21) * want.abs() + tiny).all()


def check_attention(model, store, table, lengths, before, qkv, out):
    """Every sequence's slots hold its keys and values by the rule, and its rows are within the bounds of test_gpu_attention.py."""
    heads, group, dim, at = model.heads, model.group, model.dim, 0
    u = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[out.dtype]
    for i, (n, b) in enumerate(zip(lengths, before)):
        q, new_k, new_v = qkv[at:at + n].split([model.width, heads * dim, heads * dim], -1)
        t = torch.arange(b + n, device=qkv.device)
        page, off = table[i][t // model.page].long(), t % model.page
        k, v = (store[j][page, :, off].double() * store[j + 2][page, :, off].double()[..., None] for j in range(2))
        for have, new in ((k, new_k), (v, new_v)):
            integers, scale = quantised(new.reshape(n, heads, dim).double())
            new = integers * scale
            assert ((have[b:] - new).abs() <= 2.0 ** -22 * new.abs()).all()   # (the scale is a float)
        hidden = torch.arange(b + n, device=qkv.device)[None] > b + torch.arange(n, device=qkv.device)[:, None]
        for h in range(heads * group):
            kh, vh, qh = k[:, h // group], v[:, h // group], q[:, h * dim:(h + 1) * dim].double()
            p = torch.softmax((qh @ kh.t().contiguous() / math.sqrt(dim)).masked_fill(hidden, -math.inf), -1)
            want, size = p @ vh, p @ vh.abs()
            arg = (qh.abs() @ kh.abs().t().contiguous() / math.sqrt(dim)).masked_fill(hidden, 0).amax(-1, keepdim=True)
            e = 2.0 ** -24 * (dim + (b + n) / 16 + 64) * (1 + arg)
            small = 2.0 ** -25 * p.amax(-1, keepdim=True) * vh.abs().sum(0) + 2.0 ** -24
            got = out[at:at + n, h * dim:(h + 1) * dim].double()
            assert ((got - want).abs() <= (u + 2 * e) * size + u * want.abs() + small).all(), (i, h)
        at += n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("lengths", [[1], [7, 1, 130, 33]], ids=["one", "four"])
def test_prompt_and_steps(example, dtype, lengths):
    steps, n = 5, len(lengths)
    model = example.Decoder(heads=2, group=2, dim=64, vocab=512, seqs=n, max_kv=max(lengths) + steps + 1, dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randint(0, 512, (sum(lengths),), device="cuda", generator=gen)
    linear, attention, calls = model.linear, model.attention, []

    def checked_linear(layer, x, batch):
        out = linear(layer, x, batch)
        check_linear(layer, x, out)
        calls.append("linear")
        return out

    def checked_attention(cache, qkv, batch):
        out = attention(cache, qkv, batch)
        new = batch.new.tolist()
        before = [int(m) - c for m, c in zip(batch.kv_len.tolist(), new)]
        check_attention(model, model.stores[model.caches.index(cache)], model.table, new, before, qkv, out)
        calls.append("attention")
        return out

    def checked_run(tokens, batch):
        model.linear, model.attention = checked_linear, checked_attention
        try:
            return model.run(tokens, batch)
        finally:
            model.linear, model.attention = linear, attention

    batch = example.Batch(model, lengths)
    batch.place(model, torch.zeros(n, dtype=torch.int64, device="cuda"))
    logits = checked_run(prompt, batch)
    answer = example.Answer(model, logits[batch.q_start[1:].long() - 1].argmax(-1), batch.kv_len.long())
    eager = example.Batch(model, [1] * n)
    for step in range(steps):
        tokens, length = answer.tokens.clone(), answer.length.clone()
        assert length.tolist() == [m + step for m in lengths]
        answer.graph.replay()
        eager.place(model, length)
        again = checked_run(tokens, eager)   # (writes the same keys and values to the same slots)
        assert torch.equal(answer.logits, again) and torch.equal(answer.tokens, again.argmax(-1))
    assert int(model.flag.item()) == 0
    assert calls.count("attention") == 2 * (1 + steps) and calls.count("linear") == 9 * (1 + steps)


def test_command(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["int8_decoder.py", "--seqs", "3", "--steps", "4", "--width", "512"])
    example.main()
    assert "faults seen: 0" in capsys.readouterr().out
