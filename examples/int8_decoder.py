"""A small int8 decoder that answers prompts: the library's quantised layers, paged cache and attention together.

    python examples/int8_decoder.py [--seqs 4] [--steps 32] [--layers 2] [--width 1024]

Weights are random, so the answers mean nothing; the calls are those of a serving program.  Every linear layer is int8 with
16-bit activations and runs under the protection scheme that the library picks for its size, with one sticky flag for all
of them.  Keys and values live in pages of an int8 cache.  The prompts of all sequences run as one batch; then every step takes one
token of each sequence.  A step is recorded once as a HIP graph and replayed: what changes from step to step (the
tokens, lengths and slots) is on the device.
"""
import argparse
import math
import os
import sys
import time

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2104_09455_amd import binding as B

DEV = "cuda:0"
KINDS = {torch.float16: B.F16, torch.bfloat16: B.BF16}


class Linear:
    """An int8 layer: weights (N x K) with a scale per channel, and the checksums that the global scheme wants of them."""

    def __init__(self, weight, relu=False):
        self.N, self.K = weight.shape
        self.w_scale = weight.abs().amax(1) / 127
        self.w = torch.round(weight / self.w_scale[:, None]).to(torch.int8)
        self.act = B.ACT_RELU if relu else B.ACT_NONE
        self.beta = {}   # by the width of a checksum's block, which follows the rows of a call

    def checksums(self, rows):
        width = B.abft_region_shape(rows, self.N, self.K, B.I8, self.K % 16 == 0)[1]
        if width not in self.beta:
            self.beta[width] = torch.empty(B.abft_beta_bytes(self.K, self.N, width), device=DEV, dtype=torch.uint8)
            B.abft_weight_checksum(self.K, self.N, self.w, self.K, B.B_NK, B.I8, self.beta[width], width)
        return self.beta[width]


class Batch:
    """What one pass works on: `q_len` new tokens of each sequence, behind what the cache already holds of it."""

    def __init__(self, model, q_len):
        self.total, self.max_q, n = sum(q_len), max(q_len), len(q_len)
        at = [0]
        for count in q_len:
            at.append(at[-1] + count)
        self.q_start = torch.tensor(at, dtype=torch.int32, device=DEV)
        self.kv_len = torch.zeros(n, dtype=torch.int32, device=DEV)
        self.seq = torch.repeat_interleave(torch.arange(n, device=DEV), torch.tensor(q_len, device=DEV))
        self.index = torch.arange(self.total, device=DEV) - self.q_start[:-1].long()[self.seq]
        self.new = torch.tensor(q_len, device=DEV)
        self.slots = torch.zeros(self.total, dtype=torch.int64, device=DEV)
        # one workspace each, as large as the pass's largest call wants; attention's begins with zeros
        self.linear_ws = torch.empty(max(B.abft_linear_scaled_workspace_bytes(self.total, l.N, l.K, B.AUTO) for l in model.linears),
                                     device=DEV, dtype=torch.uint8)
        self.attention_ws = torch.zeros(B.abft_attention_workspace_bytes(model.caches[0], n, self.total, self.max_q, model.max_kv,
                                                                         model.heads * model.group, model.kind), device=DEV, dtype=torch.uint8)
        for l in model.linears:
            l.checksums(self.total)

    def place(self, model, before):
        """Lengths and slots of the tokens that follow `before` (a device tensor, one number for each sequence)."""
        at = before[self.seq] + self.index
        self.kv_len.copy_(before + self.new)
        self.slots.copy_(model.table[self.seq, at // model.page].long() * model.page + at % model.page)


class Decoder:
    def __init__(self, layers=2, heads=4, group=2, dim=128, vocab=2048, seqs=4, max_kv=1024, page=16, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.heads, self.group, self.dim, self.page, self.dtype, self.kind = heads, group, dim, page, dtype, KINDS[dtype]
        self.max_kv, self.width = max_kv, heads * group * dim

        def weight(n, k):
            return torch.randn(n, k, device=DEV, generator=gen) / math.sqrt(k)

        d, kv = self.width, heads * dim
        self.embedding = torch.randn(vocab, d, device=DEV, generator=gen).to(dtype)
        self.blocks = [{"qkv": Linear(weight(d + 2 * kv, d)), "out": Linear(weight(d, d)), "up": Linear(weight(4 * d, d), relu=True),
                        "down": Linear(weight(d, 4 * d))} for _ in range(layers)]
        self.head = Linear(weight(vocab, d))
        self.linears = [l for block in self.blocks for l in block.values()] + [self.head]
        # the cache: pages of every sequence wherever they are free
        need = -(-max_kv // page)
        self.pages = seqs * need
        self.table = torch.randperm(self.pages, device=DEV, generator=gen).to(torch.int32).reshape(seqs, need)
        self.stores, self.caches = [], []
        for _ in range(layers):
            store = [torch.zeros(self.pages, heads, page, dim, device=DEV, dtype=torch.int8) for _ in range(2)]
            store += [torch.zeros(self.pages, heads, page, device=DEV) for _ in range(2)]
            self.stores.append(store)
            self.caches.append(B.kv_cache(*store, B.I8, self.pages, page, heads, dim))
        self.flag = torch.zeros(1, dtype=torch.int32, device=DEV)   # set by any layer whose check fails

    def linear(self, layer, x, batch):
        out = torch.empty(x.shape[0], layer.N, device=DEV, dtype=self.dtype)
        B.abft_linear_scaled(x.shape[0], layer.N, layer.K, x, x.stride(0), self.kind, layer.w, layer.K, B.B_NK, layer.w_scale, None,
                             layer.act, out, layer.N, B.AUTO, beta=layer.checksums(x.shape[0]), workspace=batch.linear_ws,
                             workspace_bytes=batch.linear_ws.numel(), fault_flag=self.flag)
        return out

    def attention(self, cache, qkv, batch):
        d, kv = self.width, self.heads * self.dim
        k, v = qkv[:, d:d + kv], qkv[:, d + kv:]
        B.abft_kv_write(cache, batch.total, batch.slots, k, qkv.stride(0), v, qkv.stride(0), self.kind)
        out = torch.empty(batch.total, d, device=DEV, dtype=self.dtype)
        B.abft_attention(cache, batch.kv_len.numel(), batch.q_start, batch.kv_len, self.table, self.table.stride(0), batch.total, batch.max_q,
                         self.max_kv, qkv, qkv.stride(0), self.heads * self.group, self.kind, 1 / math.sqrt(self.dim), True, 0, out, d,
                         batch.attention_ws, batch.attention_ws.numel())
        return out

    def norm(self, x):
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(self.dtype)

    def run(self, tokens, batch):
        """Logits of the new tokens (total x vocabulary); their keys and values are in the cache afterwards."""
        x = self.embedding[tokens].float()
        for block, cache in zip(self.blocks, self.caches):
            x = x + self.linear(block["out"], self.attention(cache, self.linear(block["qkv"], self.norm(x), batch), batch), batch)
            x = x + self.linear(block["down"], self.linear(block["up"], self.norm(x), batch), batch)
        return self.linear(self.head, self.norm(x), batch)


class Answer:
    """A step of every sequence, recorded once: takes `tokens`, leaves the next ones there and counts `length` up."""

    def __init__(self, model, tokens, length):
        self.model, self.batch = model, Batch(model, [1] * len(tokens))
        self.tokens, self.length = tokens.clone(), length.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):   # (what only a first call does, before the recording; nothing of it stays)
            self.step()
            self.tokens.copy_(tokens)
            self.length.copy_(length)
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step()

    def step(self):
        self.batch.place(self.model, self.length)
        self.logits = self.model.run(self.tokens, self.batch)
        self.tokens.copy_(self.logits.argmax(-1))
        self.length.add_(1)


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--seqs", type=int, default=4)
    parser.add_argument("--steps", type=int, default=32)
    parser.add_argument("--layers", type=int, default=2)
    parser.add_argument("--width", type=int, default=1024, help="a multiple of 256: query heads of 128, two for each head of the cache")
    args = parser.parse_args()
    lengths = [1 + 37 * i % 251 for i in range(args.seqs)]
    model = Decoder(layers=args.layers, heads=args.width // 256, seqs=args.seqs, max_kv=max(lengths) + args.steps)
    prompt = torch.randint(0, model.embedding.shape[0], (sum(lengths),), device=DEV)
    batch = Batch(model, lengths)
    batch.place(model, torch.zeros(args.seqs, dtype=torch.int64, device=DEV))
    logits = model.run(prompt, batch)
    answer = Answer(model, logits[batch.q_start[1:].long() - 1].argmax(-1), batch.kv_len.long())
    told = [answer.tokens.clone()]
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(args.steps - 1):
        answer.graph.replay()
        told.append(answer.tokens.clone())
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    for i, row in enumerate(torch.stack(told, 1).tolist()):
        print(f"prompt of {lengths[i]:4d} tokens ->", " ".join(str(t) for t in row[:12]), "...")
    print(f"{1e6 * took / max(1, args.steps - 1):.1f} us a step of {args.seqs} sequences; faults seen: {int(model.flag.item())}")


if __name__ == "__main__":
    main()
