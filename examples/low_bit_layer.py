"""A decoder layer that is stored losslessly, runs from 4-bit weights and keeps an 8-bit cache.

    python examples/low_bit_layer.py [--hidden 4096 --ffn 11008 --heads 32 --kv-heads 8 --dtype bf16]

The layer's matrices are held as ENEC streams (the exact weights, as a checkpoint would hold them).  Loading brings each back bit for
bit and quantises it to 4 bits; what the layer then reads on a step are the 4-bit weights and the paged 8-bit cache.  A step takes the
newest tokens of several sequences, whatever their number: whole prompts first, then one token a sequence, the latter also as a graph.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_03298_amd import enec, lowbit  # noqa: E402


def check(status):
    if status != enec.OK:
        raise RuntimeError(enec.strerror(status))


def stored(matrix):
    """A matrix as an ENEC stream, cut to its size."""
    ws = enec.new_workspace(matrix.numel())
    out = torch.empty(enec.compress_bound(matrix.numel(), enec.dtype_of(matrix)), dtype=torch.uint8, device=matrix.device)
    size = torch.zeros(1, dtype=torch.int64, device=matrix.device)
    check(enec.compress(matrix, enec.tune(matrix, ws), out, ws, out_bytes=size))
    return out[:int(size.item())].clone()


def loaded(stream, rows, cols, dtype):
    """The 4-bit form of a stored matrix."""
    exact = torch.empty(rows, cols, dtype=dtype, device=stream.device)
    check(enec.decompress(stream, exact))
    codes, scales = lowbit.mx4_empty(rows, cols)
    check(lowbit.mx4_quantize(exact, codes, scales))
    return codes, scales


def rms_norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Layer:
    def __init__(self, streams, hidden, ffn, heads, kv_heads, head_dim, pages, page_tokens=64, dtype=torch.bfloat16):
        """streams: {"qkv", "out", "up", "down"}: ((heads + 2 kv_heads) head_dim, hidden), (hidden, heads head_dim), (2 ffn, hidden) -- gate
        and up -- and (hidden, ffn)."""
        self.hidden, self.ffn, self.heads, self.kv_heads, self.head_dim, self.dtype = hidden, ffn, heads, kv_heads, head_dim, dtype
        shapes = {"qkv": ((heads + 2 * kv_heads) * head_dim, hidden), "out": (hidden, heads * head_dim), "up": (2 * ffn, hidden), "down": (hidden, ffn)}
        self.weights = {name: loaded(streams[name], *shape, dtype) for name, shape in shapes.items()}
        self.shapes = shapes
        self.cache = lowbit.Cache.empty(pages, kv_heads, head_dim, page_tokens)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")      # what only the device can see
        self.workspace = None

    def reserve(self, batch, tokens, max_new, max_length):
        """Scratch memory for steps of at most these sizes; one piece serves the calls of a stream, one after the other."""
        tokens = max(tokens, batch)                                         # (what serves the largest call serves all smaller ones)
        need = [lowbit.cache_attention_workspace(self.cache, batch, tokens, self.heads, max(max_new, 1), max_length)]
        for n, k in self.shapes.values():
            need += [lowbit.mx4_linear_workspace(tokens, n, k), lowbit.mx4_matmul_workspace(tokens, n, k)]
        self.workspace = torch.empty(max(max(need), 16), dtype=torch.uint8, device="cuda")

    def product(self, x, name, four_bits=False):
        """x w^T; four_bits: with x quantised as well, which is what a prompt's many tokens gain from."""
        n, k = self.shapes[name]
        out = torch.empty(x.shape[0], n, dtype=x.dtype, device=x.device)
        if four_bits:
            held = lowbit.mx4_empty(x.shape[0], k)
            check(lowbit.mx4_quantize(x, *held))
            check(lowbit.mx4_matmul(*held, *self.weights[name], out, self.workspace))
        else:
            check(lowbit.mx4_linear(x, *self.weights[name], out, self.workspace))
        return out

    def step(self, x, table, starts, lengths, max_new, max_length, four_bits=False):
        """The layer over the newest tokens x (tokens, hidden) of the sequences; their keys and values go to the cache."""
        qkv = self.product(rms_norm(x), "qkv").view(x.shape[0], -1, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)                      # views of a row will do
        check(lowbit.cache_write(self.cache, k, v, table, starts, lengths, self.status))
        seen = torch.empty(x.shape[0], self.heads, self.head_dim, dtype=x.dtype, device=x.device)
        check(lowbit.cache_attention(self.cache, q, seen, table, starts, lengths, max_new, max_length, self.workspace, status=self.status))
        x = x + self.product(seen.flatten(1), "out")
        gate, up = self.product(rms_norm(x), "up", four_bits).float().chunk(2, 1)
        return x + self.product((torch.nn.functional.silu(gate) * up).to(x.dtype), "down", four_bits)


def starts_of(counts):
    return torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(device="cuda", dtype=torch.int32)


def run(hidden=4096, ffn=11008, heads=32, kv_heads=8, head_dim=128, prompts=(1000, 33, 0, 2047), new_tokens=4, page_tokens=64,
        dtype=torch.bfloat16, four_bits=True, seed=1):
    """Prompts, then new_tokens single tokens for each sequence (an idle one, of length 0, stays idle).  -> (layer, exact weights, inputs
    and outputs of every step, what it measured)."""
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape, std=1.0: (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    exact = {"qkv": normal((heads + 2 * kv_heads) * head_dim, hidden, std=hidden ** -0.5), "out": normal(hidden, heads * head_dim, std=(heads * head_dim) ** -0.5),
             "up": normal(2 * ffn, hidden, std=hidden ** -0.5), "down": normal(hidden, ffn, std=ffn ** -0.5)}
    streams = {name: stored(w) for name, w in exact.items()}

    batch, last = len(prompts), max(prompts) + new_tokens
    per = -(-last // page_tokens)
    pages = batch * per
    layer = Layer(streams, hidden, ffn, heads, kv_heads, head_dim, pages, page_tokens, dtype)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(batch, per)       # pages lie anywhere
    layer.reserve(batch, sum(prompts), max(prompts), last)

    figures = {"bf16 or fp16 MB": sum(w.numel() for w in exact.values()) * 2e-6, "stored MB": sum(s.numel() for s in streams.values()) * 1e-6,
               "4-bit MB": sum(t.numel() for w in layer.weights.values() for t in w) * 1e-6}
    starts, lengths = starts_of(list(prompts)), torch.tensor(prompts, dtype=torch.int32, device="cuda")
    steps = []
    x = normal(sum(prompts), hidden)
    layer.step(x, table, starts, lengths, max(prompts), last, four_bits)                             # (warms up: a page written again holds the same)
    torch.cuda.synchronize()
    begin = time.perf_counter()
    y = layer.step(x, table, starts, lengths, max(prompts), last, four_bits)
    torch.cuda.synchronize()
    figures["prompts us"] = (time.perf_counter() - begin) * 1e6
    steps.append((x, starts, lengths.clone(), y))

    # single tokens: a captured step, replayed as the lengths grow.  The warm-up writes the first token, which is then written again.
    active = (lengths > 0).to(torch.int32)
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    lengths += active
    x = normal(batch, hidden)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(x, table, starts, lengths, 1, last)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(x, table, starts, lengths, 1, last)
    spent = 0.0
    for i in range(new_tokens):
        if i:
            lengths += active
            x.copy_(normal(batch, hidden))
        torch.cuda.synchronize()
        begin = time.perf_counter()
        graph.replay()
        torch.cuda.synchronize()
        spent += time.perf_counter() - begin
        steps.append((x.clone(), starts, lengths.clone(), y.clone()))
    figures["token step us"] = spent / max(new_tokens, 1) * 1e6
    if int(layer.status.item()) != enec.OK:
        raise RuntimeError(enec.strerror(int(layer.status.item())))

    # what the cache holds of a sequence, as a user who moves it elsewhere would read it
    whole = lengths.clone()
    count = int(whole.sum())
    k, v = (torch.empty(count, kv_heads, head_dim, dtype=dtype, device="cuda") for _ in range(2))
    check(lowbit.cache_read(layer.cache, k, v, table, starts_of(whole.tolist()), whole, layer.status))
    figures["cache bytes a token"] = 2 * kv_heads * (head_dim + 1 / page_tokens)
    return layer, exact, steps, (k, v), figures


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("hidden", 4096), ("ffn", 11008), ("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("new-tokens", 32)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--prompts", type=int, nargs="+", default=[1000, 33, 0, 2047])
    p.add_argument("--dtype", choices=("bf16", "fp16"), default="bf16")
    a = p.parse_args()
    *_, figures = run(a.hidden, a.ffn, a.heads, a.kv_heads, a.head_dim, a.prompts, a.new_tokens, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float16)
    for name, value in figures.items():
        print(f"{name:22s} {value:10.1f}")


if __name__ == "__main__":
    main()
