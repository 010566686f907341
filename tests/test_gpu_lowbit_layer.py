"""The low-bit operators together, as examples/low_bit_layer.py runs them, against the same layer in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

from conftest import ROOT
import lowbit_plain as plain

sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def norm(x):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("four_bits", [False, True])
def test_layer(dtype, four_bits):
    """Values are rounded to the format where the layer rounds them.  What is left are roundings that fall the other way: at most ten of
    them on a path, 2^-9 each, and 4-bit codes that one flips -- a change of 2^-8 flips a code of spacing 1/4 to 1/2 about once in 64
    times, by 0.3 of the value: 0.04 in the root mean square.  Twice their sum is 0.1; a step that is wired wrongly is off by 0.3 and
    more."""
    import low_bit_layer as example
    hidden, ffn, heads, kv_heads, dim, page = 200, 328, 4, 2, 64, 16
    prompts = (37, 0, 1, 70)
    layer, exact, steps, held, _ = example.run(hidden, ffn, heads, kv_heads, dim, prompts, 3, page, dtype, four_bits)
    near = lambda x: plain.rounded(x, dtype).double().numpy()  # noqa: E731
    quantised = lambda x: plain.mx4_decode(*plain.mx4_encode(x), x.shape[1])  # noqa: E731
    weights = {}
    for name, w in exact.items():
        w = w.double().cpu().numpy()
        codes, scales = plain.mx4_encode(w)
        assert np.array_equal(layer.weights[name][0].cpu().numpy(), codes) and np.array_equal(layer.weights[name][1].cpu().numpy(), scales)
        weights[name] = plain.mx4_decode(codes, scales, w.shape[1])
    keys, values = plain.PlainCache(page, kv_heads, dim), plain.PlainCache(page, kv_heads, dim)
    per = 100
    table = np.arange(len(prompts) * per).reshape(len(prompts), per)            # where pages lie does not matter
    for i, (x, starts, lengths, y) in enumerate(steps):
        x, starts, lengths = x.double().cpu().numpy(), starts.tolist(), lengths.tolist()
        if i:                                                                   # a token of an idle sequence: no place in the cache
            assert lengths[1] == 0
        qkv = near(near(norm(x)) @ weights["qkv"].T).reshape(len(x), -1, dim)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        keys.write(k, table, starts, lengths)
        values.write(v, table, starts, lengths)
        seen = np.zeros(q.shape)
        for b in range(len(prompts)):
            if lengths[b]:
                rows = slice(starts[b], starts[b + 1])
                seen[rows] = plain.attention(q[rows], keys.read(table[b], lengths[b]), values.read(table[b], lengths[b]), dim ** -0.5, dtype)[0]
        after = near(x + near(near(seen).reshape(len(x), -1) @ weights["out"].T))
        through = quantised if four_bits and i == 0 else lambda t: t
        gate, up = np.split(near(through(near(norm(after))) @ weights["up"].T), 2, axis=1)
        made = near(through(near(gate / (1 + np.exp(-gate)) * up)) @ weights["down"].T)
        want, got = made + after - x, y.double().cpu().numpy() - x
        assert np.isfinite(got).all()
        off = np.sqrt(((got - want) ** 2).mean() / (want ** 2).mean())
        assert off < 0.1, (i, off)
    for got, cache in zip(held, (keys, values)):
        want = np.concatenate([cache.read(table[b], n) for b, n in enumerate(lengths)])
        off = np.sqrt(((got.double().cpu().numpy() - want) ** 2).mean() / (want ** 2).mean())
        assert off < 0.1, off


def test_scratch_memory_for_the_largest_step_serves_smaller_ones():
    import low_bit_layer as example
    hidden, ffn, heads, kv_heads, dim, batch = 256, 384, 32, 8, 128, 4
    g = torch.Generator("cuda").manual_seed(2)
    normal = lambda *shape: (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(torch.bfloat16)  # noqa: E731
    matrices = {"qkv": normal((heads + 2 * kv_heads) * dim, hidden), "out": normal(hidden, heads * dim), "up": normal(2 * ffn, hidden), "down": normal(hidden, ffn)}
    layer = example.Layer({name: example.stored(w) for name, w in matrices.items()}, hidden, ffn, heads, kv_heads, dim, 2 * batch)
    table = torch.arange(2 * batch, dtype=torch.int32, device="cuda").view(batch, 2)
    longest = 131072
    layer.reserve(batch, 400, 100, longest)
    for new in (100, 64, 32, 16, 5, 1):
        x = normal(batch * new, hidden)
        lengths = torch.full((batch,), 100, dtype=torch.int32, device="cuda")
        layer.workspace.fill_(0xFF)                        # (NaN, were it read unwritten)
        for four_bits in (False, True):
            y = layer.step(x, table, example.starts_of([new] * batch), lengths, new, longest, four_bits)
            assert torch.isfinite(y).all()
    assert layer.status.item() == 0
