"""Kernels are launched on the current GPU: every low-bit call refuses tensors on another one, and a stream of another one, before it enqueues anything; pinned host
memory among the tensors hides none of them."""
import os
import types

import pytest

from test_decoding_arguments import FakeTensor


@pytest.fixture(scope="module")
def lowbit():
    from paper_2604_03298_amd import enec, lowbit as module
    if not os.path.exists(enec.LIB_PATH):
        from paper_2604_03298_amd import build
        build.build()
    module.lib()
    return module


class Pinned(FakeTensor):
    """In host memory that a GPU reaches."""

    def __init__(self, held):
        super().__init__(held, -1)

    def is_pinned(self):
        return True


def calls(lowbit, gpu, pinned=()):
    """Every call, its tensors on that GPU but for the ones named."""
    import torch
    from paper_2604_03298_amd import sampling

    def make(kind):
        return lambda name, *shape: Pinned(torch.zeros(*shape, dtype=kind)) if name in pinned else FakeTensor(torch.zeros(*shape, dtype=kind), gpu)
    z, bf, f, i = make(torch.uint8), make(torch.bfloat16), make(torch.float32), make(torch.int32)
    cache = lowbit.Cache(z("", 3, 2, 16, 64), z("", 3, 2), z("", 3, 2, 64, 16), z("", 3, 2))
    cache.device = gpu
    x, y, codes, scales = bf("in", 2, 200), bf("out", 2, 4), z("codes", 4, 128), z("scales", 4, 8)
    codes8, scales8, src, back = z("codes", 4, 256), z("scales", 4, 4), bf("in", 4, 200), bf("out", 4, 200)
    k, v, q, o = bf("in", 5, 2, 64), bf("out", 5, 2, 64), bf("in", 5, 4, 64), bf("out", 5, 4, 64)
    batch = (i("table", 1, 2), i("starts", 2), i("lengths", 1))
    return {
        "mx4_quantize": lambda **how: lowbit.mx4_quantize(src, codes, scales, **how),
        "mx4_dequantize": lambda **how: lowbit.mx4_dequantize(codes, scales, back, **how),
        "mx4_linear": lambda **how: lowbit.mx4_linear(x, codes, scales, y, **how),
        "mx4_matmul": lambda **how: lowbit.mx4_matmul(z("in", 2, 128), z("in", 2, 8), codes, scales, y, **how),
        "fp8_quantize": lambda **how: lowbit.fp8_quantize(src, codes8, scales8, **how),
        "fp8_dequantize": lambda **how: lowbit.fp8_dequantize(codes8, scales8, back, **how),
        "fp8_linear": lambda **how: lowbit.fp8_linear(x, codes8, scales8, y, **how),
        "fp8_matmul": lambda **how: lowbit.fp8_matmul(z("in", 2, 256), z("in", 2, 4), codes8, scales8, y, **how),
        "cache_write": lambda **how: lowbit.cache_write(cache, k, v, *batch, **how),
        "cache_read": lambda **how: lowbit.cache_read(cache, k, v, *batch, **how),
        "cache_attention": lambda **how: lowbit.cache_attention(cache, q, o, *batch, 5, 20, **how),
        "cache_write_rotated": lambda **how: lowbit.cache_write_rotated(cache, k, v, q, o, f("turns", 9, 32, 2), *batch, **how),
        "sample": lambda **how: sampling.sample(f("in", 4, 9), f("codes", 4), i("out", 4), **how),
    }


NAMES = ["mx4_quantize", "mx4_dequantize", "mx4_linear", "mx4_matmul", "fp8_quantize", "fp8_dequantize", "fp8_linear", "fp8_matmul", "cache_write", "cache_read",
         "cache_attention", "cache_write_rotated", "sample"]


@pytest.mark.parametrize("pinned", [(), ("codes", "scales", "table"), ("in",), ("out",)])
@pytest.mark.parametrize("name", NAMES)
def test_another_gpu_is_refused(lowbit, monkeypatch, name, pinned):
    import torch

    def reached(*_):
        raise AssertionError("the call went on to the library")
    monkeypatch.setattr(lowbit, "_raw_stream", reached)
    monkeypatch.setattr(lowbit.enec, "_stream_handle", reached)
    stream = types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=0)
    call = calls(lowbit, 1, pinned)[name]
    for current, how in ((0, {}), (1, {"stream": stream})):
        monkeypatch.setattr(lowbit, "_current_device", lambda: current)
        with pytest.raises(ValueError, match="current one"):
            call(**how)


@pytest.mark.parametrize("name", NAMES)
def test_the_current_gpu_s_own_stream_is_taken(lowbit, monkeypatch, name):
    class Taken(Exception):
        pass

    def stream_of(device):
        raise Taken(device)
    monkeypatch.setattr(lowbit, "_current_device", lambda: 1)
    monkeypatch.setattr(lowbit, "_raw_stream", stream_of)
    with pytest.raises(Taken) as e:
        calls(lowbit, 1)[name]()
    assert e.value.args == (1,)
