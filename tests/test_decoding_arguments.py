"""What the entry points of the 8-bit matrices, the rotation and the draw of a token refuse, found on the host: no GPU is needed, no pointer is
followed."""
import ctypes as C
import os
import re
import types

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def lowbit():
    from paper_2604_03298_amd import enec, lowbit as module
    if not os.path.exists(enec.LIB_PATH):
        from paper_2604_03298_amd import build
        build.build()
    module.lib()
    return module


@pytest.fixture(scope="module")
def sampling(lowbit):
    from paper_2604_03298_amd import sampling as module
    module.lib()
    return module


P, ODD = 0x1000, 0x1001                                    # never dereferenced


def test_library_exports_every_declared_symbol(sampling):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "enec_sampling.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(enec_[a-z_0-9]+)\s*\(", text))
    assert declared == set(sampling.EXPORTS), declared ^ set(sampling.EXPORTS)
    plain = C.CDLL(sampling.enec.LIB_PATH)
    for name in declared:
        assert hasattr(plain, name), name
    assert C.sizeof(sampling.SamplingStruct) == 40 and sampling.SamplingStruct.uniform.offset == 32


def test_headers_compile_as_c(tmp_path):
    import subprocess
    source = tmp_path / "all.c"
    source.write_text('#include "enec_lowbit.h"\n#include "enec_sampling.h"\nint main(void) { return sizeof(enec_sampling) == 40 ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-fsyntax-only", str(source)], check=True)


def test_sizes_of_matrices(lowbit):
    assert lowbit.fp8_bytes(3, 1) == (3 * 128, 3 * 4)
    assert lowbit.fp8_bytes(3, 512) == (3 * 512, 3 * 4)
    assert lowbit.fp8_bytes(3, 513) == (3 * 640, 3 * 8)
    assert lowbit.fp8_bytes(0, 500) == (0, 0) and lowbit.fp8_bytes(5, 0) == (0, 0)
    assert lowbit.fp8_bytes(1 << 27, 128) == (1 << 34, 1 << 29)
    for rows, cols in (((1 << 27) + 1, 128), (1, (1 << 31) + 1), (1 << 34, 1), ((1 << 64) - 1, (1 << 64) - 1)):
        with pytest.raises(lowbit.enec.EnecError):
            lowbit.fp8_bytes(rows, cols)


def test_matrices_that_are_refused(lowbit):
    L = lowbit.lib()
    quantize = lambda src=P, rows=4, cols=32, stride=32, dtype=0, codes=P, scales=P: L.enec_fp8_quantize(src, rows, cols, stride, dtype, codes, scales, None)  # noqa: E731
    back = lambda codes=P, scales=P, rows=4, cols=32, out=P, stride=32, dtype=0: L.enec_fp8_dequantize(codes, scales, rows, cols, out, stride, dtype, None)  # noqa: E731
    for call, name in ((quantize, "src"), (back, "out")):
        assert call(dtype=3) == call(dtype=-1) == lowbit.E_DTYPE
        for bad in ({name: None}, {name: ODD}, {"codes": None}, {"codes": 0x1008}, {"scales": None}, {"scales": 0x1002}, {"stride": 31},
                    {"rows": 1 << 40}, {"cols": 1 << 40}):
            assert call(**bad) == lowbit.E_ARG, bad
        assert call(**{name: 0x1002, "dtype": 2}) == lowbit.E_ARG           # fp32 at an address of 16 bits
        assert call(rows=0) == call(cols=0) == lowbit.OK                    # nothing to do, nothing enqueued


def test_products_that_are_refused(lowbit):
    L = lowbit.lib()

    def linear(x=P, m=4, x_stride=64, dtype=0, codes=P, scales=P, n=8, k=64, y=P, y_stride=8, ws=P, size=1 << 40):
        return L.enec_fp8_linear(x, m, x_stride, dtype, codes, scales, n, k, y, y_stride, ws, size, None)

    def matmul(x=P, x_scales=P, m=4, codes=P, scales=P, n=8, k=64, y=P, y_stride=8, dtype=0, ws=P, size=1 << 40):
        return L.enec_fp8_matmul(x, x_scales, m, codes, scales, n, k, y, y_stride, dtype, ws, size, None)

    assert linear(dtype=2) == linear(dtype=7) == matmul(dtype=3) == matmul(dtype=-1) == lowbit.E_DTYPE
    for bad in ({"x": None}, {"codes": None}, {"scales": None}, {"y": None}, {"y": ODD}, {"codes": 0x1008}, {"scales": 0x1002}, {"y_stride": 7},
                {"m": 1 << 40}, {"n": 1 << 40}, {"k": 1 << 40, "x_stride": 1 << 40}, {"n": 1 << 25, "k": 1 << 20, "y_stride": 1 << 25, "x_stride": 1 << 20}):
        assert linear(**bad) == lowbit.E_ARG, bad
        bad.pop("x_stride", None)
        assert matmul(**bad) == lowbit.E_ARG, bad
    assert linear(x=ODD) == linear(x_stride=63) == matmul(x=0x1008) == matmul(x_scales=0x1001) == matmul(x_scales=None) == lowbit.E_ARG
    assert matmul(y=0x1002, dtype=2) == lowbit.E_ARG
    assert linear(m=0) == linear(n=0, y_stride=0) == matmul(m=0) == matmul(n=0) == lowbit.OK
    for call, space in ((linear, lowbit.fp8_linear_workspace), (matmul, lowbit.fp8_matmul_workspace)):
        assert space(0, 5, 5) == space(5, 0, 5) == space(5, 5, 0) == space(1 << 40, 5, 5) == 0
        for m, n, k in ((1, 64, 8192), (40, 512, 4096), (200, 300, 8192)):
            need = space(m, n, k)
            if need:
                sizes = dict(m=m, n=n, k=k, y_stride=n, **({"x_stride": k} if call is linear else {}))
                assert call(**sizes, ws=None, size=0) == lowbit.E_CAPACITY
                assert call(**sizes, ws=P, size=need - 1) == lowbit.E_CAPACITY
                assert call(**sizes, ws=None, size=need) == lowbit.E_CAPACITY
                assert call(**sizes, ws=0x1008, size=need) == lowbit.E_ARG
        for n, k in ((64, 8192), (11008, 4096), (4096, 11008), (100, 300), (32003, 2047)):
            sizes = [space(m, n, k) for m in (1, 2, 16, 17, 32, 33, 64, 65, 96, 128, 129, 256, 500, 1000, 4096)]
            assert sizes == sorted(sizes)                   # what serves many rows serves fewer


def test_rotations_that_are_refused(lowbit):
    L = lowbit.lib()

    def write(k=P, v=P, q=P, q_out=0x2000, q_heads=8, dtype=0, turns=P, positions=100, rotary=128, q_strides=(1024, 128), o_strides=(1024, 128), codes=P, v_codes=P,
              k_scales=P, v_scales=P, pages=10, page=64, heads=4, dim=128, table=P, starts=P, lengths=P, stride=8, batch=3, tokens=5, status=None):
        c = lowbit.CacheStruct(codes, k_scales, v_codes, v_scales, pages, page, heads, dim)
        b = lowbit.BatchStruct(table, starts, lengths, stride, batch, tokens, status)
        return L.enec_cache_write_rotated(C.byref(c), C.byref(b), k, 512, 128, v, 512, 128, q, *q_strides, q_out, *o_strides, q_heads, dtype, turns, positions,
                                          rotary, 0, None)

    assert write(dtype=2) == write(dtype=5) == lowbit.E_DTYPE
    assert write(page=24) == write(dim=96) == lowbit.E_BLOCK
    for bad in ({"codes": None}, {"v_codes": None}, {"k_scales": None}, {"v_scales": None}, {"codes": 0x1008}, {"table": None}, {"starts": None}, {"lengths": None},
                {"status": ODD}, {"stride": 0}, {"heads": 0}, {"pages": 0}, {"tokens": 1 << 24}, {"k": None}, {"v": None}, {"k": ODD}, {"v": ODD}, {"turns": None},
                {"turns": 0x1004}, {"rotary": 0}, {"rotary": 24}, {"rotary": 144}, {"rotary": 256}, {"q": None}, {"q_out": None}, {"q": ODD}, {"q_out": ODD},
                {"q_heads": 0}, {"q_heads": 6}, {"q": None, "q_out": None}, {"q_out": P, "o_strides": (1024, 256)}, {"q_out": P, "o_strides": (2048, 128)}):
        assert write(**bad) == lowbit.E_ARG, bad
    assert write(batch=0) == write(tokens=0) == write(tokens=0, k=None, v=None, turns=None, q=None, q_out=None, q_heads=0) == lowbit.OK


def test_draws_that_are_refused(sampling):
    L = sampling.lib()

    def sample(logits=P, rows=3, vocab=100, stride=100, dtype=2, tokens=P, log_probs=None, ws=P, size=1 << 40, **how):
        h = sampling.SamplingStruct(how.get("temperature"), how.get("top_k"), how.get("top_p"), how.get("min_p"), how.get("uniform", P))
        return L.enec_sample(logits, rows, vocab, stride, dtype, C.byref(h), tokens, log_probs, ws, size, None)

    assert sample(dtype=3) == sample(dtype=-1) == sampling.E_DTYPE
    for bad in ({"logits": None}, {"logits": 0x1002}, {"logits": ODD, "dtype": 0}, {"tokens": None}, {"tokens": 0x1002}, {"log_probs": ODD}, {"uniform": None},
                {"uniform": 0x1002}, {"temperature": ODD}, {"top_k": ODD}, {"top_p": ODD}, {"min_p": ODD}, {"vocab": 0}, {"vocab": (1 << 22) + 1, "stride": 1 << 23},
                {"stride": 99}, {"rows": (1 << 24) + 1}):
        assert sample(**bad) == sampling.E_ARG, bad
    assert L.enec_sample(P, 3, 100, 100, 2, None, P, None, P, 1 << 40, None) == sampling.E_ARG
    assert sample(rows=0) == sampling.OK
    assert sampling.sample_workspace(0, 5) == sampling.sample_workspace(5, 0) == sampling.sample_workspace(5, 1 << 23) == 0
    for vocab in (10, 32003, 131072):
        sizes = [sampling.sample_workspace(r, vocab) for r in (1, 2, 8, 31, 64, 100, 255, 256, 1000)]
        assert sizes == sorted(sizes)
        if sizes[0]:
            assert sample(rows=1, vocab=vocab, stride=vocab, ws=None, size=0) == sampling.E_CAPACITY
            assert sample(rows=1, vocab=vocab, stride=vocab, size=sizes[0] - 1) == sampling.E_CAPACITY
            assert sample(rows=1, vocab=vocab, stride=vocab, ws=0x1008) == sampling.E_ARG


class FakeTensor:
    """Looks like a tensor on GPU 0 to the binding's checks."""

    def __init__(self, held, device=0):
        self.held, self.device = held, device

    def __getattr__(self, name):
        return getattr(self.held, name)

    def get_device(self):
        return self.device


def test_tensors_that_the_binding_refuses(lowbit, sampling):
    import torch
    z = lambda *shape, dtype=torch.uint8, device=0: FakeTensor(torch.zeros(*shape, dtype=dtype), device)  # noqa: E731
    bf = lambda *shape, **how: z(*shape, dtype=torch.bfloat16, **how)  # noqa: E731
    f, i = (lambda *shape, **how: z(*shape, dtype=torch.float32, **how)), (lambda *shape, **how: z(*shape, dtype=torch.int32, **how))
    c, s = z(4, 256), z(4, 4)
    for call in (lambda: lowbit.fp8_quantize(bf(4, 100), c, s), lambda: lowbit.fp8_quantize(bf(3, 200), c, s), lambda: lowbit.fp8_quantize(bf(4, 200), c, z(4, 2)),
                 lambda: lowbit.fp8_quantize(bf(4, 200), z(4, 200), s), lambda: lowbit.fp8_quantize(bf(4, 200), c, FakeTensor(s.held.t())), lambda: lowbit.fp8_quantize(bf(200), c, s),
                 lambda: lowbit.fp8_quantize(bf(4, 200, device=1), c, s), lambda: lowbit.fp8_quantize(torch.zeros(4, 200), c, s),
                 lambda: lowbit.fp8_dequantize(c, s, bf(4, 300)), lambda: lowbit.fp8_dequantize(c, i(4, 4), bf(4, 200)),
                 lambda: lowbit.fp8_linear(bf(2, 200), c, s, bf(2, 5)), lambda: lowbit.fp8_linear(bf(2, 200), c, s, f(2, 4)), lambda: lowbit.fp8_linear(bf(2, 300), c, s, bf(2, 4)),
                 lambda: lowbit.fp8_linear(bf(2, 200), c, s, bf(2, 4), z(9, device=1)), lambda: lowbit.fp8_matmul(z(2, 128), z(2, 4), c, s, f(2, 4)),
                 lambda: lowbit.fp8_matmul(z(2, 256), z(2, 4), c, s, f(3, 4)), lambda: lowbit.fp8_matmul(z(2, 256, device=1), z(2, 4), c, s, f(2, 4)),
                 lambda: sampling.sample(f(4, 9), f(3), i(4)), lambda: sampling.sample(f(4, 9), f(4), f(4)), lambda: sampling.sample(f(4, 9), f(4), i(4), f(4, 1)),
                 lambda: sampling.sample(f(4, 9), f(4), i(4), top_k=f(4)), lambda: sampling.sample(f(4, 9), f(4), i(4), top_p=f(4, device=1)),
                 lambda: sampling.sample(f(4, 9, device=-1), f(4), i(4)), lambda: sampling.sample(f(4, 9), f(4), i(4), workspace=z(9, device=1)),
                 lambda: sampling.sample(FakeTensor(f(4, 9).held.t()), f(9), i(9)), lambda: sampling.sample(f(4, 9), FakeTensor(f(8).held[::2]), i(4))):
        with pytest.raises(ValueError):
            call()
    cache = lowbit.Cache(z(3, 2, 16, 64), z(3, 2), z(3, 2, 64, 16), z(3, 2))
    cache.device = 0

    def write(k=None, v=None, q=None, q_out=None, turns=None):
        kv = lambda: bf(5, 2, 64)  # noqa: E731
        lowbit.cache_write_rotated(cache, k or kv(), v or kv(), q, q_out, turns or f(9, 32, 2), i(1, 2), i(2), i(1))

    for bad in ({"k": bf(5, 3, 64)}, {"v": bf(5, 2, 65)}, {"q": bf(5, 4, 64)}, {"q_out": bf(5, 4, 64)}, {"q": bf(4, 4, 64), "q_out": bf(4, 4, 64)},
                {"q": f(5, 4, 64), "q_out": f(5, 4, 64)}, {"q": bf(5, 4, 64), "q_out": bf(5, 2, 64)}, {"q": bf(5, 4, 64, device=1), "q_out": bf(5, 4, 64)},
                {"turns": f(9, 32)}, {"turns": f(9, 32, 3)}, {"turns": bf(9, 32, 2)}, {"turns": f(9, 32, 2, device=1)}):
        with pytest.raises(ValueError):
            write(**bad)


def test_another_gpu_than_the_current_one(lowbit, sampling, monkeypatch):
    """Kernels are launched on the current GPU: tensors on another one, or a stream of another one, are refused before that."""
    import torch
    z = lambda *shape, dtype=torch.uint8: FakeTensor(torch.zeros(*shape, dtype=dtype), 1)  # noqa: E731
    bf, i = (lambda *shape: z(*shape, dtype=torch.bfloat16)), (lambda *shape: z(*shape, dtype=torch.int32))
    f = lambda *shape: z(*shape, dtype=torch.float32)  # noqa: E731
    cache = lowbit.Cache(z(3, 2, 16, 64), z(3, 2), z(3, 2, 64, 16), z(3, 2))
    cache.device = 1
    c, s, stream = z(4, 256), z(4, 4), types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=0)
    for current, how in ((0, {}), (1, {"stream": stream})):
        monkeypatch.setattr(lowbit, "_current_device", lambda: current)
        for call in (lambda: lowbit.fp8_quantize(bf(4, 200), c, s, **how), lambda: lowbit.fp8_dequantize(c, s, bf(4, 200), **how),
                     lambda: lowbit.fp8_linear(bf(2, 200), c, s, bf(2, 4), **how), lambda: lowbit.fp8_matmul(z(2, 256), z(2, 4), c, s, f(2, 4), **how),
                     lambda: sampling.sample(f(4, 9), f(4), i(4), **how),
                     lambda: lowbit.cache_write_rotated(cache, bf(5, 2, 64), bf(5, 2, 64), None, None, f(9, 32, 2), i(1, 2), i(2), i(1), **how)):
            with pytest.raises(ValueError, match="current one"):
                call()
