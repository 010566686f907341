"""What the low-bit entry points refuse, found on the host: no GPU is needed, no pointer is followed."""
import ctypes as C
import os
import re

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


P, ODD = 0x1000, 0x1001                                    # never dereferenced


def test_library_exports_every_declared_symbol(lowbit):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "enec_lowbit.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(enec_[a-z_0-9]+)\s*\(", text))
    assert declared == set(lowbit.EXPORTS), declared ^ set(lowbit.EXPORTS)
    plain = C.CDLL(lowbit.enec.LIB_PATH)
    for name in declared:
        assert hasattr(plain, name), name


def test_structures_have_the_header_s_layout(lowbit):
    assert C.sizeof(lowbit.CacheStruct) == 48 and lowbit.CacheStruct.n_pages.offset == 32
    assert C.sizeof(lowbit.BatchStruct) == 48 and lowbit.BatchStruct.status.offset == 40


def test_sizes_of_matrices(lowbit):
    assert lowbit.mx4_bytes(3, 1) == (3 * 64, 3 * 4)
    assert lowbit.mx4_bytes(3, 128) == (3 * 64, 3 * 4)
    assert lowbit.mx4_bytes(3, 129) == (3 * 128, 3 * 8)
    assert lowbit.mx4_bytes(0, 500) == (0, 0) and lowbit.mx4_bytes(5, 0) == (0, 0)
    assert lowbit.mx4_bytes(1 << 27, 128) == (1 << 33, 1 << 29)
    for rows, cols in (((1 << 27) + 1, 128), (1, (1 << 31) + 1), (1 << 34, 1), ((1 << 64) - 1, (1 << 64) - 1)):
        with pytest.raises(lowbit.enec.EnecError):
            lowbit.mx4_bytes(rows, cols)


def test_matrices_that_are_refused(lowbit):
    L = lowbit.lib()
    quantize = lambda src=P, rows=4, cols=32, stride=32, dtype=0, codes=P, scales=P: L.enec_mx4_quantize(src, rows, cols, stride, dtype, codes, scales, None)  # noqa: E731
    back = lambda codes=P, scales=P, rows=4, cols=32, out=P, stride=32, dtype=0: L.enec_mx4_dequantize(codes, scales, rows, cols, out, stride, dtype, None)  # noqa: E731
    for call, name in ((quantize, "src"), (back, "out")):
        assert call(dtype=3) == call(dtype=-1) == lowbit.E_DTYPE
        for bad in ({name: None}, {name: ODD}, {"codes": None}, {"codes": 0x1008}, {"scales": None}, {"scales": 0x1002}, {"stride": 31},
                    {"rows": 1 << 40}, {"cols": 1 << 40}):
            assert call(**bad) == lowbit.E_ARG, bad
        assert call(**{name: 0x1002, "dtype": 2}) == lowbit.E_ARG           # fp32 at an address of 16 bits
        assert call(rows=0) == call(cols=0) == lowbit.OK                    # nothing to do, nothing enqueued


def test_products_that_are_refused(lowbit):
    L = lowbit.lib()

    def linear(x=P, m=4, x_stride=64, dtype=0, codes=P, scales=P, n=8, k=64, y=P, y_stride=8, ws=None, size=0):
        return L.enec_mx4_linear(x, m, x_stride, dtype, codes, scales, n, k, y, y_stride, ws, size, None)

    def matmul(x=P, x_scales=P, m=4, codes=P, scales=P, n=8, k=64, y=P, y_stride=8, dtype=0, ws=None, size=0):
        return L.enec_mx4_matmul(x, x_scales, m, codes, scales, n, k, y, y_stride, dtype, ws, size, None)

    assert linear(dtype=2) == linear(dtype=7) == matmul(dtype=3) == matmul(dtype=-1) == lowbit.E_DTYPE
    for bad in ({"x": None}, {"codes": None}, {"scales": None}, {"y": None}, {"y": ODD}, {"codes": 0x1008}, {"scales": 0x1002}, {"y_stride": 7},
                {"m": 1 << 40}, {"n": 1 << 40}, {"k": 1 << 40, "x_stride": 1 << 40} ):
        assert linear(**bad) == lowbit.E_ARG, bad
        bad.pop("x_stride", None)
        assert matmul(**bad) == lowbit.E_ARG, bad
    assert linear(x=ODD) == linear(x_stride=63) == matmul(x=0x1008) == matmul(x_scales=0x1001) == matmul(x_scales=None) == lowbit.E_ARG
    assert matmul(y=0x1002, dtype=2) == lowbit.E_ARG
    assert linear(m=0) == linear(n=0, y_stride=0) == matmul(m=0) == matmul(n=0) == lowbit.OK
    for call, space in ((linear, lowbit.mx4_linear_workspace), (matmul, lowbit.mx4_matmul_workspace)):
        for m, n, k in ((1, 64, 8192), (40, 512, 4096), (200, 300, 8192)):
            need = space(m, n, k)
            if need:
                sizes = dict(m=m, n=n, k=k, y_stride=n, **({"x_stride": k} if call is linear else {}))
                assert call(**sizes) == lowbit.E_CAPACITY
                assert call(**sizes, ws=P, size=need - 1) == lowbit.E_CAPACITY
                assert call(**sizes, ws=None, size=need) == lowbit.E_CAPACITY
                assert call(**sizes, ws=0x1008, size=need) == lowbit.E_ARG


def test_caches_that_are_refused(lowbit):
    L = lowbit.lib()

    def structs(codes=P, v_codes=P, k_scales=P, v_scales=P, pages=10, page=64, heads=4, dim=128, table=P, starts=P, lengths=P, stride=8, batch=3, tokens=5, status=None):
        return (lowbit.CacheStruct(codes, k_scales, v_codes, v_scales, pages, page, heads, dim),
                lowbit.BatchStruct(table, starts, lengths, stride, batch, tokens, status))

    def write(k=P, v=P, dtype=0, **s):
        c, b = structs(**s)
        return L.enec_cache_write(C.byref(c), C.byref(b), k, 512, 128, v, 512, 128, dtype, None)

    def read(k=P, v=P, dtype=0, **s):
        c, b = structs(**s)
        return L.enec_cache_read(C.byref(c), C.byref(b), k, 512, 128, v, 512, 128, dtype, None)

    def attend(k=P, v=P, dtype=0, q_heads=8, new=1, most=500, ws=P, size=1 << 40, scale=0.1, **s):
        c, b = structs(**s)
        return L.enec_cache_attention(C.byref(c), C.byref(b), k, 1024, 128, v, 1024, 128, dtype, q_heads, new, most, scale, ws, size, None)

    for call in (write, read, attend):
        for page in (0, 1, 8, 24, 100, 512):
            assert call(page=page) == lowbit.E_BLOCK
        for dim in (0, 32, 96, 127, 512):
            assert call(dim=dim) == lowbit.E_BLOCK
        for bad in ({"codes": None}, {"v_codes": None}, {"k_scales": None}, {"v_scales": None}, {"codes": 0x1008}, {"v_codes": 0x1004},
                    {"table": None}, {"starts": None}, {"lengths": None}, {"table": 0x1002}, {"starts": ODD}, {"lengths": 0x1002}, {"status": ODD},
                    {"stride": 0}, {"heads": 0}, {"heads": 70000}, {"batch": 70000}, {"tokens": 1 << 31}, {"pages": 1 << 31}, {"k": None}, {"v": None},
                    {"k": ODD}, {"v": ODD}):
            assert call(**bad) == lowbit.E_ARG, bad
        assert call(pages=0) == call(tokens=1 << 24) == lowbit.E_ARG
        assert call(dtype=3) == call(dtype=-1) == lowbit.E_DTYPE
        assert call(batch=0) == call(tokens=0) == lowbit.OK
        assert call(batch=0, table=None, starts=None, lengths=None) == lowbit.OK
    assert write(dtype=2) == attend(dtype=2) == lowbit.E_DTYPE
    assert read(dtype=2, k=0x1002) == lowbit.E_ARG
    for bad in ({"q_heads": 0}, {"q_heads": 6}, {"q_heads": 1 << 20}, {"new": 0}, {"new": 1 << 31}, {"new": 1 << 20}, {"batch": 65535, "heads": 256, "q_heads": 256}, {"most": (1 << 30) + 1}):
        assert attend(**bad) == lowbit.E_ARG, bad
    for scale in (0.0, -0.1, float("nan"), float("inf")):
        assert attend(scale=scale) == lowbit.E_ARG, scale
    assert L.enec_cache_write(None, None, P, 1, 1, P, 1, 1, 0, None) == lowbit.E_ARG
    c, _ = structs()
    need = L.enec_cache_attention_workspace(C.byref(c), 3, 3, 8, 1, 100000)
    assert need > 0                                        # one long sequence is split
    assert attend(tokens=3, most=100000, ws=None, size=0) == attend(tokens=3, most=100000, size=need - 1) == attend(tokens=3, most=100000, ws=None, size=need) == lowbit.E_CAPACITY
    assert attend(tokens=3, most=100000, ws=0x1008, size=need) == lowbit.E_ARG
    assert L.enec_cache_attention_workspace(None, 3, 3, 8, 1, 100) == 0


def test_shapes_that_the_binding_refuses(lowbit):
    import torch
    bf = torch.bfloat16
    byte = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    x, codes, scales = torch.zeros(4, 200, dtype=bf), byte(6, 128), byte(6, 16)
    with pytest.raises(ValueError):
        lowbit.mx4_quantize(x, codes, scales)               # rows
    with pytest.raises(ValueError):
        lowbit.mx4_quantize(x, byte(4, 64), byte(4, 8))     # padding
    with pytest.raises(ValueError):
        lowbit.mx4_quantize(x.t(), codes, scales)           # columns apart
    with pytest.raises(ValueError):
        lowbit.mx4_dequantize(codes, scales[:, :15], torch.zeros(6, 200))
    with pytest.raises(ValueError):
        lowbit.mx4_linear(x, codes, scales, torch.zeros(4, 6))                     # another format
    with pytest.raises(ValueError):
        lowbit.mx4_linear(x, codes, scales, torch.zeros(4, 7, dtype=bf))
    with pytest.raises(ValueError):
        lowbit.mx4_matmul(byte(4, 64), byte(4, 8), codes, scales, torch.zeros(4, 6))


def test_caches_that_the_binding_refuses(lowbit):
    import torch
    byte = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError):
        lowbit.Cache(byte(4, 2, 16, 64), byte(4, 2), byte(4, 2, 16, 64), byte(4, 2))       # values not transposed
    with pytest.raises(ValueError):
        lowbit.Cache(byte(4, 2, 16, 64), byte(4, 3), byte(4, 2, 64, 16), byte(4, 2))
    c = lowbit.Cache(byte(4, 2, 16, 64), byte(4, 2), byte(4, 2, 64, 16), byte(4, 2))
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    for bad in (dict(table=i(4)), dict(starts=i(3)), dict(lengths=i(4)), dict(table=i(2, 3)), dict(starts=i(4).long()), dict(k=k[:, :1]), dict(v=k[:4]),
                dict(v=k.half()), dict(k=k[..., ::2])):
        a = dict(k=k, v=k, table=i(3, 2), starts=i(4), lengths=i(3)) | bad
        with pytest.raises(ValueError):
            lowbit.cache_write(c, a["k"], a["v"], a["table"], a["starts"], a["lengths"])
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lowbit.cache_attention(c, q, q[:4], i(3, 2), i(4), i(3), 1, 32)


def test_a_workspace_for_the_largest_attention_serves_smaller_ones(lowbit):
    """Fewer tokens can mean more splits: what is said for the largest covers them."""
    import random
    L, rng = lowbit.lib(), random.Random(5)

    def need(c, batch, tokens, q_heads, new, most):
        return L.enec_cache_attention_workspace(C.byref(c), batch, tokens, q_heads, new, most)

    shape = lambda heads, dim: lowbit.CacheStruct(P, P, P, P, 10, 64, heads, dim)  # noqa: E731
    c = shape(8, 128)
    assert need(c, 4, 128, 32, 32, 131072) <= need(c, 4, 400, 32, 100, 131072)
    assert need(c, 2, 128, 32, 64, 8192) <= need(c, 2, 300, 32, 150, 8192)
    met = 0
    for _ in range(20000):
        heads, dim, group = rng.choice((1, 2, 3, 8, 32, 300)), rng.choice((64, 128, 256)), rng.choice((1, 2, 4, 7, 16, 17, 32, 33, 40))
        c, sizes = shape(heads, dim), []
        large = (rng.randint(1, 70), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 18)))
        small = tuple(rng.randint(1, v) if rng.random() < 0.7 else v for v in large)
        tokens = large[0] * large[1] if rng.random() < 0.5 else rng.randint(1, large[0] * large[1])
        fewer = min(tokens, small[0] * small[1])
        for (batch, new, most), n in ((large, tokens), (small, fewer)):
            sizes.append(need(c, batch, n, heads * group, new, most))
        assert sizes[1] <= sizes[0] <= 35 << 20, (heads, dim, group, large, small, tokens, fewer, sizes)
        met += sizes[1] > 0
    assert met > 5000                                      # (the draw does reach calls that are split)
    # and such a workspace is large enough for the call itself: the next thing wrong with it is its address
    c, b = shape(8, 128), lowbit.BatchStruct(P, P, P, 8, 4, 128, None)
    size = need(c, 4, 400, 32, 100, 131072)
    assert L.enec_cache_attention(C.byref(c), C.byref(b), P, 4096, 128, P, 4096, 128, 0, 32, 32, 131072, 0.1, 0x1008, size, None) == lowbit.E_ARG


def test_a_workspace_for_many_rows_serves_products_of_fewer(lowbit):
    """Fewer rows can mean more splits: what is said for the most rows covers them."""
    import random
    rng = random.Random(6)
    linear, matmul = lowbit.mx4_linear_workspace, lowbit.mx4_matmul_workspace
    assert linear(115, 4285, 5818) <= linear(230, 4285, 5818) and matmul(692, 801, 10103) <= matmul(1854, 801, 10103)
    met = 0
    for _ in range(20000):
        n, k, m = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 13))
        fewer = rng.randint(1, m)
        copied = 2 * m * -(-k // 128) * 128
        assert linear(fewer, n, k) <= linear(m, n, k) <= copied + (68 << 20), (fewer, m, n, k)
        assert matmul(fewer, n, k) <= matmul(m, n, k) <= 136 << 20, (fewer, m, n, k)
        met += matmul(fewer, n, k) > 0
    assert met > 3000
    # and such a workspace is large enough for the call itself: the next thing wrong with it is its address
    L = lowbit.lib()
    assert L.enec_mx4_linear(P, 115, 5818, 0, P, P, 4285, 5818, P, 4285, 0x1008, linear(230, 4285, 5818), None) == lowbit.E_ARG
    assert L.enec_mx4_matmul(P, P, 692, P, P, 801, 10103, P, 801, 0, 0x1008, matmul(1854, 801, 10103), None) == lowbit.E_ARG


def test_types_and_places_that_the_binding_refuses(lowbit):
    """What the kernels would read as something else, or not reach at all."""
    import torch
    byte = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    c = lowbit.Cache(byte(4, 2, 16, 64), byte(4, 2), byte(4, 2, 64, 16), byte(4, 2))
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k, q = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 4, 64, dtype=torch.bfloat16)

    def calls(table, starts, lengths, status=None):
        yield lambda: lowbit.cache_write(c, k, k, table, starts, lengths, status)
        yield lambda: lowbit.cache_read(c, k, k, table, starts, lengths, status)
        yield lambda: lowbit.cache_attention(c, q, q, table, starts, lengths, 1, 32, status=status)

    good = dict(table=i(3, 2), starts=i(4), lengths=i(3))
    for name in good:
        for other in (torch.float32, torch.uint8, torch.int64):
            for call in calls(**good | {name: good[name].to(other)}):
                with pytest.raises(ValueError, match="int32"):
                    call()
    for status in (byte(4), i(0), torch.zeros(1), torch.zeros(1, dtype=torch.int64)):
        for call in calls(**good, status=status):
            with pytest.raises(ValueError, match="status"):
                call()
    for call in calls(**good):                             # all well, but in the host's memory
        with pytest.raises(ValueError, match="GPU"):
            call()
    x, codes, scales, x4 = torch.zeros(4, 200, dtype=torch.bfloat16), byte(6, 128), byte(6, 8), (byte(4, 128), byte(4, 8))
    out = torch.zeros(4, 6, dtype=torch.bfloat16)
    for call in (lambda: lowbit.mx4_quantize(x, *x4), lambda: lowbit.mx4_dequantize(*x4, x), lambda: lowbit.mx4_linear(x, codes, scales, out),
                 lambda: lowbit.mx4_matmul(*x4, codes, scales, out)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_scales_that_leave_the_range_of_32_bits_are_refused(lowbit):
    """The kernels have the scale times log2 e, which has to be finite too."""
    L = lowbit.lib()
    c, b = lowbit.CacheStruct(P, P, P, P, 10, 64, 4, 128), lowbit.BatchStruct(P, P, P, 8, 3, 5, None)
    call = lambda scale, ws: L.enec_cache_attention(C.byref(c), C.byref(b), P, 1024, 128, P, 1024, 128, 0, 8, 1, 1 << 20, scale, ws, 1 << 40, None)  # noqa: E731
    for scale in (3e38, 2.0 ** 127 * 1.5, 2.4e38):
        assert call(scale, P) == lowbit.E_ARG, scale
    need = L.enec_cache_attention_workspace(C.byref(c), 3, 5, 8, 1, 1 << 20)
    assert need > 0                                        # the next thing wrong with these is that there is no workspace
    for scale in (2.0 ** 127, 1e-40, 0.1):
        assert call(scale, None) == lowbit.E_CAPACITY, scale
