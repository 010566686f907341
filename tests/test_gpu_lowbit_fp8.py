"""Matrices in 8 bits with a scale for each block of 128, and their products, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from decoding_plain import fp8_decode, fp8_encode, products_bound
from lowbit_plain import rounded

pytestmark = pytest.mark.gpu
FORMATS = [torch.bfloat16, torch.float16, torch.float32]
OK = 0


@pytest.fixture(scope="module")
def lowbit():
    from paper_2604_03298_amd import lowbit as module
    module.lib()
    return module


def values(rng, rows, cols, dtype):
    x = rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-3, 3, (rows, 1)))
    x[rng.random((rows, cols)) < 0.01] *= 30
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def doubles(t):
    return t.float().numpy().astype(np.float64)


def packed(lowbit, rng, rows, cols):
    codes, scales = fp8_encode(doubles(values(rng, rows, cols, torch.bfloat16)))
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), fp8_decode(codes, scales, cols)


def quantized(lowbit, x, cols=None):
    codes, scales = lowbit.fp8_empty(*x.shape)
    codes.fill_(0xAA), scales.fill_(0xAA)
    assert lowbit.fp8_quantize(x, codes, scales) == OK
    torch.cuda.synchronize()
    return codes.cpu().numpy(), scales.cpu().numpy()


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 127), (3, 128), (5, 129), (7, 1000), (33, 513), (2, 5001), (70, 384)])
def test_codes_and_scales(lowbit, rows, cols, dtype):
    rng = np.random.default_rng(rows * 10000 + cols)
    x = values(rng, rows, cols, dtype)
    x[0, cols // 2] = 0
    if rows > 2:
        x[1], x[2, ::2] = 0, -0.0
    codes, scales = quantized(lowbit, x.cuda())
    want, bytes_ = fp8_encode(doubles(x))
    assert np.array_equal(scales, bytes_) and np.array_equal(codes, want)


def test_values_at_the_formats_ends(lowbit):
    """Borders of the scale (448 2^e and just above), the smallest and largest values, ties between codes, values that are none."""
    blocks = []
    for e in (-149, -140, -133, -127, -120, -20, 0, 3, 100, 119):
        for a in (448.0, 448.0 * (1 + 2.0 ** -23), 447.9, 256.0, 2.0 ** -9, 1.0):
            v = np.zeros(128)
            v[0] = a * 2.0 ** e
            v[1:100] = np.random.default_rng(e + 200).uniform(-1, 1, 99) * v[0]
            v[100:110] = v[0] * np.array([17, 19, 21, 23, 25, 27, 29, 31, 33, 35]) / 512
            blocks.append(v)
    v = np.zeros(128)
    v[:3] = 3.4028234663852886e38, -3.4028234663852886e38, 2.0 ** -149
    blocks.append(v)
    for bad in (np.nan, np.inf, -np.inf):
        v = np.ones(128)
        v[77] = bad
        blocks.append(v)
    with np.errstate(over="ignore"):
        x = np.stack(blocks).astype(np.float32)
    assert np.isfinite(x[:-3]).all()
    codes, scales = quantized(lowbit, torch.from_numpy(x).cuda())
    want, bytes_ = fp8_encode(x.astype(np.float64))
    assert np.array_equal(scales, bytes_) and np.array_equal(codes, want)
    assert (scales[-3:, 0] == 255).all() and (codes[-3:] == 0).all()


def test_rows_apart_and_at_odd_addresses(lowbit):
    rng = np.random.default_rng(3)
    for dtype in FORMATS:
        held = values(rng, 9, 400, dtype).cuda().reshape(-1)
        x = held[1:1 + 8 * 399].as_strided((8, 301), (399, 1), 1)
        codes, scales = quantized(lowbit, x)
        want, bytes_ = fp8_encode(doubles(x.cpu()))
        assert np.array_equal(scales, bytes_) and np.array_equal(codes, want)
        out = torch.full((9 * 400,), 7.0, dtype=dtype, device="cuda")
        back = out.as_strided((8, 301), (399, 1), 1)
        assert lowbit.fp8_dequantize(torch.from_numpy(want).cuda(), torch.from_numpy(bytes_).cuda(), back) == OK
        torch.cuda.synchronize()
        assert torch.equal(back.cpu(), rounded(fp8_decode(want, bytes_, 301), dtype))
        out = out.cpu()
        back = out.as_strided((8, 301), (399, 1), 1)
        back.fill_(7.0)
        assert (out == 7).all()                             # nothing between the rows was written


@pytest.mark.parametrize("dtype", FORMATS)
def test_a_large_matrix_as_its_parts(lowbit, dtype):
    """A matrix of more than 2^25 values, whose threads have more of them, and its rows in two calls."""
    rows, cols = 8201, 4203
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    x[5, 7], x[8200, 4202], x[4100, :128] = float("nan"), float("-inf"), 0
    whole, parts = lowbit.fp8_empty(rows, cols), lowbit.fp8_empty(rows, cols)
    for t in whole + parts:
        t.fill_(77)
    assert lowbit.fp8_quantize(x, *whole) == OK
    for part in (slice(0, 4000), slice(4000, rows)):
        assert lowbit.fp8_quantize(x[part], *(t[part] for t in parts)) == OK
    assert all(torch.equal(a, b) for a, b in zip(whole, parts))


@pytest.mark.parametrize("dtype", FORMATS)
def test_every_code_and_scale_back(lowbit, dtype):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.zeros((256, 4), dtype=np.uint8)
    scales[:, 0] = scales[:, 1] = np.arange(256)
    out = torch.empty(256, 256, dtype=dtype, device="cuda")
    assert lowbit.fp8_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out) == OK
    with np.errstate(over="ignore"):
        want = rounded(fp8_decode(codes, scales, 256), dtype)
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=5.0), torch.nan_to_num(want, nan=5.0))


def check(out, x, w, dtype):
    y, got = x @ w.T, doubles(out.cpu())
    bound = products_bound(x, w, y, dtype)
    # fp16 ends at 65504: from half a step above on, 65520, the nearest value is an infinity
    over = (np.abs(y) + bound >= 65520) & (got == np.copysign(np.inf, y)) if dtype == torch.float16 else False
    assert ((np.abs(got - y) <= bound) | over).all()


PRODUCTS = [(1, 16, 128), (1, 1, 1), (2, 33, 100), (1, 700, 2047), (7, 1001, 512), (15, 64, 4096), (16, 131, 5000), (17, 64, 130), (31, 200, 640), (33, 300, 1000),
            (64, 257, 900), (65, 130, 1280), (100, 500, 2049), (128, 128, 128), (129, 129, 257), (200, 300, 1100), (257, 513, 700), (300, 1000, 300)]


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("m, n, k", PRODUCTS)
def test_products_of_codes(lowbit, m, n, k, dtype):
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    xc, xs, x = packed(lowbit, rng, m, k)
    wc, ws, w = packed(lowbit, rng, n, k)
    held = torch.full((m, n + 5), 7.0, dtype=dtype, device="cuda")
    space = torch.empty(lowbit.fp8_matmul_workspace(m, n, xc.shape[1]) + 16, dtype=torch.uint8, device="cuda")
    assert lowbit.fp8_matmul(xc, xs, wc, ws, held[:, 3:3 + n], space) == OK
    torch.cuda.synchronize()
    check(held[:, 3:3 + n], x, w, dtype)
    assert (held[:, :3] == 7).all() and (held[:, 3 + n:] == 7).all()


@pytest.mark.parametrize("dtype", FORMATS[:2])
@pytest.mark.parametrize("m, n, k", PRODUCTS)
def test_products_of_values(lowbit, m, n, k, dtype):
    rng = np.random.default_rng(m * 5 + n + k)
    held = values(rng, m, k + 3, dtype)
    wc, ws, w = packed(lowbit, rng, n, k)
    out = torch.full((m + 1, n), 7.0, dtype=dtype, device="cuda")
    space = torch.empty(lowbit.fp8_linear_workspace(m, n, k) + 16, dtype=torch.uint8, device="cuda")
    assert lowbit.fp8_linear(held.cuda()[:, 1:1 + k], wc, ws, out[:m], space) == OK
    torch.cuda.synchronize()
    check(out[:m], fp8_decode(*fp8_encode(doubles(held[:, 1:1 + k])), k), w, dtype)
    assert (out[m] == 7).all()


@pytest.mark.parametrize("sizes", [((1, 5000, 16384), (16, 300, 30000), (40, 600, 16384), (96, 4096, 2560), (513, 2050, 1000), (1100, 2304, 640), (3, 70000, 257)),
                                   ((409, 21914, 787), (263, 22171, 803), (131, 22829, 794)), ((65, 17501, 782), (65, 4239, 6236), (67, 4139, 4739)),
                                   ((34, 16515, 798), (2062, 68, 4672), (2069, 65, 3561)), ((33, 8321, 813), (2118, 17, 3139), (66, 4194, 791), (1276, 17, 2435)),
                                   ((68, 17, 784), (33, 17, 4718), (65, 17, 1540), (1, 17, 17567)), ((1, 17, 4100), (17, 17, 4595), (34, 17, 4400), (2, 8200, 2047))])
def test_every_tile_and_split(lowbit, sizes):
    """Long sums and many rows, and sizes at which each tile, alone and with splits of the columns, and each kernel for few tokens is the one that is chosen; compared in
    64 bits on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for m, n, k in sizes:
        x, w = (torch.randn(r, k, generator=g, device="cuda").to(torch.bfloat16) for r in (m, n))
        xc, xs = lowbit.fp8_empty(m, k)
        wc, ws = lowbit.fp8_empty(n, k)
        assert lowbit.fp8_quantize(x, xc, xs) == lowbit.fp8_quantize(w, wc, ws) == OK
        xv, wv = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
        assert lowbit.fp8_dequantize(xc, xs, xv) == lowbit.fp8_dequantize(wc, ws, wv) == OK
        y, most = xv.double() @ wv.double().t().contiguous(), xv.double().abs() @ wv.double().abs().t().contiguous()
        for dtype in (torch.float32, torch.bfloat16):
            out = torch.empty(m, n, dtype=dtype, device="cuda")
            space = torch.empty(max(lowbit.fp8_linear_workspace(m, n, k), lowbit.fp8_matmul_workspace(m, n, k), 16), dtype=torch.uint8, device="cuda")
            calls = [lambda: lowbit.fp8_matmul(xc, xs, wc, ws, out, space)]
            if dtype == torch.bfloat16:
                calls.append(lambda: lowbit.fp8_linear(x, wc, ws, out, space))
            for call in calls:
                out.fill_(7.0)
                assert call() == OK
                # (of products_bound's last term an upper bound: the largest product of eight columns is at most the sum of all eight)
                bound = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * y.abs() + ((k + 8) * 2.0 ** -23 + (7 * 2.0 ** -13 if dtype == torch.bfloat16 else 0)) * most
                assert ((out.double() - y).abs() <= bound).all(), (m, n, k, dtype)


@pytest.mark.parametrize("m", [1, 5, 40, 150])
def test_blocks_without_values(lowbit, m):
    """A NaN or an infinity makes the sums that read its block NaN, and no others."""
    rng = np.random.default_rng(m)
    n, k = 70, 600
    x, w = values(rng, m, k, torch.bfloat16), values(rng, n, k, torch.bfloat16)
    x[m // 2, 300], w[13, 599], w[14, 0] = float("nan"), float("inf"), float("-inf")
    wc, ws = lowbit.fp8_empty(n, k)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    space = torch.empty(lowbit.fp8_linear_workspace(m, n, k) + 16, dtype=torch.uint8, device="cuda")
    assert lowbit.fp8_quantize(w.cuda(), wc, ws) == OK and lowbit.fp8_linear(x.cuda(), wc, ws, out, space) == OK
    want = torch.zeros(m, n, dtype=torch.bool)
    want[m // 2], want[:, 13], want[:, 14] = True, True, True
    assert torch.equal(torch.isnan(out).cpu(), want)


def test_no_columns_and_no_rows(lowbit):
    for dtype in FORMATS:
        for m, n in ((3, 5), (20, 301)):
            out = torch.full((m, n), 7.0, dtype=dtype, device="cuda")
            assert lowbit.fp8_matmul(*lowbit.fp8_empty(m, 0), *lowbit.fp8_empty(n, 0), out) == OK
            assert (out == 0).all()
    out = torch.empty(0, 5, dtype=torch.bfloat16, device="cuda")
    assert lowbit.fp8_linear(torch.empty(0, 300, dtype=torch.bfloat16, device="cuda"), *lowbit.fp8_empty(5, 300), out) == OK


def test_one_piece_of_memory_serves_fewer_rows(lowbit):
    rng = np.random.default_rng(8)
    n, k = 600, 8192
    wc, ws, w = packed(lowbit, rng, n, k)
    space = torch.empty(lowbit.fp8_linear_workspace(300, n, k), dtype=torch.uint8, device="cuda")
    for m in (1, 3, 16, 17, 32, 63, 64, 65, 100, 129, 256, 300):
        assert lowbit.fp8_linear_workspace(m, n, k) <= space.numel() and lowbit.fp8_matmul_workspace(m, n, k) <= lowbit.fp8_matmul_workspace(300, n, k)
        x = values(rng, m, k, torch.bfloat16)
        out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        assert lowbit.fp8_linear(x.cuda(), wc, ws, out, space) == OK
        check(out, fp8_decode(*fp8_encode(doubles(x)), k), w, torch.bfloat16)


@pytest.mark.parametrize("m", [1, 24, 300])
def test_captured_and_replayed(lowbit, m):
    rng = np.random.default_rng(4)
    n, k = 500, 4096
    wc, ws, w = packed(lowbit, rng, n, k)
    x, out = torch.empty(m, k, dtype=torch.bfloat16, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    space = torch.empty(lowbit.fp8_linear_workspace(m, n, k) + 16, dtype=torch.uint8, device="cuda")
    x.copy_(values(rng, m, k, torch.bfloat16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert lowbit.fp8_linear(x, wc, ws, out, space) == OK
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert lowbit.fp8_linear(x, wc, ws, out, space) == OK
    for _ in range(3):
        x.copy_(values(rng, m, k, torch.bfloat16))
        out.fill_(7.0)
        graph.replay()
        eager = torch.empty_like(out)
        torch.cuda.synchronize()
        assert lowbit.fp8_linear(x, wc, ws, eager, space) == OK
        assert torch.equal(out, eager)
        check(out, fp8_decode(*fp8_encode(doubles(x.cpu())), k), w, torch.bfloat16)
