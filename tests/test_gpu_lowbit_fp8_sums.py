"""Sums of products of 8-bit matrices, with whole numbers as values, so that every sum is exact in 32 bits and y is known to the last bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
OK = 0


@pytest.fixture(scope="module")
def lowbit():
    from paper_2604_03298_amd import lowbit as module
    module.lib()
    return module


def whole_numbers(g, rows, cols):
    return torch.randint(-7, 8, (rows, cols), generator=g, device="cuda").float()


def products(lowbit, x, w, dtype):
    """y of every call that gives it in this format."""
    (m, k), n = x.shape, w.shape[0]
    xc, xs, wc, ws = *lowbit.fp8_empty(m, k), *lowbit.fp8_empty(n, k)
    assert lowbit.fp8_quantize(x, xc, xs) == lowbit.fp8_quantize(w, wc, ws) == OK
    space = torch.empty(max(lowbit.fp8_linear_workspace(m, n, k), lowbit.fp8_matmul_workspace(m, n, k), 16), dtype=torch.uint8, device="cuda")
    out = torch.full((m, n), 7.0, dtype=dtype, device="cuda")
    assert lowbit.fp8_matmul(xc, xs, wc, ws, out, space) == OK
    yield "matmul", out
    if dtype != torch.float32:
        out = torch.full((m, n), 7.0, dtype=dtype, device="cuda")
        assert lowbit.fp8_linear(x.to(dtype), wc, ws, out, space) == OK
        yield "linear", out


# every kernel for few tokens, with values brought into 8 bits inside and before, and every tile, with splits of the columns and without: test_fp8_sizes.py holds them to that
SIZES = [(1, 17, 130), (1, 64, 1000), (2, 8200, 2047), (1, 4096, 4096), (1, 17, 4100), (16, 300, 5000), (17, 17, 4595), (40, 600, 4096), (64, 257, 900), (34, 17, 4400), (100, 500, 2049), (67, 4139, 4739),
         (128, 128, 128), (409, 21914, 787), (300, 1000, 300), (513, 2050, 1000), (1100, 2304, 640), (96, 4096, 11008), (20, 700, 1500), (263, 22171, 803), (131, 22829, 794), (65, 4239, 6236),
         (2062, 68, 4672), (33, 8321, 813), (40, 600, 16384), (2118, 17, 3139), (33, 17, 4718), (1, 17, 17567), (1, 5000, 16384)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m, n, k", SIZES)
def test_every_product_counts(lowbit, m, n, k, dtype):
    """Whole numbers up to 7: sums below 2^24 and products that no instruction drops anything of, so that y is its exact value, rounded once, and a column, a block or a split that is left out
    or counted twice shows in most of y."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m * 3 + n + k)
    x, w = whole_numbers(g, m, k), whole_numbers(g, n, k)
    y = x.double() @ w.double().t().contiguous()
    for call, out in products(lowbit, x, w, dtype):
        assert torch.equal(out, y.to(dtype)), call


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("m, n, k", SIZES)
def test_large_products_that_cancel_leave_the_small_ones(lowbit, m, n, k, dtype):
    """448^2 and -448^2 among eight columns whose other products are below 50: whatever a sum of fewer bits than 32 drops beside the large ones is missing in y.  All partial sums stay below
    2^24, so that y is its exact value, rounded once."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    x, w = whole_numbers(g, m, k), whole_numbers(g, n, k)
    pairs = k // 8
    x[:, 0:8 * pairs:8], x[:, 1:8 * pairs:8] = 448, 448
    w[:, 0:8 * pairs:8], w[:, 1:8 * pairs:8] = 448, -448
    y = x.double() @ w.double().t().contiguous()
    for call, out in products(lowbit, x, w, dtype):
        assert torch.equal(out, y.to(dtype)), call
