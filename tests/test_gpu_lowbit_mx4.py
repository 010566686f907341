"""Matrices in microscaled 4-bit floating point and their products on the GPU against plain forms in 64 bits."""
import numpy as np
import pytest

import lowbit_plain as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def lowbit():
    assert torch.cuda.is_available(), "needs the MI355X"
    from paper_2604_03298_amd import lowbit as module
    module.lib()
    return module


def on_gpu(x, stride=None, offset=0):
    """x on the GPU, its rows `stride` elements apart in a buffer of NaN that begins `offset` elements late."""
    rows, cols = x.shape
    stride = stride or cols
    buf = torch.full((offset + max(1, rows) * stride + 64,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[offset:offset + rows * stride].view(rows, stride)[:, :cols]
    view.copy_(x)
    return view


def special_rows(cols, dtype):
    """Rows whose blocks are at the format's edges."""
    g = torch.Generator().manual_seed(cols)
    top = torch.finfo(dtype)
    x = torch.randn(12, cols, generator=g)
    x[1] = 0
    x[2] = -0.0
    x[3, cols // 2] = float("nan")
    x[4, 0], x[5, cols - 1] = float("inf"), float("-inf")
    x[6] *= top.max / 8
    x[6, cols // 3] = top.max
    x[7] *= top.tiny * top.eps
    x[8] *= top.tiny
    x[9] = (torch.arange(cols) % 57 - 28) / 4.0           # every tie
    x[10] = torch.tensor([6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25]).repeat(cols // 8 + 1)[:cols] * 2.0 ** (torch.arange(cols) // 32 % 9 - 4)
    x[11] = -x[10] * 1.0078125
    return x.to(dtype)


def same_bits(got, want):
    """Equal as bit patterns, any NaN for a NaN."""
    view = torch.int32 if got.dtype == torch.float32 else torch.int16
    got, want = got.cpu(), want.cpu()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got.contiguous().view(view)[~nan], want.contiguous().view(view)[~nan])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,stride,offset", [(1, 1, 0), (7, 9, 1), (31, 31, 3), (32, 32, 0), (33, 40, 5), (127, 127, 1), (128, 128, 0), (129, 131, 7), (1000, 1000, 0), (4096, 4099, 1)])
def test_codes_and_scales_are_those_of_the_definition(lowbit, dtype, cols, stride, offset):
    x = special_rows(cols, dtype)
    src = on_gpu(x, stride, offset)
    codes, scales = lowbit.mx4_empty(x.shape[0], cols)
    codes.fill_(0xA5), scales.fill_(0xA5)
    assert lowbit.mx4_quantize(src, codes, scales) == lowbit.OK
    want_codes, want_scales = plain.mx4_encode(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    got = codes.cpu().numpy()
    # the sign of a zero inside a block of zeros is kept too
    assert np.array_equal(got, want_codes)
    for out_dtype in DTYPES:
        out = on_gpu(torch.full((x.shape[0], cols), 7.0, dtype=out_dtype), stride, offset)
        assert lowbit.mx4_dequantize(codes, scales, out) == lowbit.OK
        same_bits(out, plain.rounded(plain.mx4_decode(want_codes, want_scales, cols), out_dtype))


@pytest.mark.parametrize("dtype", DTYPES)
def test_every_code_with_every_scale_reads_back(lowbit, dtype):
    codes = np.tile((np.arange(64) * 0x11 + 0x10 * (np.arange(64) // 16)).astype(np.uint8), (64, 1))
    scales = np.arange(256, dtype=np.uint8).reshape(64, 4)
    out = torch.empty(64, 128, dtype=dtype, device="cuda")
    assert lowbit.mx4_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out) == lowbit.OK
    want = plain.mx4_decode(codes, scales, 128)
    with np.errstate(over="ignore"):
        same_bits(out, plain.rounded(want, dtype))


def test_many_rows_and_few_columns(lowbit):
    x = torch.randn(70001, 3, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    codes, scales = lowbit.mx4_empty(70001, 3)
    assert lowbit.mx4_quantize(x.cuda(), codes, scales) == lowbit.OK
    at = np.r_[0:50, 35000:35050, 69951:70001]
    want_codes, want_scales = plain.mx4_encode(x[at].double().numpy())
    assert np.array_equal(codes.cpu().numpy()[at], want_codes) and np.array_equal(scales.cpu().numpy()[at], want_scales)
    back = torch.empty_like(x, device="cuda")
    assert lowbit.mx4_dequantize(codes, scales, back) == lowbit.OK
    same_bits(back[at], plain.rounded(plain.mx4_decode(want_codes, want_scales, 3), x.dtype))


# ---- products -----------------------------------------------------------------------

def weights(n, k, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(n, k, generator=g) * torch.exp(2 * torch.randn(n, 1, generator=g)) * 0.02
    return plain.mx4_encode(w.double().numpy())


def close(got, x, w, dtype):
    want = x @ w.T
    got = got.double().cpu().numpy()
    off = np.abs(got - want) - plain.product_bound(x, w, want, dtype)
    assert np.isfinite(got).all() and off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))


def space(nbytes):
    return torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda") if nbytes else None       # NaN, were it read unwritten


SHAPES = [(1, 1, 1), (1, 16, 32), (1, 100, 129), (2, 5, 31), (3, 257, 512), (15, 33, 513), (16, 64, 1000), (17, 48, 2047), (31, 300, 256),
          (33, 17, 640), (64, 130, 1023), (65, 257, 384), (100, 64, 4096), (130, 515, 1536), (257, 129, 255), (300, 1000, 130), (1, 4099, 2048),
          (5, 2050, 8192), (515, 770, 1025)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_with_16_bit_activations(lowbit, m, n, k, dtype):
    codes, scales = weights(n, k, m + n + k)
    x = (torch.randn(m, k, generator=torch.Generator().manual_seed(k)) * 2).to(dtype)
    odd = m % 2                                          # odd strides and places for some, aligned ones for others
    src = on_gpu(x, k + 3 if odd else -(-k // 8) * 8, 1 if odd else 0)
    out = on_gpu(torch.full((m, n), float("nan"), dtype=dtype), n + 1 if odd else -(-n // 8) * 8, 1 if odd else 0)
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    assert lowbit.mx4_linear(src, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out, ws) == lowbit.OK
    close(out, x.double().numpy(), plain.mx4_decode(codes, scales, k), dtype)
    if odd:                                               # nothing beside the rows is touched
        beside = out.as_strided((m, 1), (n + 1, 1), out.storage_offset() + n)
        assert torch.isnan(beside).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_with_both_in_4_bits(lowbit, m, n, k, dtype):
    codes, scales = weights(n, k, m + n + k)
    x_codes, x_scales = weights(m, k, 7)
    out = on_gpu(torch.full((m, n), float("nan"), dtype=dtype), n + 3, 1)
    ws = space(lowbit.mx4_matmul_workspace(m, n, k))
    gpu = [torch.from_numpy(t).cuda() for t in (x_codes, x_scales, codes, scales)]
    assert lowbit.mx4_matmul(*gpu, out, ws) == lowbit.OK
    close(out, plain.mx4_decode(x_codes, x_scales, k), plain.mx4_decode(codes, scales, k), dtype)
    assert torch.isnan(out.as_strided((m, 3), (n + 3, 1), out.storage_offset() + n)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m", [1, 20, 150])
def test_scales_at_the_format_s_ends(lowbit, m, dtype):
    """Weights far outside fp16's range, times activations that bring the result back into it."""
    n, k = 40, 256
    codes, scales = weights(n, k, 3)
    scales = np.where(np.arange(n)[:, None] % 2, 107, 141).astype(np.uint8) + (np.arange(k // 32) % 3).astype(np.uint8)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(2)).to(dtype)
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    x[:, 1::2] *= 2.0 ** -13
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    codes[1 - np.arange(n) % 2 == 1] &= 0xF0            # the large rows meet the small activations only
    assert lowbit.mx4_linear(x.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out, ws) == lowbit.OK
    close(out, x.double().numpy(), plain.mx4_decode(codes, scales, k), dtype)


@pytest.mark.parametrize("m", [1, 20, 150])
def test_a_bad_block_stays_in_its_row(lowbit, m):
    n, k = 70, 300
    codes, scales = weights(n, k, 4)
    scales[5, 2] = scales[69, 9] = 255
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(5)).to(torch.float16)
    x[m // 2, 7] = float("inf")
    x[0, 299] = float("nan")
    out = torch.empty(m, n, dtype=torch.float16, device="cuda")
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    assert lowbit.mx4_linear(x.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out, ws) == lowbit.OK
    w = plain.mx4_decode(codes, scales, k)
    with np.errstate(invalid="ignore"):
        want = torch.from_numpy(x.double().numpy() @ w.T)
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    # both in 4 bits
    x_codes, x_scales = weights(m, k, 6)
    x_scales[0, 1] = 255
    full = torch.empty(m, n, device="cuda")
    ws = space(lowbit.mx4_matmul_workspace(m, n, k))
    assert lowbit.mx4_matmul(*[torch.from_numpy(t).cuda() for t in (x_codes, x_scales, codes, scales)], full, ws) == lowbit.OK
    bad = np.zeros((m, n), dtype=bool)
    bad[0], bad[:, 5], bad[:, 69] = True, True, True
    assert np.array_equal(torch.isnan(full).cpu().numpy(), bad)


def test_nothing_to_sum_and_nothing_to_do(lowbit):
    out = torch.full((3, 5), 7.0, dtype=torch.bfloat16, device="cuda")
    codes, scales = lowbit.mx4_empty(5, 0)
    x = torch.empty(3, 0, dtype=torch.bfloat16, device="cuda")
    assert lowbit.mx4_linear(x, codes, scales, out, space(lowbit.mx4_linear_workspace(3, 5, 0))) == lowbit.OK
    assert torch.equal(out, torch.zeros_like(out))
    out.fill_(7)
    x_codes, x_scales = lowbit.mx4_empty(3, 0)
    assert lowbit.mx4_matmul(x_codes, x_scales, codes, scales, out, space(lowbit.mx4_matmul_workspace(3, 5, 0))) == lowbit.OK
    assert torch.equal(out, torch.zeros_like(out))
    codes, scales = lowbit.mx4_empty(5, 64)
    assert lowbit.mx4_linear(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), codes, scales, torch.empty(0, 5, dtype=torch.bfloat16, device="cuda"),
                             space(lowbit.mx4_linear_workspace(0, 5, 64))) == lowbit.OK
    codes, scales = lowbit.mx4_empty(0, 64)
    assert lowbit.mx4_quantize(torch.empty(0, 64, device="cuda"), codes, scales) == lowbit.OK


@pytest.mark.parametrize("m", [1, 40])
def test_weights_of_more_than_4_gib(lowbit, m):
    n, k = 1 << 20, 8448
    codes, scales = lowbit.mx4_empty(n, k)
    codes.zero_(), scales.fill_(127)
    few, few_scales = weights(32, k, 8)
    codes[-32:], scales[-32:] = torch.from_numpy(few).cuda(), torch.from_numpy(few_scales).cuda()
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    assert lowbit.mx4_linear(x.cuda(), codes, scales, out, ws) == lowbit.OK
    close(out[:, -32:], x.double().numpy(), plain.mx4_decode(few, few_scales, k), torch.bfloat16)
    assert not out[:, :-32].any()
    x_codes, x_scales = weights(m, k, 10)
    ws = space(lowbit.mx4_matmul_workspace(m, n, k))
    assert lowbit.mx4_matmul(torch.from_numpy(x_codes).cuda(), torch.from_numpy(x_scales).cuda(), codes, scales, out, ws) == lowbit.OK
    close(out[:, -32:], plain.mx4_decode(x_codes, x_scales, k), plain.mx4_decode(few, few_scales, k), torch.bfloat16)
    assert not out[:, :-32].any()


def test_another_stream_and_a_graph_give_the_same(lowbit):
    """A layer's chain (quantise, both products, back) on a side stream, then captured and replayed on other inputs."""
    m, n, k = 40, 300, 1000
    g = torch.Generator().manual_seed(11)
    w = (torch.randn(n, k, generator=g) * 0.02).to(torch.bfloat16).cuda()
    xs = [torch.randn(m, k, generator=g).to(torch.bfloat16).cuda() for _ in range(3)]
    x = torch.empty_like(xs[0])
    codes, scales = lowbit.mx4_empty(n, k)
    x_codes, x_scales = lowbit.mx4_empty(m, k)
    y, z, back = (torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), torch.empty(m, n, device="cuda"), torch.empty_like(w))
    ws = torch.empty(max(16, lowbit.mx4_linear_workspace(m, n, k), lowbit.mx4_matmul_workspace(m, n, k)), dtype=torch.uint8, device="cuda")

    def chain(stream=None):
        assert lowbit.mx4_quantize(w, codes, scales, stream) == lowbit.OK
        assert lowbit.mx4_quantize(x, x_codes, x_scales, stream) == lowbit.OK
        assert lowbit.mx4_linear(x, codes, scales, y, ws, stream) == lowbit.OK
        assert lowbit.mx4_matmul(x_codes, x_scales, codes, scales, z, ws, stream) == lowbit.OK
        assert lowbit.mx4_dequantize(codes, scales, back, stream) == lowbit.OK

    want = []
    for v in xs:
        x.copy_(v)
        chain()
        want.append([t.clone() for t in (y, z, back)])
    side = torch.cuda.Stream()
    x.copy_(xs[1])
    y.zero_(), z.zero_(), back.zero_()
    side.wait_stream(torch.cuda.current_stream())
    chain(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((y, z, back), want[1]):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for i in (2, 0, 1, 2):
        x.copy_(xs[i])
        y.zero_(), z.zero_(), back.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, z, back), want[i]):
            assert torch.equal(a, b)


def any_codes(n, k, seed):
    """A matrix of any codes, with scales around 1 / 50: as it might come from elsewhere."""
    g = np.random.default_rng(seed)
    padded = -(-k // 128) * 128
    codes = g.integers(0, 256, (n, padded // 2), dtype=np.uint8)
    for c in range(k, padded):                            # padding is zeros
        codes[:, c // 2] &= 0xF0 if c % 2 == 0 else 0x0F
    return codes, g.integers(118, 125, (n, padded // 32), dtype=np.uint8)


# ragged sizes that are large enough, in one direction or another, for large tiles and for columns that are split over workgroups
LARGE = [(1000, 4100, 300), (2100, 5000, 129), (700, 8200, 200), (40, 9000, 1200), (300, 5000, 1200), (3, 20, 8100), (20, 1030, 16380), (70, 500, 16380),
         (40, 1030, 16380), (130, 5000, 16380), (300, 5000, 16380), (300, 2050, 40000), (20, 1030, 40000),
         (2000, 4090, 130), (500, 2050, 1300), (700, 2050, 1300), (300, 500, 16380), (500, 1030, 8100), (500, 4090, 130), (130, 8100, 130)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k", LARGE)
def test_large_products_with_16_bit_activations(lowbit, m, n, k, dtype):
    codes, scales = any_codes(n, k, m + n + k)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(k)).to(dtype)
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    gpu = [torch.from_numpy(t).cuda() for t in (codes, scales)]
    w = plain.mx4_decode(codes, scales, k)
    for src in (x.cuda(), on_gpu(x, k + 1, 1)):
        out.fill_(float("nan"))
        assert lowbit.mx4_linear(src, *gpu, out, ws) == lowbit.OK
        close(out, x.double().numpy(), w, dtype)


@pytest.mark.parametrize("m,n,k", LARGE + [(2050, 4097, 130)])
def test_large_products_with_both_in_4_bits(lowbit, m, n, k):
    codes, scales = any_codes(n, k, m + n + k)
    x_codes, x_scales = any_codes(m, k, 8)
    out = torch.full((m, n), float("nan"), device="cuda")
    ws = space(lowbit.mx4_matmul_workspace(m, n, k))
    gpu = [torch.from_numpy(t).cuda() for t in (x_codes, x_scales, codes, scales)]
    assert lowbit.mx4_matmul(*gpu, out, ws) == lowbit.OK
    close(out, plain.mx4_decode(x_codes, x_scales, k), plain.mx4_decode(codes, scales, k), torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m", [1, 30, 50, 600])
def test_least_and_largest_activations(lowbit, m, dtype):
    """Values of the format's smallest exponents are not lost: beside weights that bring them back, and alone."""
    n, k = 1030, 256
    codes, scales = any_codes(n, k, 9)
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(10)).double()
    x[:, ::3] *= 2.0 ** -22
    x[:, 1::3] *= 2.0 ** 13
    x = x.to(dtype)
    x[:, 128:] = x[:, 128:] * 2.0 ** -10
    scales[::2] += 20
    codes[1::2, :32] = 0
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    w = plain.mx4_decode(codes, scales, k)
    if dtype == torch.float16:                            # results within the format
        x[:, :128] = x[:, :128] * 2.0 ** -14
        w = plain.mx4_decode(codes, scales, k)
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    assert lowbit.mx4_linear(x.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out, ws) == lowbit.OK
    got, xx = out.double().cpu().numpy(), x.double().numpy()
    want = xx @ w.T
    fits = np.abs(want) < 60000 if dtype == torch.float16 else np.isfinite(want)
    off = np.abs(got - want) - plain.product_bound(xx, w, want, dtype)
    assert fits.mean() > 0.4 and (off[fits] <= 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k", [(1, 70, 300), (20, 70, 300), (50, 70, 300), (150, 70, 300), (300, 600, 300), (3, 20, 8100), (600, 1030, 256)])
def test_blocks_without_values_make_their_row_of_weights_nan(lowbit, m, n, k, dtype):
    """A scale byte of 255, whatever the codes: of the first block and of the last, of one row and of a tile's all; and only those rows."""
    codes, scales = weights(n, k, 4)
    blocks = -(-k // 32)
    bad = [5, n - 1] + list(range(16, min(32, n)))
    scales[5, 0] = scales[n - 1, blocks - 1] = 255
    scales[16:32, blocks // 2] = 255
    x = (torch.randn(m, k, generator=torch.Generator().manual_seed(5)).abs() + 0.1).to(dtype)
    want = x.double().numpy() @ plain.mx4_decode(np.where(scales.repeat(16, 1) == 255, 0, codes).astype(np.uint8), np.where(scales == 255, 0, scales).astype(np.uint8), k).T
    bound = plain.product_bound(x.double().numpy(), np.abs(plain.mx4_decode(codes, np.where(scales == 255, 0, scales).astype(np.uint8), k)), want, dtype)
    ok = np.ones(n, dtype=bool)
    ok[bad] = False
    for fill in (0x00, 0x22, 0x77, 0xAA, 0xF2, None):      # zeros, ones, sixes, minus ones, mixed signs, any
        held = codes if fill is None else np.where(scales.repeat(16, 1) == 255, fill, codes).astype(np.uint8)
        out = torch.empty(m, n, dtype=dtype, device="cuda")
        ws = space(lowbit.mx4_linear_workspace(m, n, k))
        assert lowbit.mx4_linear(x.cuda(), torch.from_numpy(held).cuda(), torch.from_numpy(scales).cuda(), out, ws) == lowbit.OK
        got = out.double().cpu().numpy()
        assert np.isnan(got[:, ~ok]).all(), (fill, np.isnan(got[:, ~ok]).mean())
        assert np.isfinite(got[:, ok]).all() and (np.abs(got - want)[:, ok] <= bound[:, ok]).all(), fill


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m", [1, 20, 50, 150, 600])
def test_activations_that_are_not_finite_reach_their_own_row_only(lowbit, m, dtype):
    n, k = 1030, 300
    codes, scales = weights(n, k, 14)
    codes[7] = 0                                           # infinity times zero
    x = torch.randn(m, k, generator=torch.Generator().manual_seed(15)).to(dtype)
    x[m // 2, 7] = float("inf")
    if m > 1:
        x[0, 299], x[m - 1, 0] = float("nan"), float("-inf")
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    ws = space(lowbit.mx4_linear_workspace(m, n, k))
    assert lowbit.mx4_linear(x.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out, ws) == lowbit.OK
    with np.errstate(invalid="ignore"):
        want = torch.from_numpy(x.double().numpy() @ plain.mx4_decode(codes, scales, k).T)
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])


@pytest.mark.parametrize("m", [1, 20, 150, 600])
def test_blocks_without_values_on_either_side_of_a_4_bit_product(lowbit, m):
    n, k = 600, 300
    codes, scales = weights(n, k, 4)
    x_codes, x_scales = weights(m, k, 6)
    scales[5, 0] = scales[n - 1, 9] = x_scales[m // 2, 1] = 255
    bad = np.zeros((m, n), dtype=bool)
    bad[m // 2], bad[:, 5], bad[:, n - 1] = True, True, True
    for fill in (0x00, 0x22, 0xF2):
        held, x_held = (np.where(s.repeat(16, 1) == 255, fill, c).astype(np.uint8) for c, s in ((codes, scales), (x_codes, x_scales)))
        out = torch.empty(m, n, device="cuda")
        ws = space(lowbit.mx4_matmul_workspace(m, n, k))
        assert lowbit.mx4_matmul(*[torch.from_numpy(t).cuda() for t in (x_held, x_scales, held, scales)], out, ws) == lowbit.OK
        assert np.array_equal(torch.isnan(out).cpu().numpy(), bad), fill
