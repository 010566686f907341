"""The paged 8-bit cache and its attention on the GPU against plain forms in 64 bits."""
import numpy as np
import pytest

import lowbit_plain as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def lowbit():
    assert torch.cuda.is_available(), "needs the MI355X"
    from paper_2604_03298_amd import lowbit as module
    module.lib()
    return module


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts_of(counts):
    return [0] + list(np.cumsum(counts))


class Both:
    """The same cache on the GPU and in its plain form, with pages in random order and rubbish in every byte that nothing was written to."""

    def __init__(self, lowbit, lengths, page, heads, dim, seed=0):
        self.lowbit, self.rng = lowbit, np.random.default_rng(seed)
        self.most = max(1, max(-(-n // page) for n in lengths))
        pages = sum(-(-n // page) for n in lengths) + 2
        order = self.rng.permutation(pages)
        self.table = np.full((len(lengths), self.most), -7, dtype=np.int32)
        at = 0
        for b, n in enumerate(lengths):
            need = -(-n // page)
            self.table[b, :need] = order[at:at + need]
            at += need
        self.cache = lowbit.Cache.empty(pages, heads, dim, page)
        for t in self.cache.tensors:
            t.copy_(torch.from_numpy(self.rng.integers(0, 256, tuple(t.shape), dtype=np.uint8)))
        self.k, self.v = plain.PlainCache(page, heads, dim), plain.PlainCache(page, heads, dim)
        self.heads, self.dim = heads, dim
        self.gpu_table = torch.from_numpy(self.table).cuda()

    def values(self, tokens, dtype, scale=1.0, layout=0):
        """Random keys or values: plain, as a slice of a wider tensor at an odd place, or with heads outermost."""
        x = torch.from_numpy(self.rng.standard_normal((tokens, self.heads, self.dim)).astype(np.float32) * scale).to(dtype)
        return x, self.laid_out(x, layout)

    def laid_out(self, x, layout):
        tokens, heads, dim = x.shape
        if layout == 1:
            buf = torch.full((tokens, heads + 1, dim + 3), float("nan"), dtype=x.dtype, device="cuda")
            out = buf[:, 1:, 1:dim + 1]
        elif layout == 2:
            out = torch.empty(heads, tokens, dim, dtype=x.dtype, device="cuda").transpose(0, 1)
        else:
            out = torch.empty(tokens, heads, dim, dtype=x.dtype, device="cuda")
        out.copy_(x)
        return out

    def write(self, counts, lengths, k, v, status=None):
        """k, v: pairs of (values, values on the GPU)."""
        starts = starts_of(counts)
        assert self.lowbit.cache_write(self.cache, k[1], v[1], self.gpu_table, ints(starts), ints(lengths), status) == self.lowbit.OK
        self.k.write(k[0].double().numpy(), self.table, starts, lengths)
        self.v.write(v[0].double().numpy(), self.table, starts, lengths)

    def fill(self, lengths, dtype, layout=0):
        n = sum(lengths)
        self.write(lengths, lengths, self.values(n, dtype, 2.0, layout), self.values(n, dtype, 1.0, layout))

    def check(self, lengths, dtype=torch.float32, layout=0):
        """Everything that is cached, read back."""
        n, starts = sum(lengths), starts_of(lengths)
        out = [self.laid_out(torch.full((n, self.heads, self.dim), 9.0, dtype=dtype), layout) for _ in range(2)]
        assert self.lowbit.cache_read(self.cache, *out, self.gpu_table, ints(starts), ints(lengths)) == self.lowbit.OK
        for got, form in zip(out, (self.k, self.v)):
            want = np.concatenate([form.read(self.table[b], n) for b, n in enumerate(lengths)])
            want = plain.rounded(want, dtype)
            assert torch.equal(torch.isnan(got).cpu(), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got).cpu(), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("page,dim,heads", [(16, 64, 3), (32, 128, 2), (64, 64, 1), (64, 128, 2), (128, 128, 1), (256, 64, 1), (16, 256, 2), (256, 256, 1)])
def test_prompts_then_single_tokens_then_a_few(lowbit, dtype, page, dim, heads):
    """Appending to pages that hold tokens: the scale grows (each step's values are larger), keeps, or the page is new."""
    first = [2 * page + 5, 1, page, 0, page - 1]
    last = [n + 1 + 3 + 2 + (page + 1) for n in first]
    c = Both(lowbit, last, page, heads, dim, seed=page + dim)
    lengths = list(first)
    c.write(first, lengths, c.values(sum(first), dtype, 1.0), c.values(sum(first), dtype, 0.5))
    c.check(lengths)
    for counts, scale, layout in (([1] * 5, 40.0, 1), ([3] * 5, 0.01, 2), ([2, 2, 2, 2, 2], 700.0, 1), ([page + 1] * 5, 1.0, 0)):
        lengths = [n + m for n, m in zip(lengths, counts)]
        c.write(counts, lengths, c.values(sum(counts), dtype, scale, layout), c.values(sum(counts), dtype, scale / 3, layout))
        c.check(lengths)
    for out, layout in ((torch.bfloat16, 1), (torch.float16, 2), (torch.float32, 1)):
        c.check(lengths, out, layout)


@pytest.mark.parametrize("dtype", HALF)
def test_values_at_the_formats_ends(lowbit, dtype):
    page, heads, dim = 32, 6, 64
    c = Both(lowbit, [40], page, heads, dim, 5)
    x = torch.randn(40, heads, dim, generator=torch.Generator().manual_seed(1))
    top = torch.finfo(dtype)
    x[:, 0] = 0                                           # zeros
    x[3, 1, 5], x[7, 1, 9], x[9, 1, 63] = float("inf"), float("-inf"), float("nan")
    x[:, 2] *= top.tiny * top.eps * 4                     # subnormal
    x[:, 3] = top.max * torch.sign(x[:, 3])               # the largest
    x[:, 4] = 448.0 * torch.sign(x[:, 4])                 # exactly the largest code ...
    x[20, 4, 1] = 448.0 * 2 if dtype == torch.bfloat16 else 449.0  # ... and one page needs more
    x[:, 5] = float("nan")
    x = x.to(dtype)
    c.write([40], [40], (x, x.cuda()), (x, x.cuda()))
    c.check([40])
    # the next token of the second page of head 0 is far larger than its zeros; the NaN of head 5 meet numbers
    y = torch.full((1, heads, dim), 100.0).to(dtype)
    c2 = Both(lowbit, [41], page, heads, dim, 6)
    c2.write([40], [40], (x, x.cuda()), (x, x.cuda()))
    c2.write([1], [41], (y, y.cuda()), (y, y.cuda()))
    c2.check([41])


def test_idle_slots_and_tokens_before_a_sequence(lowbit):
    page, heads, dim = 16, 2, 64
    lengths, counts = [5, 0, 2, 17, 0], [1, 1, 4, 1, 0]   # the second sequence is an idle slot, the third has two tokens at negative positions
    c = Both(lowbit, [20, 0, 20, 20, 0], page, heads, dim, 7)
    prior = [4, 0, 0, 16, 0]
    c.write(prior, prior, c.values(20, torch.bfloat16), c.values(20, torch.bfloat16))
    k, v = c.values(7, torch.bfloat16), c.values(7, torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = [t.clone() for t in c.cache.tensors]
    assert lowbit.cache_write(c.cache, k[1], v[1], c.gpu_table, ints(starts_of(counts)), ints(lengths), status) == lowbit.OK
    starts = starts_of(counts)
    kk, vv = k[0].double().numpy(), v[0].double().numpy()
    # the same without the tokens that have no place
    keep = [0, 4, 5, 6]
    for form, x in ((c.k, kk), (c.v, vv)):
        form.write(x[keep], c.table, starts_of([1, 0, 2, 1, 0]), lengths)
    c.check(lengths)
    assert status.item() == 0
    used = {int(c.table[b, (lengths[b] - 1) // page]) for b in (0, 2, 3)}
    for t, old in zip(c.cache.tensors, before):
        for p in range(t.shape[0]):
            if p not in used:
                assert torch.equal(t[p], old[p])
    out = [torch.full((7, heads, dim), 3.0, device="cuda") for _ in range(2)]
    assert lowbit.cache_read(c.cache, *out, c.gpu_table, ints(starts), ints(lengths), status) == lowbit.OK
    for t, form in zip(out, (c.k, c.v)):
        assert not t[[1, 2, 3]].any()
        assert np.array_equal(t[[0]].cpu().double().numpy(), form.read(c.table[0], 5)[4:])
        assert np.array_equal(t[[4, 5]].cpu().double().numpy(), form.read(c.table[2], 2))
    assert status.item() == 0


def test_what_only_the_device_can_see_is_left_out_and_told(lowbit):
    page, heads, dim = 16, 2, 64
    c = Both(lowbit, [30, 30, 30], page, heads, dim, 8)
    c.fill([30, 30, 30], torch.bfloat16)
    x = torch.randn(90, heads, dim, device="cuda").to(torch.bfloat16)
    q = torch.randn(3, 4, dim, device="cuda").to(torch.bfloat16)
    good = c.gpu_table.clone()
    pages = c.cache.n_pages

    def attend(table, starts, lengths, max_new=1, max_length=32):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 5.0)
        ws = torch.empty(max(16, lowbit.cache_attention_workspace(c.cache, 3, 3, 4, max_new, max_length)), dtype=torch.uint8, device="cuda")
        assert lowbit.cache_attention(c.cache, q, out, table, ints(starts), ints(lengths), max_new, max_length, ws, status=status) == lowbit.OK
        return out, status.item()

    want, told = attend(good, [0, 1, 2, 3], [30, 30, 30])
    assert told == 0
    # a length beyond the table, or beyond max_length
    for lengths, most in (([30, 33, 30], 40), ([30, 30, 30], 29), ([30, -1, 30], 32)):
        out, told = attend(good, [0, 1, 2, 3], lengths, max_length=most)
        assert told == lowbit.E_ARG
        for b in range(3):
            assert torch.equal(out[b], want[b]) if 0 <= lengths[b] <= min(32, most) else bool((out[b] == 5).all())
    # starts out of order, or beyond the tokens
    for starts in ([0, 2, 1, 3], [0, 1, 2, 4], [-1, 1, 2, 3]):
        assert attend(good, starts, [30, 30, 30])[1] == lowbit.E_ARG
    # more tokens than max_new
    out, told = attend(good, [0, 2, 2, 3], [30, 30, 30])
    assert told == lowbit.E_ARG and bool((out[:2] == 5).all()) and torch.equal(out[2], want[2])
    # page numbers outside the cache: their tokens are not seen
    for bad in (-1, pages, 0x7FFFFFFF):
        table = good.clone()
        table[1, 1] = bad
        out, told = attend(table, [0, 1, 2, 3], [30, 30, 30])
        assert told == lowbit.E_ARG and torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
        short, _ = attend(good, [0, 1, 2, 3], [30, 16, 30])
        assert torch.allclose(out[1].float(), short[1].float(), rtol=0.02, atol=0.02)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        before = [t.clone() for t in c.cache.tensors]
        back = [torch.full((90, heads, dim), 9.0, device="cuda") for _ in range(2)]
        assert lowbit.cache_read(c.cache, *back, table, ints([0, 30, 60, 90]), ints([30, 30, 30]), status) == lowbit.OK
        assert status.item() == lowbit.E_ARG
        for t, form in zip(back, (c.k, c.v)):
            full = np.concatenate([form.read(c.table[b], 30) for b in range(3)])
            full[46:60] = 0
            assert np.array_equal(t.cpu().double().numpy(), full)
        status.zero_()
        assert lowbit.cache_write(c.cache, x[:3], x[3:6], table, ints([0, 1, 2, 3]), ints([30, 30, 30]), status) == lowbit.OK
        assert status.item() == lowbit.E_ARG
        page = int(good[1, 1])
        for t, old in zip(c.cache.tensors, before):
            assert torch.equal(t[page], old[page])
            t.copy_(old)
    status = torch.zeros(1, dtype=torch.int32).pin_memory()          # a word in host memory is told too
    before = [t.clone() for t in c.cache.tensors]
    assert lowbit.cache_write(c.cache, x, x, good, ints([0, 30, 60, 90]), ints([33, 33, 33]), status) == lowbit.OK
    torch.cuda.synchronize()
    assert status.item() == lowbit.E_ARG
    for t, old in zip(c.cache.tensors, before):
        assert torch.equal(t, old)


# ---- attention ----------------------------------------------------------------------

def attend(c, q, counts, lengths, scale=None, layout=0, max_new=None, max_length=None):
    lowbit = c.lowbit
    src = c.laid_out(q, layout)
    out = c.laid_out(torch.full(q.shape, 77.0, dtype=q.dtype), layout)
    new, most = max_new or max(counts), max_length or max(1, max(lengths))
    need = lowbit.cache_attention_workspace(c.cache, len(counts), q.shape[0], q.shape[1], new, most)
    ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda")       # NaN, were it read unwritten
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert lowbit.cache_attention(c.cache, src, out, c.gpu_table, ints(starts_of(counts)), ints(lengths), new, most, ws, scale, status) == lowbit.OK
    assert status.item() == 0
    return out


def check_attention(c, out, q, counts, lengths, scale=None):
    scale = c.dim ** -0.5 if scale is None else scale
    starts = starts_of(counts)
    for b, n in enumerate(lengths):
        k, v = c.k.read(c.table[b], n), c.v.read(c.table[b], n)
        rows = slice(starts[b], starts[b + 1])
        want, bound = plain.attention(q[rows].double().numpy(), k, v, scale, q.dtype)
        got = out[rows].double().cpu().numpy()
        assert np.isfinite(got).all(), (b, n)
        off = np.abs(got - want) - bound
        assert off.size == 0 or off.max() <= 0, (b, n, off.max(), np.unravel_index(off.argmax(), off.shape))


CALLS = [
    # page, head_dim, heads, group, new tokens, lengths
    (64, 128, 2, 4, [1, 1, 1, 1], [1, 64, 65, 300]),
    (16, 64, 1, 1, [1] * 5, [15, 16, 17, 0, 1]),
    (32, 128, 2, 8, [1, 1], [33, 700]),
    (64, 256, 1, 5, [1, 1, 1], [2, 129, 640]),
    (128, 64, 2, 3, [1], [1700]),
    (16, 128, 1, 16, [1, 1], [5, 1100]),
    (64, 128, 1, 40, [1, 1], [63, 500]),                  # more rows than one tile
    (64, 128, 2, 4, [3, 1, 0, 5], [3, 100, 50, 260]),     # a few tokens each, none
    (32, 64, 2, 2, [7, 40], [7, 333]),
    (64, 128, 2, 1, [130, 64, 1], [130, 200, 64]),        # prompts, one behind a cached beginning
    (16, 128, 1, 5, [77, 33], [77, 190]),
    (64, 64, 1, 8, [150], [150]),
    (16, 256, 1, 2, [70, 10], [101, 10]),
    (256, 128, 1, 3, [65], [400]),
    (64, 128, 1, 4, [4, 6], [2, 6]),                      # more tokens than the sequence has
]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("call", range(len(CALLS)))
def test_attention_is_that_of_the_definition(lowbit, call, dtype):
    page, dim, heads, group, counts, lengths = CALLS[call]
    c = Both(lowbit, lengths, page, heads, dim, seed=call)
    c.fill(lengths, dtype)
    q = torch.from_numpy(c.rng.standard_normal((sum(counts), heads * group, dim)).astype(np.float32) * 1.5).to(dtype)
    check_attention(c, attend(c, q, counts, lengths), q, counts, lengths)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("layout", [1, 2])
def test_strides_scale_and_generous_bounds(lowbit, layout, dtype):
    counts, lengths = [1, 9, 100], [500, 9, 164]
    c = Both(lowbit, lengths, 32, 2, 64, seed=layout)
    c.fill(lengths, dtype, layout)
    q = torch.from_numpy(c.rng.standard_normal((110, 6, 64)).astype(np.float32)).to(dtype)
    for new, most in ((None, None), (120, 512), (100, 100000)):
        check_attention(c, attend(c, q, counts, lengths, 0.3, layout, new, most), q, counts, lengths, 0.3)


@pytest.mark.parametrize("dtype", HALF)
def test_pages_of_very_different_scales(lowbit, dtype):
    """Zeros, small and large pages side by side: no weight is lost to another page's scale."""
    page, heads, dim, n = 16, 1, 64, 16 * 12
    c = Both(lowbit, [n], page, heads, dim, 12)
    k, v = c.values(n, dtype), c.values(n, dtype)
    for i in range(12):
        f = (0.0, 2.0 ** -12, 1.0, 2.0 ** 8)[i % 4]
        v[0][16 * i:16 * i + 16] *= f
        k[0][16 * i:16 * i + 16] *= (0.0, 1.0, 2.0 ** -10)[i % 3]
    k, v = (k[0], k[0].cuda()), (v[0], v[0].cuda())
    c.write([n], [n], k, v)
    for counts in ([1], [30], [n]):
        q = torch.randn(counts[0], 2, dim, generator=torch.Generator().manual_seed(3)).to(dtype)
        check_attention(c, attend(c, q, counts, [n]), q, counts, [n])


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("counts", [[1], [20], [90]])
def test_large_scores_and_one_certain_key(lowbit, counts, dtype):
    c = Both(lowbit, [300], 64, 1, 128, 13)
    k, v = c.values(300, dtype), c.values(300, dtype)
    c.write([300], [300], k, v)
    q = (torch.randn(counts[0], 2, 128, generator=torch.Generator().manual_seed(4)) * 40).to(dtype)
    check_attention(c, attend(c, q, counts, [300]), q, counts, [300])


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("new", [6, 90])
def test_what_a_row_does_not_see_cannot_reach_it(lowbit, new, dtype):
    """NaN in a late token's key or value: rows before it are as without it, rows from it on are NaN where they have to be."""
    n, heads, dim = 200, 1, 128
    at = n - new // 2                                     # a token that the first half of the rows does not see
    for what in ("k", "v"):
        c = Both(lowbit, [n], 64, heads, dim, 14)
        k, v = c.values(n, dtype), c.values(n, dtype)
        q = torch.randn(new, 3, dim, generator=torch.Generator().manual_seed(5)).to(dtype)
        c.write([n], [n], k, v)
        clean = attend(c, q, [new], [n])
        x = k if what == "k" else v
        x[0][at, 0, 17] = float("nan")
        c.write([n], [n], (k[0], k[0].cuda()), (v[0], v[0].cuda()))
        out = attend(c, q, [new], [n])
        first = new - (n - at)
        assert torch.equal(out[:first], clean[:first])
        nan = torch.isnan(out[first:])
        assert nan.all() if what == "k" else (nan[:, :, 17].all() and int(nan.sum()) == nan[:, :, 17].numel())


def test_the_same_call_gives_the_same_bits(lowbit):
    lengths = [2000, 700]
    c = Both(lowbit, lengths, 64, 2, 128, 15)
    c.fill(lengths, torch.bfloat16)
    for counts in ([1, 1], [100, 3]):
        q = torch.randn(sum(counts), 8, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
        outs = [attend(c, q, counts, lengths) for _ in range(4)]
        assert all(torch.equal(outs[0], o) for o in outs)


@pytest.mark.parametrize("new", [1, 70])
def test_a_cache_of_more_than_4_gib(lowbit, new):
    """Page numbers whose codes lie behind 2^32 bytes, for keys and for values."""
    pages, page, heads, dim, n = 70000, 64, 8, 128, 150
    cache = lowbit.Cache.empty(pages, heads, dim, page)
    table = ints([[69999, 3, 69998]])
    k, v = (torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for s in (1, 2))
    assert lowbit.cache_write(cache, k.cuda(), v.cuda(), table, ints([0, n]), ints([n])) == lowbit.OK
    small = Both(lowbit, [n], page, heads, dim, 16)
    small.write([n], [n], (k, k.cuda()), (v, v.cuda()))
    out = [torch.empty(n, heads, dim, device="cuda") for _ in range(2)]
    assert lowbit.cache_read(cache, *out, table, ints([0, n]), ints([n])) == lowbit.OK
    assert np.array_equal(out[0].cpu().double().numpy(), small.k.read(small.table[0], n))
    assert np.array_equal(out[1].cpu().double().numpy(), small.v.read(small.table[0], n))
    q = torch.randn(new, 16, dim, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    want = attend(small, q, [new], [n])
    small.cache, small.gpu_table = cache, table
    assert torch.equal(attend(small, q, [new], [n]), want)


@pytest.mark.parametrize("counts,lengths", [([1, 1, 1], [1000, 3, 0]), ([60, 1, 17], [60, 900, 200])])
def test_another_stream_and_a_graph_give_the_same(lowbit, counts, lengths):
    c = Both(lowbit, lengths, 64, 2, 128, 17)
    g = torch.Generator().manual_seed(7)
    n = sum(counts)
    inputs = [[torch.randn(n, h, 128, generator=g).to(torch.bfloat16).cuda() for h in (2, 2, 8)] for _ in range(3)]
    k, v, q = (torch.empty_like(t) for t in inputs[0])
    prior = [max(0, a - b) for a, b in zip(lengths, counts)]
    old = [torch.randn(sum(prior), 2, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
    table, starts, total = c.gpu_table, ints(starts_of(counts)), ints(lengths)
    assert lowbit.cache_write(c.cache, *old, table, ints(starts_of(prior)), ints(prior)) == lowbit.OK
    held = [t.clone() for t in c.cache.tensors]
    out, back = torch.empty_like(q), [torch.empty_like(k), torch.empty_like(v)]
    new, most = max(counts), max(lengths)
    ws = torch.empty(max(16, lowbit.cache_attention_workspace(c.cache, 3, n, 8, new, most)), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        assert lowbit.cache_write(c.cache, k, v, table, starts, total, stream=stream) == lowbit.OK
        assert lowbit.cache_attention(c.cache, q, out, table, starts, total, new, most, ws, stream=stream) == lowbit.OK
        assert lowbit.cache_read(c.cache, *back, table, starts, total, stream=stream) == lowbit.OK

    def begin(i):
        for t, old_ in zip(c.cache.tensors, held):
            t.copy_(old_)
        for t, x in zip((k, v, q), inputs[i]):
            t.copy_(x)
        for t in (out, *back):
            t.zero_()

    want = []
    for i in range(3):
        begin(i)
        step()
        want.append([t.clone() for t in (out, *back)])
    side = torch.cuda.Stream()
    begin(1)
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((out, *back), want[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (2, 0, 1, 2):
        begin(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, *back), want[i]))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("page,dim,counts,lengths", [(16, 64, [1, 1, 1], [1, 17, 0]), (32, 128, [1, 1], [33, 70]), (16, 128, [3, 40], [3, 50]), (64, 256, [1, 30], [5, 65])])
def test_pages_that_nothing_was_written_to_hold_anything(lowbit, page, dim, counts, lengths, dtype):
    """Every byte of them is a NaN, scales too, and one of them is the first page."""
    c = Both(lowbit, lengths, page, 2, dim, 21)
    c.table[c.table >= 0] = [p for p in range(1, c.cache.n_pages) if p != 2][:int((c.table >= 0).sum())]
    c.gpu_table.copy_(torch.from_numpy(c.table))
    for t in c.cache.tensors:
        t.fill_(255)
    c.fill(lengths, dtype)
    q = torch.from_numpy(c.rng.standard_normal((sum(counts), 6, dim)).astype(np.float32)).to(dtype)
    check_attention(c, attend(c, q, counts, lengths), q, counts, lengths)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("counts,lengths", [([1, 1], [1, 0]), ([1, 1], [300, 40]), ([5], [2]), ([1], [9000]), ([90], [200]), ([40], [5000])])
def test_infinite_and_undefined_scores(lowbit, counts, lengths, dtype):
    """A row whose scores are all minus infinity, one with plus infinity and one with NaN have no softmax: NaN.  One that sees nothing is zeros."""
    c = Both(lowbit, lengths, 64, 1, 64, 22)
    n = sum(lengths)
    k, v = c.values(n, dtype), c.values(n, dtype)
    k[0][:, :, 7] = 1.0
    c.write(lengths, lengths, (k[0], k[0].cuda()), v)
    for what in (float("-inf"), float("inf"), float("nan")):
        q = torch.zeros(sum(counts), 3, 64, dtype=dtype)
        q[:, 1, 7] = what                                  # of three heads the middle one
        out = attend(c, q, counts, lengths).cpu()
        at = 0
        for count, length in zip(counts, lengths):
            for i in range(count):
                sees = length - count + i + 1 > 0
                assert torch.isnan(out[at, 1]).all() if sees else (out[at] == 0).all(), (what, count, length, i)
                assert torch.isfinite(out[at, ::2]).all()
                at += 1


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim,counts", [(128, [90]), (256, [70]), (64, [100]), (128, [1])])
def test_queries_with_one_value_far_above_the_others(lowbit, dim, counts, dtype):
    """Where the keys have nothing for it, the others decide; some rows, none of a wave's, or all."""
    n = 150
    c = Both(lowbit, [n], 64, 1, dim, 23)
    k, v = c.values(n, dtype), c.values(n, dtype)
    k[0][:, :, 5] = 0
    c.write([n], [n], (k[0], k[0].cuda()), v)
    for rows in (slice(0, 1), slice(40, None), slice(None)):
        q = torch.from_numpy(c.rng.standard_normal((counts[0], 3, dim)).astype(np.float32)).to(dtype)
        q[rows, :, 5] = 60000.0 if dtype == torch.float16 else 1e8
        check_attention(c, attend(c, q, counts, [n]), q, counts, [n])


@pytest.mark.parametrize("page,dim,heads,group,counts,lengths", [
    (64, 128, 2, 4, [1, 1], [300, 64]), (16, 64, 1, 8, [1], [9000]), (32, 256, 1, 3, [4], [700]), (64, 128, 1, 6, [5], [1500]),
    (64, 64, 1, 2, [90], [200]), (64, 128, 2, 1, [77, 33], [190, 80]), (16, 128, 1, 5, [8], [5000]), (32, 256, 1, 2, [70], [101])])
def test_outputs_in_bf16_are_as_exact_as_their_format(lowbit, page, dim, heads, group, counts, lengths):
    """Weights keep the bits of two bf16 numbers for the product with the values, as for fp16 tensors: beside the output's one rounding nothing
    of the order of bf16's is left, which shows where values cancel."""
    c = Both(lowbit, lengths, page, heads, dim, seed=30 + dim)
    c.fill(lengths, torch.bfloat16)
    q = torch.from_numpy(c.rng.standard_normal((sum(counts), heads * group, dim)).astype(np.float32) * 1.5).to(torch.bfloat16)
    out, starts = attend(c, q, counts, lengths), starts_of(counts)
    for b, n in enumerate(lengths):
        rows = slice(starts[b], starts[b + 1])
        want, bound = plain.attention(q[rows].double().numpy(), c.k.read(c.table[b], n), c.v.read(c.table[b], n), dim ** -0.5, torch.float16)
        bound += plain.UNIT[torch.bfloat16] * np.abs(want)
        off = np.abs(out[rows].double().cpu().numpy() - want) - bound
        assert off.max() <= 0, (b, n, off.max(), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("far", [2.0 ** 14, 2.0 ** 16, 2.0 ** 20, 1e8])
@pytest.mark.parametrize("dim,counts", [(128, [90]), (256, [70]), (64, [100]), (128, [3])])
def test_queries_with_half_of_their_values_far_above_the_others(lowbit, dim, counts, far, dtype):
    """Where the keys have nothing for the large half, the small one decides."""
    if dtype == torch.float16 and far > 2.0 ** 14:
        far = 2.0 ** 14                                   # (what the format holds)
    n = 150
    c = Both(lowbit, [n], 64, 1, dim, 24)
    k, v = c.values(n, dtype), c.values(n, dtype)
    k[0][:, :, ::2] = 0
    c.write([n], [n], (k[0], k[0].cuda()), v)
    for rows in (slice(0, 1), slice(None)):
        q = torch.from_numpy(c.rng.standard_normal((counts[0], 3, dim)).astype(np.float32)).to(dtype)
        q[rows, :, ::2] = ((1 + 0.5 * torch.rand(q[rows, :, ::2].shape, generator=torch.Generator().manual_seed(dim))) * far).to(dtype)
        check_attention(c, attend(c, q, counts, [n]), q, counts, [n])


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim,counts,n", [(64, [100], 500), (128, [90], 700), (256, [70], 300), (128, [90], 5000), (128, [20], 900)])
def test_a_row_does_not_depend_on_the_others(lowbit, dim, counts, n, dtype):
    """Not a bit of it: the others with values that lose bits in eight, that are not finite, or with scores that grow from tile to tile."""
    c = Both(lowbit, [n], 64, 1, dim, 25)
    k, v = c.values(n, dtype), c.values(n, dtype)
    k[0][:, :, 3] = torch.linspace(-3, 3, n)[:, None].to(dtype)
    c.write([n], [n], (k[0], k[0].cuda()), v)
    q = torch.from_numpy(c.rng.standard_normal((counts[0], 3, dim)).astype(np.float32)).to(dtype)
    want = attend(c, q, counts, [n])
    for value in (1e-3, 200.0, 3e4, float("inf"), float("nan")):
        others = q.clone()
        others[1::2, :, 3] = value
        out = attend(c, others, counts, [n])
        differ = int((out[::2] != want[::2]).sum())
        assert differ == 0, (value, differ)


# starts that do not ascend from 0 to the tokens of the call, and the sequences that are in order all the same
BAD_STARTS = [([100, 1], [], 1), ([-5, 1], [], 1), ([0, 1, -1000, 3], [0], 3), ([0, 100, 2, 3], [2], 3), ([0, 1, 2, 9], [0, 1], 3), ([-1, 1, 2, 3], [1, 2], 3),
              ([0, 2, 1, 1], [0], 3), ([0, 1, 2, 3, 2 ** 31 - 1, 5], [0, 1, 2], 5), ([0, 1, -2 ** 31, 3, 4, 5], [0, 3, 4], 5),
              ([5000 if i == 10 else -7 if i == 3 else i for i in range(71)], [i for i in range(70) if i not in (2, 3, 9, 10)], 70),
              ([-1 if i < 66 else i for i in range(71)], [66, 67, 68, 69], 70)]


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("starts,good,tokens", BAD_STARTS)
def test_starts_out_of_order_are_told_and_leave_the_other_sequences_alone(lowbit, starts, good, tokens, page):
    batch, heads, dim = len(starts) - 1, 2, 64
    prior = [page - 3 + b % 7 for b in range(batch)]
    c = Both(lowbit, [n + 2 for n in prior], page, heads, dim, 40)
    c.fill(prior, torch.bfloat16)
    lengths = list(prior)
    for b in good:
        lengths[b] += starts[b + 1] - starts[b]
    k, v = c.values(tokens, torch.bfloat16), c.values(tokens, torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert lowbit.cache_write(c.cache, k[1], v[1], c.gpu_table, ints(starts), ints(lengths), status) == lowbit.OK
    assert status.item() == lowbit.E_ARG
    for b in good:
        rows = slice(starts[b], starts[b + 1])
        for form, x in ((c.k, k[0]), (c.v, v[0])):
            form.write(x[rows].double().numpy(), c.table[b:b + 1], [0, starts[b + 1] - starts[b]], [lengths[b]])
    c.check(lengths)                                       # all that is cached: nothing else was stored
    status.zero_()
    out = [torch.full((tokens, heads, dim), 9.0, device="cuda") for _ in range(2)]
    assert lowbit.cache_read(c.cache, *out, c.gpu_table, ints(starts), ints(lengths), status) == lowbit.OK
    assert status.item() == lowbit.E_ARG
    for t, form in zip(out, (c.k, c.v)):
        want = np.full((tokens, heads, dim), 9.0)
        for b in good:
            want[starts[b]:starts[b + 1]] = form.read(c.table[b], lengths[b])[lengths[b] - (starts[b + 1] - starts[b]):]
        assert np.array_equal(t.cpu().double().numpy(), want)


@pytest.mark.parametrize("starts,good,tokens", BAD_STARTS)
def test_starts_out_of_order_leave_the_attention_of_the_other_sequences_alone(lowbit, starts, good, tokens):
    """Also where the cached tokens are split, and the splits joined."""
    batch, heads, dim, page = len(starts) - 1, 1, 64, 64
    lengths = [70 + 31 * (b % 5) for b in range(batch)]
    lengths[good[0] if good else 0] = 2500
    c = Both(lowbit, lengths, page, heads, dim, 41)
    c.fill(lengths, torch.bfloat16)
    q = torch.from_numpy(c.rng.standard_normal((tokens, 2, dim)).astype(np.float32)).to(torch.bfloat16)
    for most in (2500, 20000):
        out = torch.full_like(q, 77.0, device="cuda")
        ws = torch.full((max(16, lowbit.cache_attention_workspace(c.cache, batch, tokens, 2, 2, most)),), 0xFF, dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        assert lowbit.cache_attention(c.cache, q.cuda(), out, c.gpu_table, ints(starts), ints(lengths), 2, most, ws, status=status) == lowbit.OK
        assert status.item() == lowbit.E_ARG
        left = torch.ones(tokens, dtype=torch.bool)
        for b in good:
            rows = slice(starts[b], starts[b + 1])
            want, bound = plain.attention(q[rows].double().numpy(), c.k.read(c.table[b], lengths[b]), c.v.read(c.table[b], lengths[b]), dim ** -0.5, q.dtype)
            assert (np.abs(out[rows].double().cpu().numpy() - want) <= bound).all(), b
            left[rows] = False
        assert bool((out.cpu()[left] == 77).all())


def test_places_that_the_binding_refuses_and_pinned_memory(lowbit):
    c = Both(lowbit, [20], 16, 1, 64, 50)
    c.fill([20], torch.bfloat16)
    q = torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    want = attend(c, q, [1], [20])
    good = dict(q=q.cuda(), out=torch.empty_like(q, device="cuda"), table=c.gpu_table, starts=ints([0, 1]), lengths=ints([20]), status=torch.zeros(1, dtype=torch.int32, device="cuda"),
                workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    call = lambda q, out, table, starts, lengths, status, workspace: lowbit.cache_attention(c.cache, q, out, table, starts, lengths, 1, 20, workspace, status=status)  # noqa: E731
    for name, t in good.items():
        with pytest.raises(ValueError, match="GPU"):
            call(**good | {name: t.cpu()})                  # refused on the host: no kernel sees the address
    pinned = {name: good[name].cpu().pin_memory() for name in ("table", "starts", "lengths", "status")}
    assert call(**good | pinned) == lowbit.OK
    torch.cuda.synchronize()
    assert torch.equal(good["out"], want) and pinned["status"].item() == 0


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("counts,lengths", [([1, 1], [300, 0]), ([90], [200]), ([40, 60], [5000, 60])])
def test_infinite_and_undefined_scores_of_wide_heads(lowbit, dim, counts, lengths, dtype):
    """As test_infinite_and_undefined_scores, of three heads the middle one; the others' rows are those of the definition."""
    c = Both(lowbit, lengths, 64, 1, dim, 42)
    n = sum(lengths)
    k, v = c.values(n, dtype), c.values(n, dtype)
    k[0][:, :, 7] = 1.0
    c.write(lengths, lengths, (k[0], k[0].cuda()), v)
    for what in (float("-inf"), float("inf"), float("nan")):
        q = torch.from_numpy(c.rng.standard_normal((sum(counts), 3, dim)).astype(np.float32)).to(dtype)
        q[:, 1] = 0
        q[:, 1, 7] = what
        out = attend(c, q, counts, lengths)
        at = 0
        for count, length in zip(counts, lengths):
            for i in range(count):
                sees = length - count + i + 1 > 0
                assert torch.isnan(out[at, 1]).all() if sees else (out[at] == 0).all(), (what, count, length, i)
                at += 1
        check_attention(c, out[:, ::2], q[:, ::2].contiguous(), counts, lengths)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("layout", [1, 2])
def test_strides_of_wide_heads(lowbit, layout, dim, dtype):
    counts, lengths = [1, 9, 60], [900, 9, 164]
    c = Both(lowbit, lengths, 32, 2, dim, seed=43 + layout)
    c.fill(lengths, dtype, layout)
    q = torch.from_numpy(c.rng.standard_normal((70, 6, dim)).astype(np.float32)).to(dtype)
    for new, most in ((None, None), (100, 100000)):
        check_attention(c, attend(c, q, counts, lengths, 0.2, layout, new, most), q, counts, lengths, 0.2)
    few = [1, 0, 5]
    check_attention(c, attend(c, q[:6], few, lengths, None, layout), q[:6], few, lengths)
