"""Keys and queries rotated by their positions on the way into the 8-bit cache, byte for byte against plain forms."""
import numpy as np
import pytest
import torch

from decoding_plain import turned
from lowbit_plain import PlainCache

pytestmark = pytest.mark.gpu
OK, E_ARG = 0, 1


@pytest.fixture(scope="module")
def lowbit():
    from paper_2604_03298_amd import lowbit as module
    module.lib()
    return module


def angles(positions, rotary):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def tokens_of(rng, n, heads, dim, dtype):
    return torch.from_numpy((rng.standard_normal((n, heads, dim)) * np.exp(rng.standard_normal((1, heads, 1)))).astype(np.float32)).to(dtype)


class Both:
    """The library's cache and the plain one, side by side."""

    def __init__(self, lowbit, seed, batch, kv, dim, page, pages_each, rotary, positions, interleaved, dtype):
        self.lowbit, self.rng, self.dtype, self.kv, self.dim, self.page, self.interleaved = lowbit, np.random.default_rng(seed), dtype, kv, dim, page, interleaved
        n = batch * pages_each + 2
        self.cache = lowbit.Cache.empty(n, kv, dim, page)
        for t in self.cache.tensors:
            t.copy_(torch.from_numpy(self.rng.integers(0, 256, t.shape).astype(np.uint8)))
        self.before = [t.cpu().numpy().copy() for t in self.cache.tensors]
        self.table = self.rng.permutation(n)[:batch * pages_each].reshape(batch, pages_each).astype(np.int32)
        self.turns = angles(positions, rotary)
        self.k, self.v = PlainCache(page, kv, dim), PlainCache(page, kv, dim)

    def write(self, new, lengths, group, in_place=False, status=None):
        t, starts = sum(new), [0] + list(np.cumsum(new))
        k, v = (tokens_of(self.rng, t, self.kv, self.dim, self.dtype) for _ in range(2))
        q = tokens_of(self.rng, t, self.kv * group, self.dim, self.dtype) if group else None
        q_in = None if q is None else q.cuda()
        out = q_in if in_place or q is None else torch.full_like(q_in, 7.0)
        assert self.lowbit.cache_write_rotated(self.cache, k.cuda(), v.cuda(), q_in, out, torch.from_numpy(self.turns).cuda(), ints(self.table.tolist()),
                                               ints(starts), ints(lengths), interleaved=self.interleaved, status=status) == OK
        torch.cuda.synchronize()
        plain = lambda x: x.float().numpy()  # noqa: E731
        rk, rq = np.zeros(k.shape, np.float32), None if q is None else np.zeros(q.shape, np.float32)
        for b in range(len(new)):
            mine, first = slice(starts[b], starts[b + 1]), lengths[b] - new[b]
            rk[mine] = turned(plain(k)[mine], first, self.turns, self.interleaved)
            if q is not None:
                rq[mine] = turned(plain(q)[mine], first, self.turns, self.interleaved)
        self.k.write(rk.astype(np.float64), self.table, starts, lengths)
        self.v.write(plain(v).astype(np.float64), self.table, starts, lengths)
        if q is not None:
            assert torch.equal(out.cpu(), torch.from_numpy(rq).to(self.dtype))

    def check(self):
        kc, ks, vc, vs = (t.cpu().numpy() for t in self.cache.tensors)
        for plain, codes, scales, at, old, old_scales in ((self.k, kc, ks, lambda p, h, i: (p, h, i), self.before[0], self.before[1]),
                                                          (self.v, vc, vs, lambda p, h, i: (p, h, slice(None), i), self.before[2], self.before[3])):
            want, bytes_ = old.copy(), old_scales.copy()
            for (p, h, i), c in plain.codes.items():
                want[at(p, h, i)] = c
            for (p, h), e in plain.exponent.items():
                bytes_[p, h] = e + 127
            assert np.array_equal(scales, bytes_) and np.array_equal(codes, want)      # and nothing else was written


SHAPES = [(1, 64, 16, 64, 1, False), (2, 128, 64, 128, 4, False), (8, 128, 16, 64, 4, True), (3, 256, 32, 256, 5, True), (2, 256, 128, 128, 1, False),
          (1, 64, 16, 16, 9, False), (1, 128, 256, 48, 0, True), (4, 64, 64, 48, 2, False), (2, 128, 32, 32, 64, True)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kv, dim, page, rotary, group, interleaved", SHAPES)
def test_prompts_then_single_tokens(lowbit, kv, dim, page, rotary, group, interleaved, dtype):
    both = Both(lowbit, kv + dim + page, 4, kv, dim, page, 3, rotary, 3 * page, interleaved, dtype)
    lengths = [page + 5, 1, 2 * page, page - 1]
    both.write(lengths, lengths, group)
    both.check()
    for new in ([1, 1, 1, 1], [3, 0, 1, 2], [1, 1, 0, 1]):
        lengths = [n + t for n, t in zip(lengths, new)]
        both.write(new, lengths, group, in_place=new[0] == 3)
        both.check()


@pytest.mark.parametrize("interleaved", [False, True])
def test_idle_slots(lowbit, interleaved):
    """Negative positions: not stored, and zeros in place of rotated queries, whatever the table says."""
    both = Both(lowbit, 5, 3, 2, 128, 64, 2, 64, 100, interleaved, torch.bfloat16)
    both.table[1] = -1
    status = ints([0])
    both.write([1, 1, 70], [1, 0, 70], 4, status=status)
    both.check()
    both.write([2, 3, 1], [1, 0, 71], 4, in_place=True, status=status)
    both.check()
    assert status.item() == 0


def test_no_turn_is_the_plain_write(lowbit):
    rng = np.random.default_rng(2)
    k, v = (tokens_of(rng, 90, 4, 128, torch.bfloat16).cuda() for _ in range(2))
    table, starts, lengths = ints([[0, 3], [1, 4]]), ints([0, 50, 90]), ints([50, 90])
    turns = torch.zeros(100, 64, 2, device="cuda")
    turns[..., 0] = 1
    caches = [lowbit.Cache.empty(5, 4, 128, 64) for _ in range(2)]
    for c in caches:
        for t in c.tensors:
            t.zero_()
    assert lowbit.cache_write(caches[0], k, v, table, starts, lengths) == OK
    assert lowbit.cache_write_rotated(caches[1], k, v, None, None, turns, table, starts, lengths) == OK
    assert all(torch.equal(a, b) for a, b in zip(caches[0].tensors, caches[1].tensors))


def test_strides(lowbit):
    """Keys, values and queries as parts of one projection's output, rotated in place; two bytes off any alignment."""
    for dtype in (torch.bfloat16, torch.float16):
        for interleaved in (False, True):
            rng = np.random.default_rng(3)
            kv, group, dim, t = 2, 3, 64, 21
            held = tokens_of(rng, t, kv * (group + 2), dim + 1, dtype).reshape(t, -1)[:, 1:]
            heads = torch.nn.functional.pad(held, (0, 3))
            row = heads.shape[1]
            part = lambda x, first, n: x.as_strided((t, n, dim), (row, dim + 1, 1), first * (dim + 1))  # noqa: E731
            turns = torch.from_numpy(angles(30, 32)).cuda()
            got, table, starts, lengths = heads.cuda().clone(), ints([[1, 0]]), ints([0, t]), ints([t + 4])
            cache, other = lowbit.Cache.empty(2, kv, dim, 16), lowbit.Cache.empty(2, kv, dim, 16)
            for c in (cache, other):
                for x in c.tensors:
                    x.zero_()
            q = part(got, 2 * kv, kv * group)
            assert lowbit.cache_write_rotated(cache, part(got, 0, kv), part(got, kv, kv), q, q, turns, table, starts, lengths, interleaved=interleaved) == OK
            k, v, q = (part(heads.cuda(), f, n).contiguous() for f, n in ((0, kv), (kv, kv), (2 * kv, kv * group)))
            out = torch.empty_like(q)
            assert lowbit.cache_write_rotated(other, k, v, q, out, turns, table, starts, lengths, interleaved=interleaved) == OK
            assert all(torch.equal(a, b) for a, b in zip(cache.tensors, other.tensors))
            want = heads.cuda().clone()
            part(want, 2 * kv, kv * group).copy_(out)
            assert torch.equal(got, want)                   # and nothing around the queries was written


def test_what_only_the_device_sees(lowbit):
    """Lengths beyond the table of turns, starts out of order and pages that the cache has not: told, left out, the others done."""
    rng = np.random.default_rng(4)
    turns = torch.from_numpy(angles(40, 64)).cuda()

    def write(table, starts, lengths, t):
        k, v = (tokens_of(rng, t, 1, 64, torch.bfloat16).cuda() for _ in range(2))
        q = tokens_of(rng, t, 2, 64, torch.bfloat16).cuda()
        out, cache, status = torch.full_like(q, 7.0), lowbit.Cache.empty(8, 1, 64, 16), ints([0])
        for x in cache.tensors:
            x.fill_(0x55)
        assert lowbit.cache_write_rotated(cache, k, v, q, out, turns, ints(table), ints(starts), ints(lengths), status=status) == OK
        touched = [p for p in range(8) if any((x[p] != 0x55).any() for x in cache.tensors)]
        return touched, (out != 7).flatten(1).any(1).cpu().tolist(), status.item()

    assert write([[0, 1, 2], [3, 4, 5]], [0, 2, 4], [41, 20], 4) == ([4], [False, False, True, True], E_ARG)
    assert write([[0, 1, 2], [3, 4, 5]], [0, 2, 4], [40, 20], 4) == ([2, 4], [True] * 4, OK)
    assert write([[0, 1, 2], [3, 4, 5]], [2, 0, 4], [20, 20], 4)[2] == E_ARG
    assert write([[0, 99, 2], [3, -1, 5]], [0, 2, 4], [20, 18], 4) == ([], [True] * 4, E_ARG)     # queries need no page
    assert write([[0, 1, 2], [3, 4, 5]], [0, 2, 4], [49, -1], 4) == ([], [False] * 4, E_ARG)


def test_captured_and_replayed(lowbit):
    """Steps of single tokens as a graph: lengths grow on the device, positions and pages follow."""
    rng = np.random.default_rng(6)
    kv, group, dim, page = 2, 4, 128, 16
    turns = torch.from_numpy(angles(64, 128)).cuda()
    table, starts, lengths = ints([[0, 1, 2], [5, 4, 3]]), ints([0, 1, 2]), ints([13, 30])
    k, v = (tokens_of(rng, 2, kv, dim, torch.bfloat16).cuda() for _ in range(2))
    q = tokens_of(rng, 2, kv * group, dim, torch.bfloat16).cuda()
    caches, outs = [], [torch.empty_like(q) for _ in range(2)]
    for _ in range(2):
        caches.append(lowbit.Cache.empty(6, kv, dim, page))
        for t in caches[-1].tensors:
            t.fill_(0x31)
    call = lambda i: lowbit.cache_write_rotated(caches[i], k, v, q, outs[i], turns, table, starts, lengths)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert call(0) == OK
    torch.cuda.current_stream().wait_stream(side)
    assert call(1) == OK
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert call(0) == OK
    for _ in range(5):
        lengths += 1
        for t in (k, v):
            t.copy_(tokens_of(rng, 2, kv, dim, torch.bfloat16))
        q.copy_(tokens_of(rng, 2, kv * group, dim, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert call(1) == OK
        assert torch.equal(outs[0], outs[1]) and all(torch.equal(a, b) for a, b in zip(caches[0].tensors, caches[1].tensors))
