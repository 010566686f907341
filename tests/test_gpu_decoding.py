"""A decoding loop of the operators together: a projection by a matrix in 8 bits, its keys and queries rotated on the way into the cache, attention over the
cache, the logits by another matrix, and the draw of the next tokens, which the next step begins with.  Steps of several tokens and of one are captured
into a graph each; both use one piece of scratch memory.  Each operator's results are checked against its plain form of what the one before it gave."""
import numpy as np
import pytest
import torch

import lowbit_plain as plain
from decoding_plain import draw, fp8_decode, fp8_encode, products_bound, turned

pytestmark = pytest.mark.gpu
OK = 0
HIDDEN, HEADS, KV, DIM, PAGE, VOCAB, BATCH, PAGES, ROTARY = 200, 4, 2, 64, 16, 1003, 3, 4, 32
LONGEST = PAGE * PAGES


class Model:
    def __init__(self, dtype):
        from paper_2604_03298_amd import lowbit, sampling
        self.lowbit, self.sampling, self.dtype = lowbit, sampling, dtype
        rng = self.rng = np.random.default_rng(12)
        normal = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda()  # noqa: E731
        self.embedding = normal(VOCAB, HIDDEN)
        self.qkv, self.head = self.stored(normal((HEADS + 2 * KV) * DIM, HIDDEN) / 14), self.stored(normal(VOCAB, HEADS * DIM) / 4)
        a = np.arange(LONGEST)[:, None] * 10000.0 ** (-np.arange(0, ROTARY, 2) / ROTARY)
        self.angles = np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)
        self.turns = torch.from_numpy(self.angles).cuda()
        self.cache = lowbit.Cache.empty(BATCH * PAGES, KV, DIM, PAGE)
        for t in self.cache.tensors:
            t.zero_()
        self.pages = rng.permutation(BATCH * PAGES).reshape(BATCH, PAGES).astype(np.int32)
        self.table = torch.from_numpy(self.pages).cuda()
        self.lengths, self.status = torch.zeros(BATCH, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.k, self.v = plain.PlainCache(PAGE, KV, DIM), plain.PlainCache(PAGE, KV, DIM)
        most = BATCH * 5
        self.space = torch.empty(max(lowbit.fp8_linear_workspace(most, (HEADS + 2 * KV) * DIM, HIDDEN), lowbit.fp8_linear_workspace(BATCH, VOCAB, HEADS * DIM),
                                     lowbit.cache_attention_workspace(self.cache, BATCH, most, HEADS, 5, LONGEST), sampling.sample_workspace(BATCH, VOCAB)) + 16,
                                 dtype=torch.uint8, device="cuda")

    def stored(self, w):
        codes, scales = self.lowbit.fp8_empty(*w.shape)
        assert self.lowbit.fp8_quantize(w, codes, scales) == OK
        return codes, scales, fp8_decode(*fp8_encode(w.double().cpu().numpy()), w.shape[1])


class Step:
    """`new` tokens of each sequence, of which `active` says which are there; the last of them are read from and drawn into `drawn`."""

    def __init__(self, model, new, drawn):
        m, n = model, BATCH * new
        empty = lambda *shape, dtype=model.dtype: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.model, self.new, self.drawn = model, new, drawn
        self.ids = torch.zeros(BATCH, new, dtype=torch.int32, device="cuda")
        self.active = torch.ones(BATCH, dtype=torch.int32, device="cuda")
        self.starts = torch.arange(BATCH + 1, dtype=torch.int32, device="cuda") * new
        self.x, self.rows, self.seen, self.logits = empty(n, HIDDEN), empty(n, (HEADS + 2 * KV) * DIM), empty(n, HEADS, DIM), empty(BATCH, VOCAB)
        self.q = empty(n, HEADS, DIM)
        self.uniform, self.log_probs = empty(BATCH, dtype=torch.float32), empty(BATCH, dtype=torch.float32)
        self.how = {"temperature": torch.tensor([0.8, 1.0, 0.0]).cuda(), "top_k": torch.tensor([50, 0, 0], dtype=torch.int32).cuda(),
                    "top_p": torch.tensor([0.9, 0.95, 1.0]).cuda(), "min_p": torch.tensor([0.0, 0.02, 0.0]).cuda()}

    def launch(self):
        m, lowbit, n = self.model, self.model.lowbit, BATCH * self.new
        self.ids[:, 0].copy_(self.drawn)
        m.lengths.add_(self.active * self.new)
        torch.index_select(m.embedding, 0, self.ids.view(-1), out=self.x)
        assert lowbit.fp8_linear(self.x, *m.qkv[:2], self.rows, m.space) == OK
        heads = self.rows.view(n, HEADS + 2 * KV, DIM)
        q, k, v = heads[:, :HEADS], heads[:, HEADS:HEADS + KV], heads[:, HEADS + KV:]
        assert lowbit.cache_write_rotated(m.cache, k, v, q, self.q, m.turns, m.table, self.starts, m.lengths, status=m.status) == OK
        assert lowbit.cache_attention(m.cache, self.q, self.seen, m.table, self.starts, m.lengths, self.new, LONGEST, m.space, status=m.status) == OK
        last = self.seen.view(BATCH, self.new, HEADS * DIM)[:, -1]
        assert lowbit.fp8_linear(last, *m.head[:2], self.logits, m.space) == OK
        assert m.sampling.sample(self.logits, self.uniform, self.drawn, log_probs=self.log_probs, workspace=m.space, **self.how) == OK

    def check(self, before):
        m, new, n = self.model, self.new, BATCH * self.new
        values = lambda t: t.double().cpu().numpy()  # noqa: E731
        near = lambda got, x, w: (np.abs(values(got) - x @ w.T) <= products_bound(x, w, x @ w.T, m.dtype)).all()  # noqa: E731
        lengths, starts, x = m.lengths.tolist(), self.starts.tolist(), m.embedding[self.ids.view(-1).long()]
        assert self.ids[:, 0].tolist() == before and m.status.item() == 0 and torch.equal(self.x, x)
        assert near(self.rows, fp8_decode(*fp8_encode(values(x)), HIDDEN), m.qkv[2])
        heads = self.rows.float().cpu().numpy().reshape(n, -1, DIM)
        q, k, v = heads[:, :HEADS], heads[:, HEADS:HEADS + KV].copy(), heads[:, HEADS + KV:]
        turned_q = np.zeros(q.shape, np.float32)
        for b in range(BATCH):
            mine, first = slice(starts[b], starts[b + 1]), lengths[b] - new
            turned_q[mine], k[mine] = turned(q[mine], first, m.angles, False), turned(k[mine], first, m.angles, False)
        assert torch.equal(self.q.cpu(), torch.from_numpy(turned_q).to(m.dtype))
        m.k.write(k.astype(np.float64), m.pages, starts, lengths)
        m.v.write(v.astype(np.float64), m.pages, starts, lengths)
        codes = m.cache.tensors[0].cpu().numpy()
        assert all((codes[at] == c).all() for at, c in m.k.codes.items())
        for b in range(BATCH):
            mine = slice(starts[b], starts[b + 1])
            want, bound = np.zeros((new, HEADS, DIM)), np.zeros((new, HEADS, DIM))
            if lengths[b]:
                want, bound = plain.attention(values(self.q[mine]), m.k.read(m.pages[b], lengths[b]), m.v.read(m.pages[b], lengths[b]), DIM ** -0.5, m.dtype)
            assert (np.abs(values(self.seen[mine]) - want) <= bound).all()
        last = values(self.seen).reshape(BATCH, new, HEADS * DIM)[:, -1]
        assert near(self.logits, fp8_decode(*fp8_encode(last), HEADS * DIM), m.head[2])
        for b in range(BATCH):
            token, log_prob, weight = draw(values(self.logits[b]), uniform=self.uniform[b].item(), **{name: t[b].item() for name, t in self.how.items()})
            # one rounding to 32 bits, and half of 2^-46 of each weight
            assert self.drawn[b].item() == token and abs(self.log_probs[b].item() - log_prob) <= 2.0 ** -24 * abs(log_prob) + VOCAB * 2.0 ** -46 / weight + 2.0 ** -40


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_steps_captured_and_replayed(dtype):
    model = Model(dtype)
    drawn = torch.zeros(BATCH, dtype=torch.int32, device="cuda")
    steps = {new: Step(model, new, drawn) for new in (5, 1)}
    graphs = {}
    for new, step in steps.items():
        step.uniform.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step.launch()
        torch.cuda.current_stream().wait_stream(side)
        graphs[new] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[new]):
            step.launch()
        model.lengths.zero_()
        torch.cuda.synchronize()
    drawn.zero_()
    for i, new in enumerate((5, 1, 1, 5, 1, 5, 5, 1, 1)):
        step = steps[new]
        step.ids.copy_(torch.from_numpy(model.rng.integers(0, VOCAB, step.ids.shape)))
        step.uniform.copy_(torch.from_numpy(model.rng.random(BATCH, dtype=np.float32)))
        step.active.copy_(torch.tensor([1, 0 if i < 3 else 1, 1]))             # (the second sequence comes later: until then its tokens have no place)
        before = drawn.tolist()
        if i == 4:
            step.launch()                                                      # (an eager one between the replays)
        else:
            graphs[new].replay()
        torch.cuda.synchronize()
        step.check(before)
    assert model.lengths.tolist() == [25, 18, 25]
