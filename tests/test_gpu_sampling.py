"""A token for each row of logits, against a plain form in 64 bits."""
import math

import numpy as np
import pytest
import torch

from decoding_plain import draw

pytestmark = pytest.mark.gpu
FORMATS = [torch.bfloat16, torch.float16, torch.float32]
OK = 0


@pytest.fixture(scope="module")
def sampling():
    from paper_2604_03298_amd import sampling as module
    module.lib()
    return module


def run(sampling, logits, uniform, **how):
    rows, vocab = logits.shape
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    log_probs = torch.full((rows,), 7.0, device="cuda")
    make = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}
    how = {k: torch.tensor(v, dtype=make[k]).cuda() for k, v in how.items()}
    space = torch.empty(sampling.sample_workspace(rows, vocab) + 16, dtype=torch.uint8, device="cuda")
    assert sampling.sample(logits, torch.tensor(uniform, dtype=torch.float32).cuda(), tokens, log_probs=log_probs, workspace=space, **how) == OK
    return tokens.cpu().numpy(), log_probs.cpu().numpy().astype(np.float64), {k: v.cpu().numpy() for k, v in how.items()}


def check(sampling, logits, uniform, **how):
    tokens, log_probs, how = run(sampling, logits, uniform, **how)
    l = logits.float().cpu().numpy().astype(np.float64)
    uniform = np.asarray(uniform, dtype=np.float32)
    for r in range(l.shape[0]):
        token, log_prob, mine = draw(l[r], uniform=float(uniform[r]), **{k: v[r].item() for k, v in how.items()})
        assert tokens[r] == token, (r, token, tokens[r], {k: v[r] for k, v in how.items()}, uniform[r])
        # one rounding to 32 bits; each weight is off by half of 2^-46 (a larger vocabulary: of its unit), which all of them add to the sum
        unit = 2.0 ** -46 * max(1, l.shape[1] / 32768)
        assert math.isnan(log_prob) == math.isnan(log_probs[r])
        assert math.isnan(log_prob) or abs(log_probs[r] - log_prob) <= 2.0 ** -24 * abs(log_prob) + l.shape[1] * unit / mine + 2.0 ** -40, r


def rows_of(rng, rows, vocab, dtype, forbidden=0.02):
    x = rng.standard_normal((rows, vocab)) * 2 * np.exp(0.5 * rng.standard_normal((rows, 1)))
    x[:, 1:][rng.random((rows, vocab - 1)) < forbidden] = -np.inf
    return torch.from_numpy(x.astype(np.float32)).to(dtype).cuda()


SIZES = [(1, 1), (3, 2), (2, 63), (5, 64), (4, 1000), (3, 8191), (2, 8193), (3, 32003), (1, 70001), (1, 131072)]


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("rows, vocab", SIZES)
def test_each_filter_and_all(sampling, rows, vocab, dtype):
    rng = np.random.default_rng(rows * 100 + vocab)
    u = lambda: rng.random(rows).astype(np.float32)  # noqa: E731
    t = lambda: 0.3 + 1.5 * rng.random(rows)  # noqa: E731
    k = lambda: np.exp(rng.uniform(0, np.log(vocab + 2), rows)).astype(np.int32)  # noqa: E731
    p, least = lambda: rng.random(rows) * 1.05, lambda: 0.3 * rng.random(rows) ** 3  # noqa: E731
    for how in ({}, {"temperature": t()}, {"temperature": t(), "top_k": k()}, {"temperature": t(), "top_p": p()}, {"temperature": t(), "min_p": least()},
                {"top_k": k(), "top_p": p()}, {"temperature": t(), "top_k": k(), "top_p": p(), "min_p": least()},
                {"temperature": np.zeros(rows), "top_k": k(), "top_p": p()}):
        check(sampling, rows_of(rng, rows, vocab, dtype), u(), **how)


def test_rows_that_ask_for_different_things(sampling):
    rng = np.random.default_rng(5)
    rows, vocab = 64, 1500
    kind = rng.integers(0, 5, rows)
    check(sampling, rows_of(rng, rows, vocab, torch.float32), rng.random(rows), temperature=np.where(kind == 0, 0, 0.2 + rng.random(rows)),
          top_k=np.where(kind == 1, rng.integers(1, 200, rows), rng.integers(-3, 1, rows)), top_p=np.where(kind == 2, rng.random(rows), 1 + rng.random(rows)),
          min_p=np.where(kind == 3, 0.2 * rng.random(rows), -rng.random(rows)))


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("vocab", [10, 4096, 40000, 131072])
def test_ties(sampling, vocab, dtype):
    """All equal, two values, a few values: cuts fall inside of ties, and exactly between them."""
    rng = np.random.default_rng(vocab)
    rows = 6
    how = {"top_k": [vocab // 2, 1, vocab - 1, 3, vocab, 0], "top_p": [0.5, 0.25, 1.0, 0.75, 0.125, 0.9999]}
    u = [0.0, 0.5, 0.25, 0.75, 0.9999999, 0.125]
    same = torch.full((rows, vocab), 1.25, dtype=dtype, device="cuda")
    few = torch.from_numpy(rng.integers(0, 3, (rows, vocab)).astype(np.float32)).to(dtype).cuda()
    zeros = torch.where(few > 1, 0.0, -0.0).to(dtype)
    for logits in (same, few, zeros):
        for names in ((), ("top_k",), ("top_p",), ("top_k", "top_p")):
            check(sampling, logits, u, **{n: how[n] for n in names})
        check(sampling, logits, u, min_p=[0.0, 1.0, 1.5, 0.3, 0.36, 0.14])


def test_cuts_next_to_one_another(sampling):
    """Half of a nearly flat row's tokens, and of those all but the last hundredth: both cuts lie in one stretch of the order, which is listed beyond top_k's end."""
    rng = np.random.default_rng(19)
    for vocab, rows in ((18584, 48), (45887, 16)):
        logits = torch.from_numpy(-rng.exponential(3, (rows, vocab)).astype(np.float32)).cuda()
        check(sampling, logits, rng.random(rows), temperature=[50.0] * rows, top_k=[vocab // 2] * rows, top_p=rng.choice([0.99, 0.995, 0.98], rows))


def test_borders_that_are_exact(sampling):
    """Weights of 1, 1/2, 1/4 ... (T so that logits are powers of two): sums that a share meets exactly."""
    logits = torch.zeros(4, 8, device="cuda")
    u = [0.0, 0.25, 0.5, 0.875]
    tokens, _, _ = run(sampling, logits, u)
    assert tokens.tolist() == [0, 2, 4, 7]                      # at a border the next one
    tokens, _, _ = run(sampling, logits, [0.9999999] * 4, top_p=[0.125, 0.1250001, 0.5, 0.0])
    assert tokens.tolist() == [0, 1, 3, 0]                      # reached exactly: no further one


def test_infinities_and_rows_without_a_token(sampling):
    inf, nan = math.inf, math.nan
    logits = torch.tensor([[1.0, inf, 2.0, inf], [-inf, -inf, -inf, -inf], [1.0, nan, 2.0, 3.0], [-inf, 5.0, -inf, -inf], [nan, -inf, -inf, -inf],
                           [3e38, -3e38, 3e38, 0.0]], device="cuda")
    for u in (0.0, 0.4, 0.6, 0.99):
        check(sampling, logits, [u] * 6)
        check(sampling, logits, [u] * 6, temperature=[0.0] * 6)
        check(sampling, logits, [u] * 6, top_k=[3] * 6, top_p=[0.9] * 6, min_p=[0.1] * 6)
        check(sampling, logits, [u] * 6, top_k=[1] * 6, temperature=[1e-38] * 6)
        check(sampling, logits, [u] * 6, temperature=[3e38] * 6)
    bits = torch.tensor([[-1, 0, 0, 0], [0x7F800001, 0, 0, 0]], dtype=torch.int32, device="cuda").view(torch.float32)
    assert run(sampling, bits, [0.5, 0.5])[0].tolist() == [-1, -1]  # every NaN is one


def test_arguments_of_a_row_out_of_range(sampling):
    logits = torch.zeros(7, 100, device="cuda")
    nan = math.nan
    check(sampling, logits, [0.5, 0.5, 0.5, 1.0, -0.1, nan, 0.5], temperature=[-1.0, nan, math.inf, 1, 1, 1, 1], top_p=[1, 1, 1, 1, 1, 1, nan])
    check(sampling, logits, [0.5] * 7, min_p=[nan, 2, -1, 0, 0, 0, 1], top_k=[0, 1, -5, 2 ** 31 - 1, -2 ** 31, 3, 50], top_p=[0.5, 0.5, -1, 2, 0, math.inf, 0.01])


def test_rows_apart_and_at_odd_addresses(sampling):
    rng = np.random.default_rng(6)
    for dtype in FORMATS:
        held = rows_of(rng, 4, 3000, dtype).reshape(-1)
        check(sampling, held[1:].as_strided((4, 2900), (2999, 1), 1), rng.random(4), top_k=[5, 50, 500, 0], top_p=[0.9, 0.5, 0.99, 0.7])


def test_more_rows_than_parts_and_a_long_vocabulary(sampling):
    """Rows that are not divided, weights of which some tokens are of a coarser unit, and rows of one value, whose cuts lie among more ties than any list holds."""
    rng = np.random.default_rng(11)
    for rows, vocab in ((600, 3001), (2, 300001)):
        logits = rows_of(rng, rows, vocab, torch.float32)
        logits[-1] = 1.5
        check(sampling, logits, rng.random(rows), temperature=0.3 + rng.random(rows), top_k=rng.choice([0, 7, 1000, 2900], rows), top_p=rng.choice([0.5, 0.9, 1.0], rows),
              min_p=rng.choice([0.0, 0.01], rows))


def test_the_longest_vocabulary(sampling):
    """2^22 tokens, also with a run of them that no filter cuts; the last ones are drawn, too."""
    rng = np.random.default_rng(17)
    logits = torch.from_numpy((3 * rng.standard_normal((3, 1 << 22))).astype(np.float32)).cuda()
    logits[2, -1] = 40.0
    check(sampling, logits, [0.3, 0.999, 0.5], temperature=[1.0, 0.7, 1.0], top_k=[1000, 0, 0], top_p=[0.9, 0.5, 1.0])


def test_one_piece_of_memory_serves_fewer_rows(sampling):
    rng = np.random.default_rng(13)
    vocab = 20011
    space = torch.empty(sampling.sample_workspace(300, vocab), dtype=torch.uint8, device="cuda")
    for rows in (1, 33, 300):
        space.fill_(0xFF)                                  # (whatever it held before)
        logits, u, p = rows_of(rng, rows, vocab, torch.float32), torch.from_numpy(rng.random(rows).astype(np.float32)), torch.full((rows,), 0.9, device="cuda")
        tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
        assert sampling.sample(logits, u.cuda(), tokens, top_p=p, workspace=space) == OK
        l = logits.cpu().numpy().astype(np.float64)
        assert tokens.tolist() == [draw(l[r], top_p=float(np.float32(0.9)), uniform=u[r].item())[0] for r in range(rows)]


def test_draws_follow_the_probabilities(sampling):
    """4096 equally spaced numbers: each token is drawn as often as its share says, to within the one draw at either end."""
    rng = np.random.default_rng(7)
    l = rng.standard_normal(50).astype(np.float32)
    n = 4096
    tokens, _, _ = run(sampling, torch.from_numpy(np.tile(l, (n, 1))).cuda(), (np.arange(n) + 0.5) / n)
    p = np.exp(l.astype(np.float64))
    assert (np.abs(np.bincount(tokens, minlength=50) - n * p / p.sum()) <= 1).all() and (np.diff(tokens) >= 0).all()


def test_captured_and_replayed(sampling):
    rng = np.random.default_rng(9)
    for rows, vocab in ((3, 40000), (40, 5000)):
        logits, u = rows_of(rng, rows, vocab, torch.float32), torch.rand(rows, device="cuda")
        k, p = torch.full((rows,), 40, dtype=torch.int32, device="cuda"), torch.full((rows,), 0.9, device="cuda")
        tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        space = torch.empty(sampling.sample_workspace(rows, vocab) + 16, dtype=torch.uint8, device="cuda")
        call = lambda out: sampling.sample(logits, u, out, top_k=k, top_p=p, workspace=space)  # noqa: E731
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            assert call(tokens) == OK
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert call(tokens) == OK
        for _ in range(3):
            logits.copy_(rows_of(rng, rows, vocab, torch.float32))
            u.copy_(torch.rand(rows))
            tokens.fill_(-7)
            graph.replay()
            eager = torch.empty_like(tokens)
            torch.cuda.synchronize()
            assert call(eager) == OK
            assert torch.equal(tokens, eager)
            l = logits.cpu().numpy().astype(np.float64)
            assert tokens.tolist() == [draw(l[r], 1.0, 40, float(np.float32(0.9)), 0.0, float(u[r]))[0] for r in range(rows)]
