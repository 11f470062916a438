"""Embedding: lookup with scaling, and the weight's gradient by sorted tokens, against the definition."""
import math

import pytest
import torch

from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, close, d, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def draw(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def words(seed, rows, vocab, how="text"):
    g = torch.Generator().manual_seed(seed)
    if how == "one":
        return torch.full((rows,), vocab // 2).cuda()
    if how == "each":
        return torch.randperm(vocab, generator=g)[:rows].cuda()
    if how == "pairs":  # runs of two, half of them across a unit of an even number of rows
        return ((torch.arange(rows) + 1) // 2 % vocab).cuda()
    u = torch.rand(rows, generator=g).double()
    t = torch.exp(u * math.log(vocab + 1)).long().sub_(1).clamp_(0, vocab - 1)
    if how == "padded":
        t[torch.rand(rows, generator=g) < 0.3] = -1
        t[torch.rand(rows, generator=g) < 0.1] = vocab
        t[:1] = -(1 << 40)
        t[-1:] = 1 << 32  # a word's number in the low 32 bits
    return t.cuda()


def check_backward(got, dy, tokens, vocab, scale, rows, what):
    t = tokens.cpu().long()
    seen = (t >= 0) & (t < vocab)
    want = torch.zeros(vocab, dy.shape[1], dtype=torch.float64).index_add_(0, t[seen], d(dy)[seen] * scale)
    size = torch.zeros_like(want).index_add_(0, t[seen], d(dy)[seen].abs() * abs(scale))
    # at most 64 rows summed in 32 bits, the sum of those sums and its product with the scale rounded once each
    close(got, want, 66 * E * size + 2.0 ** -140, what)
    unseen = torch.ones(vocab, dtype=torch.bool)
    unseen[t[seen]] = False
    assert not bool(d(got)[unseen].any()), what


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
@pytest.mark.parametrize("rows,vocab,dim", [(1, 1, 1), (3, 5, 7), (1, 1000, 4096), (40, 50, 8), (17, 9, 64), (130, 300, 129),
                                            (33, 100, 500), (1000, 37, 65), (2049, 90, 40), (5, 3, 9001)])
def test_over_sizes(kind, index, rows, vocab, dim):
    t = TYPES[kind]
    op = gd.Embedding(vocab, dim, t, scale=1.5, max_rows=rows)
    weight, dy = draw(1, vocab, dim, dtype=t), draw(2, rows, dim, dtype=t)
    for how in ("text", "padded") if index is torch.int64 else ("text",):
        tokens = words(3, rows, vocab, how)
        y = op.forward(tokens.to(index), weight)
        seen = ((tokens >= 0) & (tokens < vocab)).cpu()
        want = torch.zeros(rows, dim, dtype=torch.float64)
        want[seen] = d(weight)[tokens.cpu()[seen]] * 1.5
        close(y, want, rounded(want, t) + E * want.abs(), "y")
        assert not bool(d(y)[~seen].any())
        dw = op.backward(dy, tokens.to(index))
        check_backward(dw, dy, tokens, vocab, 1.5, rows, f"{kind} {rows} {vocab} {dim} {how}")


# one launch up to 4,096 rows; sorted: units of 8 to 32 rows, one chunk of 4,096 and several, the last one full or of one
# row; runs over many units
@pytest.mark.parametrize("how", ["text", "one", "each", "pairs", "padded"])
@pytest.mark.parametrize("rows,dim", [(7, 20), (8, 20), (9, 20), (15, 20), (16, 20), (17, 300), (2048, 24), (2049, 24), (4096, 12), (4097, 12), (6144, 260), (257, 8200), (2049, 1040), (4096, 520), (300, 8192), (1500, 8200), (8192, 8),
                                      (16384, 5), (16385, 5), (30001, 9)])
def test_backward_over_rows(how, rows, dim):
    vocab = max(rows, 700) if how in ("each", "pairs") else 700
    tokens, dy = words(5, rows, vocab, how), draw(6, rows, dim, dtype=torch.bfloat16)
    op = gd.Embedding(vocab, dim, scale=0.5, max_rows=40_000)
    dw = op.backward(dy, tokens)
    check_backward(dw, dy, tokens, vocab, 0.5, rows, f"{how} {rows}")
    assert torch.equal(op.backward(dy, tokens), dw)  # the same bits again


@pytest.mark.parametrize("rows", [7, 8, 9, 16, 17, 25])
@pytest.mark.parametrize("how", ["text", "one", "pairs", "padded"])
def test_backward_of_few_long_rows(how, rows):
    """Sorted, in one unit, one and a row, and several."""
    vocab, dim = 12, (1 << 21) // rows + 1
    tokens, dy = words(5, rows, vocab, how), draw(6, rows, dim)
    dw = gd.Embedding(vocab, dim, torch.float32, max_rows=rows).backward(dy, tokens)
    check_backward(dw, dy, tokens, vocab, 1.0, rows, f"{how} {rows}")


@pytest.mark.parametrize("how", ["text", "one", "padded"])
@pytest.mark.parametrize("dim", [3, 8, 261])
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_runs_over_very_many_units(kind, dim, how):
    """More units than 64 times 64, which the search for a run's end takes in steps of."""
    rows, vocab, t = 140_001, 300, TYPES[kind]
    tokens, dy = words(5, rows, vocab, how), draw(6, rows, dim, dtype=t)
    dw = gd.Embedding(vocab, dim, t, max_rows=rows).backward(dy, tokens)
    check_backward(dw, dy, tokens, vocab, 1.0, rows, f"{kind} {dim} {how}")


@pytest.mark.parametrize("rows", [3000, 9000])
@pytest.mark.parametrize("dim", [5, 520])
def test_rows_that_no_token_names_do_not_matter(rows, dim):
    """NaN in the rows of padding, most of the batch; words of few rows and of many."""
    tokens, dy = words(5, rows, 40, "text"), draw(6, rows, dim)
    tokens[torch.arange(rows) % 5 != 0] = -1
    dy[tokens < 0] = math.nan
    dw = gd.Embedding(40, dim, torch.float32, max_rows=rows).backward(dy, tokens)
    check_backward(dw, dy, tokens, 40, 1.0, rows, f"{rows} {dim}")


@pytest.mark.parametrize("dim", [1, 3, 7, 9, 130, 1000, 5001])
@pytest.mark.parametrize("how", ["text", "one"])
def test_words_of_many_rows_added_to_what_is_there(dim, how):
    """A word's columns shared by blocks: rows below a vector, ends inside one, rows of dweight that lie apart."""
    rows, vocab = 1800, 20
    tokens, dy = words(5, rows, vocab, how), draw(6, rows, dim, dtype=torch.bfloat16)
    op = gd.Embedding(vocab, dim, max_rows=rows)
    check_backward(op.backward(dy, tokens), dy, tokens, vocab, 1.0, rows, f"{dim} {how}")
    wide = torch.full((vocab, dim + 3), 2.0, device="cuda")
    op.backward(dy, tokens, dweight=wide[:, :dim], accumulate=True)
    size = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens.cpu(), d(dy).abs())
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens.cpu(), d(dy)) + 2.0
    close(wide[:, :dim], want, 67 * E * (size + 2.0), f"{dim} {how}")
    assert bool((wide[:, dim:] == 2.0).all())


def test_a_plan_of_just_these_rows():
    """Scratch for max_rows holds the most units that any smaller number of rows makes."""
    for most in (1, 16, 17, 4000, 4096, 5000, 8191, 9000, 16384, 16385, 33000):
        dim = 529 if 3900 < most < 8000 else 33
        op = gd.Embedding(64, dim, torch.float32, max_rows=most)
        for rows in {most, min(most, 4096), min(most, 16384)}:
            dy, tokens = draw(1, rows, dim), words(2, rows, 64, "text")
            check_backward(op.backward(dy, tokens), dy, tokens, 64, 1.0, rows, f"{rows} of {most}")


@pytest.mark.parametrize("rows", [1, 8, 9, 64, 65, 700, 3000, 4096, 5000])
def test_whole_numbers_are_summed_exactly(rows):
    vocab, dim = 30, 70
    dy = torch.randint(-8, 9, (rows, dim), generator=torch.Generator().manual_seed(1)).float().cuda()
    tokens = words(2, rows, vocab)
    dw = gd.Embedding(vocab, dim, torch.float32, scale=-2.0).backward(dy, tokens)
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens.cpu(), d(dy) * -2.0)
    assert torch.equal(d(dw), want)


@pytest.mark.parametrize("rows", [1, 60, 3000])
def test_accumulate_and_strides(rows):
    """Slices of wider buffers off any alignment; with accumulate rows of tokens that do not occur stay as they are."""
    vocab, dim = 90, 37
    tokens = words(1, rows, vocab)
    dy = draw(2, rows, dim + 3)[:, 2:2 + dim]
    weight = draw(3, vocab * 41 + 1)[1:].view(vocab, 41)[:, :dim]
    op = gd.Embedding(vocab, dim, torch.float32, max_rows=rows)
    out = torch.full((rows, dim + 5), 9.0, device="cuda")
    y = op.forward(tokens, weight, out=out[:, 1:1 + dim])
    assert torch.equal(y, weight[tokens]) and bool((out[:, :1] == 9).all() and (out[:, 1 + dim:] == 9).all())
    dw = op.backward(dy, tokens)
    check_backward(dw, dy, tokens, vocab, 1.0, rows, "strided")
    wide = torch.full((vocab, dim + 6), 0.25, device="cuda")
    op.backward(dy, tokens, dweight=wide[:, 3:3 + dim])
    assert torch.equal(wide[:, 3:3 + dim], dw) and bool((wide[:, :3] == 0.25).all() and (wide[:, 3 + dim:] == 0.25).all())
    flat = draw(4, vocab * dim + 1)
    was = d(flat)[1:].view(vocab, dim)
    op.backward(dy, tokens, dweight=flat[1:].view(vocab, dim), accumulate=True)
    close(flat[1:].view(vocab, dim), was + d(dw), E * d(dw).abs() + E * (was + d(dw)).abs(), "accumulated")
    unseen = torch.ones(vocab, dtype=torch.bool)
    unseen[tokens.cpu()] = False
    assert torch.equal(d(flat)[1:].view(vocab, dim)[unseen], was[unseen])


def test_no_rows_and_only_padding():
    vocab, dim = 20, 33
    op, weight = gd.Embedding(vocab, dim, torch.float32, max_rows=100), draw(1, vocab, dim)
    none, grad = torch.empty(0, dtype=torch.int64, device="cuda"), draw(2, vocab, dim)
    was = grad.clone()
    assert op.forward(none, weight).shape == (0, dim)
    op.backward(torch.empty(0, dim, device="cuda"), none, dweight=grad, accumulate=True)
    assert torch.equal(grad, was)
    pad, dy = torch.full((100,), -1, device="cuda"), torch.full((100, dim), math.nan, device="cuda")
    op.backward(dy, pad, dweight=grad, accumulate=True)
    assert torch.equal(grad, was) and not bool(op.forward(pad, weight).any())
    assert not bool(op.backward(dy, pad, dweight=grad).any())
    grad.fill_(1.0)
    assert not bool(op.backward(torch.empty(0, dim, device="cuda"), none, dweight=grad).any())


def test_padding_and_values_that_are_not_finite():
    vocab, dim = 12, 16
    tokens = torch.tensor([3, -1, 3, 5, 12], device="cuda")
    dy = draw(1, 5, dim)
    dy[1], dy[4], dy[3, 2] = math.nan, math.inf, math.inf
    dw = gd.Embedding(vocab, dim, torch.float32).backward(dy, tokens)
    assert bool(dw[5, 2].isinf()) and int((~dw.isfinite()).sum()) == 1
    weight = draw(2, vocab, dim)
    weight[0], weight[11] = math.nan, math.nan  # rows that padding must not read its zeros from
    y = gd.Embedding(vocab, dim, torch.float32, scale=2.0).forward(tokens, weight)
    assert torch.equal(y[0], 2 * weight[3]) and not bool(y[[1, 4]].any())


def test_shapes_of_tokens_and_offsets_past_32_bits():
    tokens = words(1, 24, 50).view(2, 3, 4)
    weight = draw(2, 50, 16)
    assert torch.equal(gd.Embedding(50, 16, torch.float32).forward(tokens, weight), weight[tokens])
    vocab, dim = 70_000, 65_536  # 9.2 GB in 16 bits: rows behind 2^32 bytes and 2^32 elements
    weight = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, 32_768, 65_537, 69_999], device="cuda")
    rows = draw(3, 4, dim, dtype=torch.bfloat16)
    weight[ids] = rows
    op = gd.Embedding(vocab, dim, max_rows=8)
    assert torch.equal(op.forward(ids, weight), rows)
    del weight
    dw = op.backward(rows, ids)
    assert torch.equal(dw[ids], rows.float())
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    rest[ids] = False
    assert not any(bool(dw[a:a + 5000][rest[a:a + 5000]].any()) for a in range(0, vocab, 5000))


def test_another_stream_and_graph_replays():
    rows, vocab, dim = 3000, 500, 120
    tokens, dy, weight = words(1, rows, vocab), draw(2, rows, dim), draw(3, vocab, dim)
    op = gd.Embedding(vocab, dim, torch.float32)
    y, dw = op.forward(tokens, weight), op.backward(dy, tokens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, dw2 = op.forward(tokens, weight, stream=s), op.backward(dy, tokens, stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(dw, dw2)
    out, grad = torch.empty_like(y), torch.empty_like(dw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(tokens, weight, out=out)
        op.backward(dy, tokens, dweight=grad)
    for seed in range(4):
        tokens.copy_(words(10 + seed, rows, vocab, "padded" if seed % 2 else "text"))
        graph.replay()
        y, dw = op.forward(tokens, weight), op.backward(dy, tokens)
        torch.cuda.synchronize()
        assert torch.equal(out, y) and torch.equal(grad, dw)


def test_gradient_against_differences():
    """The loss is linear in the weight, so differences are exact up to rounding in 64 bits."""
    vocab, dim, rows = 6, 5, 9
    tokens, c = words(1, rows, vocab), draw(2, rows, dim)
    dw = gd.Embedding(vocab, dim, torch.float32, scale=3.0).backward(c, tokens)
    w = torch.zeros(vocab, dim, dtype=torch.float64)
    for k in range(vocab * dim):
        e = w.clone()
        e.view(-1)[k] = 1.0
        assert abs(float((3.0 * e[tokens.cpu()] * d(c)).sum()) - float(dw.view(-1)[k])) < 1e-5  # sums of 9 values below 4, times 3


def test_refusals():
    op = gd.Embedding(10, 8, torch.float32, max_rows=4)
    weight, tokens = draw(1, 10, 8), torch.tensor([1, 2], device="cuda")
    for bad in (lambda: op.forward(tokens.float(), weight), lambda: op.forward(tokens.cpu(), weight),
                lambda: op.forward(tokens, weight.bfloat16()), lambda: op.forward(torch.arange(8, device="cuda")[::2], weight),
                lambda: op.backward(draw(2, 2, 8, dtype=torch.bfloat16), tokens)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: op.forward(tokens, weight[:9]), lambda: op.forward(tokens, weight[:, :7]),
                lambda: op.forward(tokens, weight, out=weight[:2]), lambda: op.backward(draw(2, 3, 8), tokens),
                lambda: op.backward(draw(2, 2, 8), tokens, accumulate=True),
                lambda: op.backward(draw(2, 2, 8), tokens, dweight=draw(3, 9, 8))):
        with pytest.raises(ValueError):
            bad()
    five = torch.arange(5, device="cuda")
    assert torch.equal(op.forward(five, weight), weight[:5])  # max_rows is the backward's
    for bad in (lambda: op.backward(draw(2, 5, 8), five), lambda: gd.Embedding(0, 8), lambda: gd.Embedding(10, (1 << 20) + 1),
                lambda: gd.Embedding(10, 8, scale=math.inf).forward(tokens, weight.bfloat16())):
        with pytest.raises(gd.GDError):
            bad()
    with pytest.raises(RuntimeError):
        op.forward(tokens, weight.clone().requires_grad_())
