"""Log probabilities and the distance to a teacher where a scale meets logits of large magnitude: rows of the type's lowest
value, of -1e30, of +1e10, and ordinary ones beside them, against the 64-bit definitions.  A scale that is no power of two
rounds the product with such a logit by more than all differences that matter; one above 1 takes the product past binary32."""
import dataclasses
import math

import pytest
import torch

from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, close, d
from test_gpu_scores import check_distill, check_gradient, draw, exp_error, ids_of, sum_error, teacher64, tokens64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def extremes(seed, rows, vocab, dtype):
    """Rows of every kind in turn; float16 has what its range holds of them."""
    x = draw(seed, rows, vocab, scale=3.0)
    g = torch.Generator().manual_seed(seed + 50)
    some = (torch.rand(rows, vocab, generator=g) < 0.1).cuda()
    lowest, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    big = min(1e10, most)
    kinds = [
        lambda r: r.fill_(lowest),                                       # a mask that leaves nothing
        lambda r: r.fill_(max(-1e30, lowest)),
        lambda r: r.fill_(-big),
        lambda r: r.index_fill_(0, torch.tensor([vocab // 3]).cuda(), big),
        lambda r: r.masked_fill_(~some[0], lowest),
        lambda r: r.masked_fill_(some[0], -math.inf).masked_fill_(~some[0], lowest),
        lambda r: r.fill_(big).masked_fill_(some[0], big * (1 - 2.0 ** -7)),
        lambda r: r.fill_(most),
        lambda r: r.add_(1000.0),
        lambda r: r.fill_(-math.inf),
        lambda r: r,
    ]
    for row in range(rows):
        kinds[row % len(kinds)](x[row])
    return x.to(dtype)


def past32(v):
    """What a result in binary32 is where the definition's is past its range; others as they are."""
    return torch.where(v.abs() > torch.finfo(torch.float32).max, v * math.inf, v)


# one wave a row, of one turn and several; four waves; eight; rows in pieces
SHAPES = [(11, 5), (11, 40), (11, 2000), (11, 5000), (300, 9000), (1100, 2100), (11, 30_000), (2, 85_000), (260, 51_000)]
SCALES = [0.7, 1.0, 1.3, 2.0, 0.001]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_tokens(kind, rows, vocab):
    t = TYPES[kind]
    x, tokens, g, h = extremes(1, rows, vocab, t), ids_of(2, vocab, rows), draw(3, rows), draw(4, rows)
    tokens[3::11] = vocab // 3
    for scale in SCALES if rows < 100 else SCALES[:1] + SCALES[2:3]:
        scale32 = float(torch.tensor(scale, dtype=torch.float32))
        op, what = gd.TokenLogProbs(vocab, t, scale=scale, max_rows=rows), f"{kind} {rows}x{vocab} {scale}"
        top = min(64, vocab)
        r = op.forward(x, tokens, top=top, keep_stats=True)
        rel, lse, p, lp, logp, entropy, seen, none = tokens64(x, tokens, scale32)
        off = sum_error(p, rel)[:, 0]
        for got in (r, op.forward_backward(x, tokens, g, h)[0]):
            close(got.logp, past32(logp), off + 2 * E * torch.where(logp.isfinite(), logp, 0.0).abs(), what + " logp")
            close(got.entropy, entropy, 3 * off + (p * lp.abs() * (exp_error(rel) + 40 * E)).sum(1) + 40 * E * (1 + entropy), what + " entropy")
        order = torch.sort(d(x), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_ids.cpu(), order), what
        want = torch.where(none[:, None], -math.inf, rel.gather(1, order))
        close(r.top_logp, past32(want), off[:, None] + 3 * E * (torch.where(want.isfinite(), want, 0.0).abs() + 12), what + " alternatives")
        for dh in (None, h):
            check_gradient(op.backward(x, tokens, g, dh, scores=r), x, tokens, g, dh, scale32, what + " given")
            dx = op.forward_backward(x, tokens, g, dh)[1]
            check_gradient(dx, x, tokens, g, dh, scale32, what + " in one")
            here = x.clone()
            op.backward(here, tokens, g, dh, out=here, scores=dataclasses.replace(r))
            check_gradient(here, x, tokens, g, dh, scale32, what + " given, in place")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("top", [1, 5, 130])
def test_teacher(kind, rows, vocab, top):
    t = TYPES[kind]
    x, ids, g = extremes(1, rows, vocab, t), ids_of(2, vocab, rows, top), draw(3, rows)
    ids[3::11, 0] = vocab // 3
    teacher = draw(4, rows, top, scale=2.0)
    for row in range(0, rows, 5):  # teachers whose logits are as large
        teacher[row] = (torch.finfo(torch.float32).min, -1e30, 1e10, torch.finfo(torch.float32).max)[row // 5 % 4]
    for scale in SCALES if rows < 100 else SCALES[:1] + SCALES[2:3]:
        scale32 = float(torch.tensor(scale, dtype=torch.float32))
        op, what = gd.Distill(vocab, t, scale=scale, max_rows=rows), f"{kind} {rows}x{vocab} {top} {scale}"
        loss, stats = op.forward(x, ids, teacher, keep_stats=True)
        want = teacher64(x, ids, teacher, scale32)[5]
        for loss, dx in ((loss, op.backward(x, ids, teacher, g, stats=stats)), op.forward_backward(x, ids, teacher, g)):
            past = past32(want).isinf() & want.isfinite()
            assert bool((loss.cpu()[past] == past32(want)[past]).all()), what
            check_distill(torch.where(past, want, d(loss)), dx, x, ids, teacher, g, scale32, what)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_stats_of_ordinary_rows_add_up(kind):
    """Two numbers whose sum is the log of the sum, at any scale, up to magnitudes of 2^24."""
    rows, vocab, t = 6, 5000, TYPES[kind]
    x = draw(1, rows, vocab, scale=3.0)
    for row, at in enumerate((0.0, 100.0, -5000.0, 60_000.0, -60_000.0, 9.0)):
        x[row] += at
    x = x.to(t)
    for scale in (0.7, 1.3, 200.0):
        scale32 = float(torch.tensor(scale, dtype=torch.float32))
        r = gd.TokenLogProbs(vocab, t, scale=scale, max_rows=rows).forward(x, ids_of(2, vocab, rows), keep_stats=True)
        rel, lse, p, *_ = tokens64(x, ids_of(2, vocab, rows), scale32)
        # the log's error, and its rounding beside the rest of the largest product, which is below 1
        close(d(r.stats).sum(1), lse[:, 0], sum_error(p, rel)[:, 0] + 14 * E, f"{kind} {scale}")


@pytest.mark.parametrize("rows,vocab", [(5, 300), (300, 9000), (2, 30_000)])
@pytest.mark.parametrize("scale", [1e30, 1e-30])
def test_scales_of_any_size(rows, vocab, scale):
    """Ordinary logits: one of them is certain, or all are as likely as one another."""
    x, tokens, g, h = draw(1, rows, vocab, scale=3.0), ids_of(2, vocab, rows), draw(3, rows), draw(4, rows)
    ids, teacher = ids_of(5, vocab, rows, 3), draw(6, rows, 3)
    scale32 = float(torch.tensor(scale, dtype=torch.float32))
    op, ds = (kind(vocab, torch.float32, scale=scale, max_rows=rows) for kind in (gd.TokenLogProbs, gd.Distill))
    r = op.forward(x, tokens, keep_stats=True)
    rel, _, p, _, logp, *_ = tokens64(x, tokens, scale32)
    close(r.logp, logp, sum_error(p, rel)[:, 0] + 2 * E * logp.abs(), "logp")
    for dh in (None, h):
        check_gradient(op.backward(x, tokens, g, dh, scores=r), x, tokens, g, dh, scale32, "given")
        check_gradient(op.forward_backward(x, tokens, g, dh)[1], x, tokens, g, dh, scale32, "in one")
    loss, dx = ds.forward_backward(x, ids, teacher, g)
    check_distill(loss, dx, x, ids, teacher, g, scale32, "teacher")
