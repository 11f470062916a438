"""Log probabilities of tokens with entropy and alternatives, the distance to a teacher's top logits, and their
gradients, against the 64-bit definitions."""
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


def ids_of(seed, vocab, *shape, padded=False):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, vocab, shape, generator=g)
    if padded:
        t = torch.where(torch.rand(shape, generator=g) < 0.25, torch.tensor([-1, vocab, 1 << 32])[torch.randint(0, 3, shape, generator=g)], t)
    return t.cuda()


def softmax64(x, scale):
    """(z less what the largest and the log of the sum come to, largest, lse, p) in 64 bits; empty rows have p of 0.  The
    first is formed with the largest taken off before the log, which vanishes beside the lowest value of binary32."""
    z = d(x) * scale
    most = z.amax(1, keepdim=True)
    to = torch.where(most.isinf(), 0.0, most)
    e = torch.exp(z - to)
    total = e.sum(1, keepdim=True)
    return (z - to) - torch.log(total), most, to + torch.log(total), torch.where(total > 0, e / total, 0.0)


def exp_error(lp):
    """Relative error of p = exp(z - lse) in 32 bits.  z - largest is formed with one rounding (relative to it), less the
    log of the sum with one more, multiplied by log2 e with two, each relative to |z - lse| at most 2^-24 (the largest is
    within log V <= 12 of lse, so that difference is at most |z - lse| + 12), and the hardware's exponential errs by 2^-22.
    The sum errs by the same in its terms, weighted, by a rounding per term of a thread's (at most 400) and 14 to join."""
    a = lp.abs()
    a = torch.where(a.isfinite(), a, 0.0)
    return 4 * E * (a + 12) + 4 * E


def sum_error(p, lp):
    return (p * exp_error(lp)).sum(1, keepdim=True) + 32 * E  # roundings of a sum of 400 positive terms, well within


def tokens64(x, t, scale):
    rel, most, lse, p = softmax64(x, scale)
    t = t.reshape(-1).cpu().long()
    seen = (t >= 0) & (t < x.shape[1])
    at = rel.gather(1, torch.where(seen, t, 0)[:, None])
    none = most == -math.inf
    logp = torch.where(seen[:, None], torch.where(none, -math.inf, at), 0.0)[:, 0]
    lp = torch.where(p > 0, rel, 0.0)
    entropy = -(p * lp).sum(1)
    return rel, lse, p, lp, logp, entropy, seen, none[:, 0]


def check_scores(r, x, t, scale, top, what):
    rel, lse, p, lp, logp, entropy, seen, none = tokens64(x, t, scale)
    off = sum_error(p, rel)[:, 0]  # of log s
    fine = torch.where(logp.isfinite(), logp, 0.0).abs()
    close(r.logp.reshape(-1), logp, off + 2 * E * fine, what + " logp")
    if r.entropy is not None:
        # log s - t / s: their errors, and of a term p lp its own; the roundings of t's sum are relative to its magnitude
        close(r.entropy.reshape(-1), entropy, 3 * off + (p * lp.abs() * (exp_error(rel) + 40 * E)).sum(1) + 40 * E * (1 + entropy), what + " entropy")
    if r.stats is not None:
        stats = d(r.stats).reshape(-1, 2)
        want = torch.where(none, -math.inf, lse[:, 0])
        close(stats.sum(1), want, off + 2 * E * torch.where(none, 0.0, lse[:, 0]).abs(), what + " lse")
    if top:
        order = torch.sort(d(x), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_ids.reshape(-1, top).cpu(), order), what + " alternatives"
        want = rel.gather(1, order)
        want = torch.where(none[:, None], -math.inf, want)
        fine = torch.where(want.isfinite(), want, 0.0).abs()
        close(r.top_logp.reshape(-1, top), want, off[:, None] + 3 * E * (fine + 12), what + " alternatives")


def check_gradient(got, x, t, g, h, scale, what):
    rel, lse, p, lp, logp, entropy, seen, none = tokens64(x, t, scale)
    g64 = torch.where(seen, d(g), 0.0)[:, None]
    one = torch.zeros_like(p)
    one[torch.arange(len(seen)), torch.where(seen, t.reshape(-1).cpu().long(), 0)] = 1.0
    h64 = torch.zeros_like(g64) if h is None else d(h)[:, None]
    want = scale * (g64 * (one - p) - h64 * p * (lp + entropy[:, None]))
    want[none] = 0.0
    perr = exp_error(rel) + sum_error(p, rel)
    inner = (g64.abs() + h64.abs() * (lp.abs() + entropy[:, None])) * p * (perr + 6 * E) + g64.abs() * one * 4 * E
    inner = inner + h64.abs() * p * (3 * sum_error(p, rel) + 60 * E * (1 + entropy[:, None]) + 8 * E * (lp.abs() + 12))
    # the hardware's exponential gives 0 below 2^-126
    close(got.reshape(want.shape), want, rounded(want, got.dtype) + scale * inner + scale * 2.0 ** -125 * (g64.abs() + 100 * h64.abs()), what)


# widths of every launch shape (one, four, eight waves a row, rows in pieces), ragged ones, shorter than a vector
WIDTHS = [1, 2, 7, 8, 9, 64, 513, 2048, 2049, 5000, 8192, 8193, 20_000]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(3, v) for v in WIDTHS] + [(1, 85_000), (2, 32_001), (130, 9000), (300, 9001), (5, 100_003)])
def test_tokens_over_sizes(kind, rows, vocab):
    t = TYPES[kind]
    x = draw(1, rows, vocab, dtype=t, scale=3.0)
    for padded, scale in ((False, 1.0), (True, 0.7)):
        tokens = ids_of(2, vocab, rows, padded=padded)
        op = gd.TokenLogProbs(vocab, t, scale=scale, max_rows=rows)
        scale32 = float(torch.tensor(scale, dtype=torch.float32))
        what = f"{kind} {rows}x{vocab} {padded}"
        for top in sorted({0, 1, min(5, vocab), min(64, vocab)}):
            r = op.forward(x, tokens, top=top, keep_stats=True)
            check_scores(r, x, tokens, scale32, top, what)
        assert op.forward(x, tokens.int() if not padded else tokens, entropy=False).entropy is None
        g, h = draw(3, rows), draw(4, rows)
        for dh in (None, h):
            dx = op.backward(x, tokens, g, dh, scores=r)
            check_gradient(dx, x, tokens, g, dh, scale32, what + " given")
            r2, dx2 = op.forward_backward(x, tokens, g, dh)
            check_gradient(dx2, x, tokens, g, dh, scale32, what + " in one")
            check_scores(r2, x, tokens, scale32, 0, what + " in one")
            here = x.clone()
            assert op.backward(here, tokens, g, dh, out=here) is here
            assert torch.equal(here, dx2), what + " in place"


def masked(seed, rows, vocab, dtype, share, value=-math.inf):
    x = draw(seed, rows, vocab, dtype=dtype, scale=3.0)
    g = torch.Generator().manual_seed(seed + 100)
    return x.masked_fill_((torch.rand(rows, vocab, generator=g) < share).cuda(), value)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(6, 40), (6, 3000), (6, 8192), (6, 30_000), (300, 10_000)])
def test_masks(kind, rows, vocab):
    """Minus infinity and the type's lowest value in most places; rows of one element, of none, of only the lowest value."""
    t = TYPES[kind]
    op = gd.TokenLogProbs(vocab, t, max_rows=rows)
    tokens = ids_of(1, vocab, rows)
    g, h = draw(3, rows), draw(4, rows)
    x = masked(2, rows, vocab, t, 0.9)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, tokens[1]] = 2.0
    x[2, tokens[2]] = -math.inf
    x[3, tokens[3]] = 1.0
    for y in (x, x.clone()):
        if y is not x:
            y[3] = torch.finfo(t).min  # as likely as one another
            y[4].masked_fill_(y[4] == -math.inf, torch.finfo(t).min)
        r = op.forward(y, tokens, top=min(64, vocab), keep_stats=True)
        check_scores(r, y, tokens, 1.0, min(64, vocab), "masked")
        assert float(r.logp[0]) == -math.inf and float(r.logp[1]) == 0.0 and float(r.entropy[:2].abs().sum()) == 0
        assert float(r.logp[2]) == -math.inf
        for dh in (None, h):
            dx = op.backward(y, tokens, g, dh, scores=r)
            check_gradient(dx, y, tokens, g, dh, 1.0, "masked")
            # not the same bits: the one takes the sum of a row, the other the exponential of its log, as rounded
            again = op.forward_backward(y, tokens, g, dh)[1]
            check_gradient(again, y, tokens, g, dh, 1.0, "masked")
            assert not bool(dx[0].any() or again[0].any())


@pytest.mark.parametrize("rows,vocab", [(3, 500), (3, 2048), (1030, 2100), (2, 5000), (2, 8191), (300, 9000), (2, 40_000), (300, 110_000)])
@pytest.mark.parametrize("value", [-math.inf, torch.finfo(torch.bfloat16).min, -3.0])
@pytest.mark.parametrize("left", [0, 1, 5, 70, 300])
def test_few_words_that_a_mask_leaves(rows, vocab, value, left):
    """Most of a row equal: the alternatives are what is above, then the first of the others."""
    x = torch.full((rows, vocab), value)
    g = torch.Generator().manual_seed(left)
    for row in range(rows):
        x[row, torch.randperm(vocab, generator=g)[:left] if row % 3 else torch.arange(left) + vocab - left] = torch.randn(left, generator=g)
    x, tokens = x.bfloat16().cuda(), ids_of(1, vocab, rows)
    for top in (1, 4, 64):
        check_scores(gd.TokenLogProbs(vocab, max_rows=rows).forward(x, tokens, top=top), x, tokens, 1.0, top, "few")


@pytest.mark.parametrize("rows,vocab", [(3, 30), (3, 2048), (2, 5000), (300, 9000), (2, 40_000)])
def test_ties_go_to_the_lower_id(rows, vocab):
    """Rows of equal logits, of zeros of both signs, of few values: more elements at the bound than a list holds."""
    top = min(64, vocab)
    op = gd.TokenLogProbs(vocab, max_rows=rows)
    tokens = ids_of(1, vocab, rows)
    g = torch.Generator().manual_seed(5)
    for x in (torch.full((rows, vocab), 1.5), torch.where(torch.rand(rows, vocab, generator=g) < 0.5, 0.0, -0.0),
              torch.randint(0, 3, (rows, vocab), generator=g).float(), torch.arange(vocab).float().expand(rows, vocab) // 100,
              -(torch.arange(vocab).float().expand(rows, vocab) // 7)):
        x = x.bfloat16().cuda()
        check_scores(op.forward(x, tokens, top=top), x, tokens, 1.0, top, "ties")


@pytest.mark.parametrize("vocab", [50, 3000, 20_000])
def test_values_that_are_not_finite(vocab):
    """A row with an infinity or a NaN has NaN, its neighbours are as without it; padding passes no gradient from it."""
    rows = 6
    x, tokens = draw(1, rows, vocab), ids_of(2, vocab, rows)
    clean = x.clone()
    x[0, 3], x[2, 7], x[4, 9] = math.nan, math.inf, math.nan
    x[4] = math.nan
    op = gd.TokenLogProbs(vocab, torch.float32, max_rows=rows)
    r, want = op.forward(x, tokens, top=5, keep_stats=True), op.forward(clean, tokens, top=5, keep_stats=True)
    g, h = torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda")
    dx, dwant = op.backward(x, tokens, g, h, scores=r), op.backward(clean, tokens, g, h, scores=want)
    for row in range(rows):
        if row % 2:
            assert all(torch.equal(getattr(r, k)[row], getattr(want, k)[row]) for k in ("logp", "entropy", "stats", "top_logp", "top_ids"))
            assert torch.equal(dx[row], dwant[row])
        else:
            assert bool(r.logp[row].isnan() & r.entropy[row].isnan()) and bool(dx[row].isnan().any())
            assert bool((r.top_ids[row] >= 0).all() and (r.top_ids[row] < vocab).all())
    assert int(r.top_ids[0, 0]) == 3 and int(r.top_ids[2, 0]) == 7 and r.top_ids[4].tolist() == [0, 1, 2, 3, 4]
    pad = torch.full_like(tokens, -1)
    r, dx = op.forward_backward(x, pad, g)
    assert not bool(r.logp.any()) and not bool(dx.any())
    assert not bool(op.backward(x, tokens, torch.zeros_like(g)).any())


def teacher64(x, ids, teacher, scale):
    rel, most, lse, q = softmax64(x, scale)
    ids, a = ids.cpu().long(), d(teacher) * scale
    seen = (ids >= 0) & (ids < x.shape[1])
    a = torch.where(seen, a, -math.inf)
    top = a.amax(1, keepdim=True)
    top = torch.where(top.isinf(), 0.0, top)
    e = torch.exp(a - top)
    total = e.sum(1, keepdim=True)
    w = torch.where(total > 0, e / total, 0.0)
    log_w = torch.where(w > 0, a - top - torch.log(total), 0.0)
    at = rel.gather(1, torch.where(seen, ids, 0))
    none = (most == -math.inf)[:, 0]
    part = torch.where(w > 0, w * (log_w - at), 0.0)
    loss = torch.where(none & (total[:, 0] > 0), math.inf, part.sum(1))
    return rel, lse, q, w, log_w, loss, seen, none, part, total[:, 0] > 0


def check_distill(loss, dx, x, ids, teacher, g, scale, what):
    rel, lse, q, w, log_w, want, seen, none, part, named = teacher64(x, ids, teacher, scale)
    off = sum_error(q, rel)[:, 0]
    if loss is not None:
        # w and log w: a difference, a sum of at most 256 terms, the library's exp and log; the rest is formed in 64 bits
        size = torch.where(part.isfinite(), part, 0.0).abs().sum(1) + (w * log_w.abs()).sum(1)
        werr = 24 * E * (1 + (w * (log_w.abs() + 1)).sum(1))
        close(loss, want, off + E * torch.where(want.isfinite(), want, 0.0).abs() + werr * (1 + size), what + " loss")
    if dx is not None:
        G = d(g)[:, None]
        put = torch.zeros_like(q).scatter_add_(1, torch.where(seen, ids.cpu().long(), 0), w)
        full = scale * G * (torch.where(named[:, None], q, 0.0) - put)
        full[none] = 0.0
        qerr = exp_error(rel) + sum_error(q, rel)
        inner = scale * G.abs() * (q * (qerr + 6 * E) + put * (24 + w.shape[1]) * E)
        wrel = torch.zeros_like(q).scatter_add_(1, torch.where(seen, ids.cpu().long(), 0), w * log_w.abs()) * 4 * E
        close(dx.reshape(full.shape), full, rounded(full, dx.dtype) + inner + scale * G.abs() * (wrel + 2.0 ** -125), what + " dlogits")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,top", [(3, 1, 1), (4, 7, 3), (3, 8, 8), (5, 64, 16), (6, 2049, 64), (3, 9000, 65),
                                            (300, 8200, 32), (2, 32_000, 256), (1, 85_000, 20), (40, 3001, 128)])
def test_teacher_over_sizes(kind, rows, vocab, top):
    t = TYPES[kind]
    x, g = draw(1, rows, vocab, dtype=t, scale=3.0), draw(3, rows)
    for case, scale in (("plain", 1.0), ("padded", 0.5), ("twice", 1.0)):
        ids = ids_of(2, vocab if case != "twice" else min(vocab, max(1, top // 2)), rows, top, padded=case == "padded")
        teacher = draw(4, rows, top, scale=2.0, dtype=torch.float32 if case == "plain" else t)
        if case == "padded":
            teacher[:, ::3] = -math.inf
            teacher[0] = -math.inf  # names nothing
            ids[-1] = -1
            if rows > 2:
                ids[1, 0], teacher[1, 0] = 0, 1.0
        op = gd.Distill(vocab, t, scale=scale, max_rows=rows)
        what = f"{kind} {rows} {vocab} {top} {case}"
        loss, stats = op.forward(x, ids, teacher, keep_stats=True)
        dx = op.backward(x, ids, teacher, g, stats=stats)
        check_distill(loss, dx, x, ids, teacher, g, scale, what)
        loss2, dx2 = op.forward_backward(x, ids.int() if case == "plain" else ids, teacher, g)
        check_distill(loss2, dx2, x, ids, teacher, g, scale, what + " in one")
        here = x.clone()
        op.backward(here, ids, teacher, g, out=here)
        assert torch.equal(here, dx2)
        if case == "padded":
            assert float(loss[0]) == 0 and float(loss[-1]) == 0 and not bool(dx[0].any() or dx[-1].any())


@pytest.mark.parametrize("vocab", [30, 4000, 20_000])
def test_teacher_with_masks(vocab):
    rows, top = 5, 6
    x = masked(1, rows, vocab, torch.float32, 0.5)
    ids = torch.stack([torch.randperm(vocab, generator=torch.Generator().manual_seed(k))[:top] for k in range(rows)]).cuda()
    teacher, g = draw(2, rows, top), draw(3, rows)
    x.scatter_(1, ids, 1.0)
    x[0] = -math.inf       # an empty row
    x[1, ids[1, 2]] = -math.inf  # a named token that is masked
    x[2, 3] = math.nan
    teacher[3, 1] = -math.inf
    x[3, ids[3, 1]] = -math.inf  # masked, but not named either
    op = gd.Distill(vocab, torch.float32, max_rows=rows)
    loss, stats = op.forward(x, ids, teacher, keep_stats=True)
    assert float(loss[0]) == math.inf and float(loss[1]) == math.inf and bool(loss[2].isnan()) and bool(loss[3:].isfinite().all())
    for dx in (op.backward(x, ids, teacher, g, stats=stats), op.forward_backward(x, ids, teacher, g)[1]):
        assert not bool(dx[0].any()) and bool(dx[2].isnan().any()) and bool(dx[[1, 3, 4]].isfinite().all())
        keep = [0, 1, 3, 4]
        check_distill(loss[keep], dx[keep], x[keep], ids[keep], teacher[keep], g[keep], 1.0, "masked")


def test_gradients_against_differences():
    rows, vocab, top, scale = 3, 40, 5, 0.5
    x, tokens, g, h = draw(1, rows, vocab), ids_of(2, vocab, rows), draw(3, rows), draw(4, rows)
    ids, teacher = ids_of(5, vocab, rows, top), draw(6, rows, top)
    op, ds = gd.TokenLogProbs(vocab, torch.float32, scale=scale), gd.Distill(vocab, torch.float32, scale=scale)

    def score(v):
        *_, logp, entropy, _, _ = tokens64(v, tokens, scale)
        return float((d(g) * logp + d(h) * entropy).sum())

    def distance(v):
        return float((d(g) * teacher64(v, ids, teacher, scale)[5]).sum())

    step = 1e-6
    for f, dx in ((score, op.backward(x, tokens, g, h)), (distance, ds.backward(x, ids, teacher, g))):
        for k in range(0, rows * vocab, 7):
            ends = []
            for sign in (-1, 1):
                v = d(x).clone()
                v.view(-1)[k] += sign * step
                ends.append(f(v))
            # differences err by about 1e-16 / step and step^2, the kernel by some 2^-22 of values below 10
            assert abs((ends[1] - ends[0]) / (2 * step) - float(dx.view(-1)[k])) < 2e-5


@pytest.mark.parametrize("kind,vocab", [("bf16", 3001), ("f32", 9003)])
def test_strides_and_shapes(kind, vocab):
    t = TYPES[kind]
    wide = draw(1, 6, vocab + 9, dtype=t, scale=2.0)
    x = wide[:, 3:3 + vocab]
    tokens, g = ids_of(2, vocab, 6), draw(3, 6)
    op = gd.TokenLogProbs(vocab, t)
    want, dwant = op.forward(x.contiguous(), tokens, top=9), op.backward(x.contiguous(), tokens, g)
    r = op.forward(x, tokens, top=9)
    check_scores(r, x, tokens, 1.0, 9, "strided")
    out = torch.full((6, vocab + 5), 7.0, dtype=t, device="cuda")
    dx = op.backward(x, tokens, g, out=out[:, 1:1 + vocab])
    assert torch.equal(dx, dwant) and bool((out[:, :1] == 7).all() and (out[:, 1 + vocab:] == 7).all())
    before = wide.clone()
    op.backward(x, tokens, g, out=x)
    assert torch.equal(x, dwant) and torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 3 + vocab:], before[:, 3 + vocab:])
    shaped = op.forward(before[:, 3:3 + vocab].contiguous().view(2, 3, vocab), tokens.view(2, 3), top=4, keep_stats=True)
    assert shaped.logp.shape == (2, 3) and shaped.stats.shape == (2, 3, 2) and shaped.top_ids.shape == (2, 3, 4)
    assert torch.equal(shaped.logp.view(-1), want.logp) and torch.equal(shaped.top_ids.view(6, 4), want.top_ids[:, :4])
    again = op.forward(before[:, 3:3 + vocab], tokens, top=9, out=r)
    assert again is r and torch.equal(r.top_logp, want.top_logp)
    ids, teacher = ids_of(4, vocab, 6, 8), draw(5, 6, 8)
    ds = gd.Distill(vocab, t)
    loss, _ = ds.forward(before[:, 3:3 + vocab], ids[:, 1:6], teacher[:, 2:7])
    assert torch.equal(loss, ds.forward(before[:, 3:3 + vocab].contiguous(), ids[:, 1:6].contiguous(), teacher[:, 2:7].contiguous())[0])


def test_offsets_past_32_bits():
    rows, vocab = 34_000, 70_000  # 2.4e9 elements
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    tokens = torch.arange(rows, device="cuda")
    x[torch.arange(rows, device="cuda"), tokens] = 5.0
    op = gd.TokenLogProbs(vocab, max_rows=rows)
    r = op.forward(x, tokens, top=2)
    want = 5.0 - math.log(vocab - 1 + math.exp(5.0))
    # 1e-5: the sum of 70,000 terms of 1 and one of e^5 is within 400 roundings, so is its log; below 2^-24 * 400
    assert bool(((r.logp - want).abs() < 400 * E).all()) and torch.equal(r.top_ids[:, 0], tokens)
    assert torch.equal(r.top_ids[:, 1], (tokens == 0).long())
    op.backward(x, tokens, torch.ones(rows, device="cuda"), out=x)
    p = math.exp(want)
    rest = -1.0 / (vocab - 1 + math.exp(5.0))
    at = x[torch.arange(rows, device="cuda"), tokens].double()
    # bfloat16's rounding, and 32-bit errors a hundredth of it
    assert bool(((at - (1 - p)).abs() < 1.02 * 2.0 ** -8 * (1 - p)).all())
    assert bool(((x[:, -1].double() - rest).abs() < 1.02 * 2.0 ** -8 * abs(rest)).all())


@pytest.mark.parametrize("rows,vocab", [(300, 5000), (2, 30_000)])
def test_another_stream_and_graph_replays(rows, vocab):
    x, tokens, g, h = draw(1, rows, vocab, dtype=torch.bfloat16), ids_of(2, vocab, rows), draw(3, rows), draw(4, rows)
    ids, teacher = ids_of(5, vocab, rows, 7), draw(6, rows, 7)
    op, ds = gd.TokenLogProbs(vocab), gd.Distill(vocab)

    def everything(stream=None):
        r = op.forward(x, tokens, top=3, keep_stats=True, stream=stream)
        r2, dx = op.forward_backward(x, tokens, g, h, stream=stream)
        loss, stats = ds.forward(x, ids, teacher, keep_stats=True, stream=stream)
        return [r.logp, r.entropy, r.stats, r.top_logp, r.top_ids, r2.logp, r2.entropy, dx, loss,
                op.backward(x, tokens, g, h, scores=r, stream=stream), ds.backward(x, ids, teacher, g, stats=stats, stream=stream),
                *ds.forward_backward(x, ids, teacher, g, stream=stream)]

    want = everything()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = everything(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for seed in range(3):
        x.copy_(draw(10 + seed, rows, vocab, dtype=torch.bfloat16))
        tokens.copy_(ids_of(20 + seed, vocab, rows, padded=True))
        graph.replay()
        want = everything()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_no_rows():
    op, ds = gd.TokenLogProbs(100), gd.Distill(100)
    x, none = torch.empty(0, 100, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    f = torch.empty(0, device="cuda")
    assert op.forward(x, none, top=3).top_ids.shape == (0, 3) and op.backward(x, none, f).shape == (0, 100)
    assert ds.forward_backward(x, none.view(0, 1).expand(0, 4), torch.empty(0, 4, device="cuda"), f)[1].shape == (0, 100)


def test_refusals():
    rows, vocab = 4, 50
    op, ds = gd.TokenLogProbs(vocab, torch.float32, max_rows=rows), gd.Distill(vocab, torch.float32, max_rows=rows)
    x, tokens, g = draw(1, rows, vocab), ids_of(2, vocab, rows), draw(3, rows)
    ids, teacher = ids_of(4, vocab, rows, 3), draw(5, rows, 3)
    r = op.forward(x, tokens, keep_stats=True)
    assert op.forward(x, tokens).stats is None and ds.forward(x, ids, teacher)[1] is None
    for bad in (lambda: op.backward(x, tokens, g, scores=op.forward(x, tokens)), lambda: op.forward(x.bfloat16(), tokens), lambda: op.forward(x, tokens.float()), lambda: op.forward(x, tokens.cpu()),
                lambda: op.backward(x, tokens, g.double()), lambda: op.backward(x, tokens, g, g, scores=gd.LogProbs(r.logp, None, r.stats)),
                lambda: ds.forward(x, ids.float(), teacher), lambda: ds.forward(x, ids, teacher.double())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: op.forward(x[:, :49], tokens), lambda: op.forward(x, tokens[:3]), lambda: op.backward(x, tokens, g[:3]),
                lambda: op.backward(x, tokens, g, out=x[:3]), lambda: ds.forward(x, ids[:3], teacher),
                lambda: ds.forward(x, ids, teacher[:, :2]), lambda: ds.forward(x, ids[:, :0], teacher[:, :0]),
                lambda: op.backward(x, tokens, x.view(-1)[:rows], out=x)):
        with pytest.raises(ValueError):
            bad()
    five = draw(6, 5, vocab)
    for bad in (lambda: op.forward(x, tokens, top=51), lambda: op.forward(five, ids_of(1, vocab, 5)),
                lambda: gd.TokenLogProbs(100, torch.float32).forward(draw(1, 1, 100), tokens[:1], top=65),
                lambda: ds.forward(x, ids[:, :1].expand(rows, 257).contiguous(), teacher[:, :1].expand(rows, 257).contiguous()),
                lambda: gd.TokenLogProbs(vocab, torch.float32, scale=0.0).forward(x, tokens), lambda: gd.Distill(0),
                lambda: gd.TokenLogProbs(vocab, torch.float32, scale=math.inf).forward(x, tokens),
                lambda: gd.Distill(vocab, torch.float32, scale=-1.0).backward(x, ids, teacher, g)):
        with pytest.raises(gd.GDError):
            bad()
    for bad in (lambda: op.forward(x.clone().requires_grad_(), tokens), lambda: ds.forward(x.clone().requires_grad_(), ids, teacher),
                lambda: op.forward_backward(x.clone().requires_grad_(), tokens, g)):
        with pytest.raises(RuntimeError):
            bad()


@pytest.mark.parametrize("top", [-1, 1 << 32, (1 << 32) + 1])
def test_refuses_a_number_of_alternatives_past_its_type(top):
    op = gd.TokenLogProbs(50, torch.float32, max_rows=2)
    with pytest.raises(gd.GDError):
        op.forward(draw(1, 2, 50), ids_of(2, 50, 2), top=top)
