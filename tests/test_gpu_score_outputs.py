"""Outputs that the caller gives to a call for log probabilities."""
import dataclasses
import itertools

import pytest
import torch

from paper_1704_05021_amd import gd

pytestmark = pytest.mark.gpu

NAMES = ("logp", "entropy", "stats", "top_logp", "top_ids")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def made(rows, vocab, dtype=torch.float32):
    g = torch.Generator().manual_seed(1)
    x, tokens = torch.randn(rows, vocab, generator=g).to(dtype).cuda(), torch.randint(0, vocab, (rows,), generator=g).cuda()
    op = gd.TokenLogProbs(vocab, dtype, max_rows=rows)
    return op, x, tokens, op.forward(x, tokens, top=4, keep_stats=True)


def within(t, at, like):
    """A tensor of the shape and type of ``like`` in the memory of t, from byte `at` on."""
    flat = t.view(-1).view(torch.uint8)
    return flat[at:at + like.nbytes].view(like.dtype).view(like.shape)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_in_what_is_read_are_refused(dtype, name):
    rows = 8
    op, x, tokens, r = made(rows, 96, dtype)
    kept = x.clone()
    for t, at in ((x, 0), (x, x.nbytes - getattr(r, name).nbytes), (tokens.repeat(8), 0)):
        out = dataclasses.replace(r, **{name: within(t, at, getattr(r, name))})
        with pytest.raises(ValueError, match="overlaps"):
            op.forward(x, tokens if t is x else t[:rows], top=4, keep_stats=True, out=out)
    assert torch.equal(x, kept)


@pytest.mark.parametrize("a,b", list(itertools.combinations(NAMES, 2)))
def test_outputs_in_one_another_are_refused(a, b):
    op, x, tokens, r = made(8, 96)
    small, large = sorted((a, b), key=lambda n: getattr(r, n).nbytes)
    out = dataclasses.replace(r, **{small: within(getattr(r, large), 0, getattr(r, small))})
    with pytest.raises(ValueError, match="overlaps"):
        op.forward(x, tokens, top=4, keep_stats=True, out=out)


def test_outputs_side_by_side_and_between_rows_are_taken():
    rows, vocab = 8, 96
    op, x, tokens, r = made(rows, vocab)
    room = torch.empty(1024, device="cuda")
    at, fields = 0, {}
    for name in NAMES[4:] + NAMES[:4]:
        fields[name] = within(room, at, getattr(r, name))
        at += getattr(r, name).nbytes
    got = op.forward(x, tokens, top=4, keep_stats=True, out=gd.LogProbs(**fields))
    wide = torch.zeros(rows, vocab + rows, device="cuda")
    wide[:, :vocab] = x
    between = op.forward(wide[:, :vocab], tokens, entropy=False, out=gd.LogProbs(wide[3, vocab:]))
    for name in NAMES:
        assert torch.equal(getattr(got, name), getattr(r, name)), name
    assert torch.equal(between.logp, r.logp) and torch.equal(wide[:, :vocab], x)


@pytest.mark.parametrize("wishes", [dict(top=4, entropy=False, keep_stats=True), dict(top=4), dict(keep_stats=True)])
def test_outputs_that_the_call_would_leave_as_they_were_are_refused(wishes):
    """Stats of other logits, taken for these ones' by a backward call, would give a wrong gradient."""
    op, x, tokens, r = made(8, 96)
    with pytest.raises(ValueError, match="not asked for"):
        op.forward(x, tokens, out=r, **wishes)
    for keep in (False, True):
        r = op.forward(x, tokens, keep_stats=keep)
        assert op.forward(x, tokens, keep_stats=keep, out=r) is r
