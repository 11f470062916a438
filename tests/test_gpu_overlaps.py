"""Given outputs that overlap what a call reads or writes are refused; those that lie between its rows, or are the same
rows where that is allowed, are taken."""
import itertools

import pytest
import torch

from paper_1704_05021_amd import gd


def test_matrices_that_meet():
    """Against the sets of addresses, over every pair of small layouts."""
    layouts = [(at, rows, stride, columns) for at in (0, 1, 3, 6, 8, 17) for rows in (0, 1, 2, 3)
               for columns in (1, 2, 4) for stride in (4, 6, 7) if stride >= columns]
    for size in (2, 4):
        places = {m: {m[0] * size + (r * m[2] + c) * size + b for r in range(m[1]) for c in range(m[3]) for b in range(size)}
                  for m in layouts}
        for a, b in itertools.product(layouts, repeat=2):
            meet = gd._meet((a[0] * size, *a[1:]), (b[0] * size, *b[1:]), size)
            assert meet or not places[a] & places[b], (a, b)
            runs = a[1] == 1 or b[1] == 1 or a[2] == a[3] or b[2] == b[3]
            if a[2] == b[2] or runs:  # rows at two distances may be called meeting where they lie between each other
                assert meet == bool(places[a] & places[b]), (a, b)


@pytest.fixture
def draw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    g = torch.Generator().manual_seed(1)
    return lambda *s, kind=torch.float32: torch.randn(*s, generator=g).to(kind).cuda()


def refused(call, *args, **kwargs):
    with pytest.raises(ValueError, match="overlaps"):
        call(*args, **kwargs)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_linear(draw, kind):
    n = 64
    x, w, b, r, pre = draw(n, n, kind=kind), draw(n, n, kind=kind), draw(n, kind=kind), draw(n, n, kind=kind), draw(n, n, kind=kind)
    op = gd.Linear(n, n, kind, "silu", max_rows=n)
    kept = [t.clone() for t in (x, w, b, r, pre)]
    refused(op.forward, x, w, out=x)
    refused(op.forward, x, w, out=w)
    refused(op.forward, x[:-1], w, out=x[1:])
    refused(op.forward, x, w, residual=x, out=x)
    refused(op.forward, x, w, keep_pre=x)
    refused(op.forward, x, w, residual=r, keep_pre=r)
    refused(op.forward, x, w, out=pre, keep_pre=pre)
    refused(op.forward, x[:1], w, b, out=b.view(1, n))
    dy = draw(n, n, kind=kind)
    refused(op.backward, dy, x, w, pre, dx=x)
    refused(op.backward, dy, x, w, pre, dx=dy)
    refused(op.backward, dy, x, w, pre, dx=w)
    refused(op.backward, dy, x, w, pre, dz=x)
    refused(op.backward, dy, x, w, pre, dz=pre, dx=pre)
    refused(gd.Linear(n, n, kind, max_rows=n).backward, dy, x, w, dx=dy)
    for a, t in zip(kept, (x, w, b, r, pre)):
        assert torch.equal(a, t)
    # taken: between the rows of an input, the residual itself, dz over dy or pre, x where no gradient needs it
    wide = draw(n, 2 * n + 3, kind=kind)
    want = op.forward(wide[:, :n].contiguous(), w)
    assert torch.equal(op.forward(wide[:, :n], w, out=wide[:, n:2 * n]), want)
    want = op.forward(x, w, b, r)
    assert torch.equal(op.forward(x, w, b, r, out=r), want)
    want = op.backward(dy, x, w, pre)
    over = x.clone()
    assert torch.equal(op.backward(dy, over, w, pre, need_dweight=False, dx=over)[0], want[0])
    over = dy.clone()
    assert torch.equal(op.backward(over, x, w, pre, dz=over)[1], want[1])
    over = pre.clone()
    assert torch.equal(op.backward(dy, x, w, over, dz=over)[1], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_norm(draw, kind):
    n = 64
    x, r, w = draw(n, n, kind=kind), draw(n, n, kind=kind), draw(n, kind=kind)
    op = gd.RMSNorm(n, kind)
    refused(op.forward, x, w, r, out=x, sum_out=x)
    refused(op.forward, x[:-1], w, out=x[1:])
    refused(op.forward, x[1:], w, sum_out=x[:-1])
    refused(op.forward, x[:1], w, out=w.view(1, n))
    refused(op.forward_int8, x[:-1], w, sum_out=x[1:])
    refused(op.backward, r, x, w, dx=x)
    for out, total in (("x", "r"), ("r", "x"), ("x", None), ("r", None), (None, "x"), (None, "r")):
        a = {"x": x.clone(), "r": r.clone(), None: None}
        y, h = op.forward(x, w, r)
        y2, h2 = op.forward(a["x"], w, a["r"], out=a[out], sum_out=a[total])
        assert torch.equal(y, y2) and torch.equal(h, h2)
    a = x.clone()
    y, h = op.forward(x, w, x)
    assert torch.equal(op.forward(a, w, a, out=a)[0], y)
    dx, dw = op.backward(r, x, w, dsum=x)
    a = r.clone()
    assert torch.equal(op.backward(a, x, w, dsum=x, dx=a)[0], dx)
