"""Layer norm, forward (in the type and in 8 bits) and backward, against the 64-bit definition."""
import math

import pytest
import torch

import plain_ops as plain
from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, close, d, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def draw(seed, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (shift + torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def forward64(x, w, b, r, eps):
    h = x if r is None else x + r
    c = h - h.mean(1, keepdim=True)
    hat = c / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    y = hat * w
    return h, (y if b is None else y + b), y


def backward64(dy, h, w, dsum, eps):
    """(dx, dweight, dbias) and the sums of magnitudes that their roundings are relative to."""
    c = h - h.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    hat, a = c * r, dy * w
    ma, mx = a.mean(1, keepdim=True), (a * hat).mean(1, keepdim=True)
    dx = r * (a - ma - hat * mx)
    # one rounding each of a and its mean, three of xhat, three of mean(a xhat), one a product and difference: at most 12
    size = r * (a.abs() + a.abs().mean(1, keepdim=True) + hat.abs() * (a * hat).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, size = dx + dsum, size + dsum.abs()
    return dx, (dy * hat).sum(0), dy.sum(0), size, (dy * hat).abs().sum(0), dy.abs().sum(0)


def sum_error(x, r):
    """How far the 32-bit sum x + r, which the norm is taken of, may be from the exact one."""
    return 0.0 if r is None else E * (x + r).abs().amax(1, keepdim=True)


def check_forward(x, w, b, r, eps, y, h, what):
    H, Y, part = forward64(d(x), d(w), d(b), d(r), eps)
    close(h, H, rounded(H, x.dtype) + E * H.abs(), what + " sum")
    # c, the factor and two products: four roundings of the product, one of the sum; the 32-bit sum's own error, at most
    # one of its largest element's, passes to c, its mean and its spread: three times, by the row's factor
    c = H - H.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    hat = c.abs() * rstd
    inner = sum_error(d(x), d(r)) * rstd * (2.0 + hat) * d(w).abs()
    close(y, Y, rounded(Y, x.dtype) + 4 * E * part.abs() + 2 * E * Y.abs() + inner * 1.01, what)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 8), (1, 64), (6, 500), (4, 512), (9, 513), (2, 1024), (3, 1025),
                                      (2, 2048), (2, 2056), (1, 4096), (3, 4100), (2, 8192), (2, 9001), (2, 16384),
                                      (1, 20000), (2, 32768)])
def test_forward_and_backward_over_sizes(kind, rows, dim):
    t, eps = TYPES[kind], 1e-5
    x, w, b = draw(1, rows, dim, dtype=t, shift=0.5), (1 + draw(2, dim, scale=0.2)).to(t), draw(7, dim, dtype=t)
    op = gd.LayerNorm(dim, t, eps)
    for r in (None, draw(3, rows, dim, dtype=t, scale=2.0)):
        for bias in (b, None):
            y, h = op.forward(x, w, bias, r)
            check_forward(x, w, bias, r, eps, y, h, f"{kind} {rows}x{dim}")
        assert r is not None or h is x
        y32 = gd.LayerNorm(dim, torch.float32, eps).forward(x.float(), w.float(), b.float(), None if r is None else r.float())[0]
        q, scale, h8 = op.forward_int8(x, w, b, r)
        assert torch.equal(h8, h)
        # the same 32-bit values, then the rounding of rows to 8 bits: equal to quantise_rows bit for bit
        q2, scale2 = gd.quantise_rows(y32)
        assert torch.equal(q, q2) and torch.equal(scale.view(torch.int32), scale2.view(torch.int32))
        dy = draw(4, rows, dim, dtype=t, scale=0.5)
        dx, dw, db = op.backward(dy, h, w, dsum=r)
        DX, DW, DB, size, wsize, bsize = backward64(d(dy), d(h), d(w), d(r), eps)
        close(dx, DX, rounded(DX, t) + 12 * E * size, "dx")
        close(dw, DW, (4 + rows) * E * wsize, "dweight")
        close(db, DB, rows * E * bsize, "dbias")


@pytest.mark.parametrize("rows,dim", [(700, 40), (2500, 512), (1300, 640), (3000, 500), (600, 2000), (1100, 4096), (700, 5000)])
def test_backward_over_many_rows(rows, dim):
    """More rows than partial sums: every thread adds several rows to its share of the gradients over rows."""
    t = torch.bfloat16
    x, dy, w = draw(1, rows, dim, dtype=t, shift=1.0), draw(2, rows, dim, dtype=t), draw(3, dim, dtype=t)
    dx, dw, db = gd.LayerNorm(dim).backward(dy, x, w)
    DX, DW, DB, size, wsize, bsize = backward64(d(dy), d(x), d(w), None, 1e-5)
    close(dx, DX, rounded(DX, t) + 12 * E * size, "dx")
    close(dw, DW, (8 + math.ceil(rows / 128)) * E * wsize, "dweight")
    close(db, DB, (8 + math.ceil(rows / 128)) * E * bsize, "dbias")


def test_gradients_against_differences():
    rows, dim, eps = 3, 24, 1e-3
    x, w, b, c = draw(1, rows, dim), draw(2, dim), draw(5, dim), draw(3, rows, dim)
    dx, dw, db = gd.LayerNorm(dim, torch.float32, eps).backward(c, x, w)
    loss = lambda a, v, s: float((forward64(a, v, s, None, eps)[1] * d(c)).sum())  # noqa: E731
    step, at = 1e-6, [d(x), d(w), d(b)]
    for k, (value, got) in enumerate(zip(at, (dx, dw, db))):
        for i in range(0, value.numel(), 5):
            ends = []
            for sign in (-1, 1):
                moved = [v.clone() for v in at]
                moved[k].view(-1)[i] += sign * step
                ends.append(loss(*moved))
            # differences in 64 bits err by about 1e-16 / step and step^2, the kernel by some 2^-24 of values below 10
            assert abs((ends[1] - ends[0]) / (2 * step) - float(got.view(-1)[i])) < 2e-5


@pytest.mark.parametrize("shift,spread", [(1e4, 1e-2), (-3e3, 1.0), (1e6, 0.5)])
def test_rows_far_from_zero(shift, spread):
    """The spread of a row that lies far from zero is that of its values as they are stored."""
    rows, dim, eps = 4, 1000, 1e-12
    x, w, dy = draw(1, rows, dim, scale=spread, shift=shift), torch.ones(dim, device="cuda"), draw(2, rows, dim)
    op = gd.LayerNorm(dim, torch.float32, eps)
    y, _ = op.forward(x, w)
    check_forward(x, w, None, None, eps, y, x, "far")
    dx, dw, _ = op.backward(dy, x, w)
    DX, DW, _, size, wsize, _ = backward64(d(dy), d(x), d(w), None, eps)
    close(dx, DX, rounded(DX, torch.float32) + 12 * E * size, "dx")
    close(dw, DW, (4 + rows) * E * wsize, "dweight")


def test_constant_rows_and_an_outlier_first():
    dim, eps = 640, 1e-5
    x = torch.full((3, dim), 7.25, device="cuda")
    x[1, 0] = 1e6  # the element that the sums are shifted by
    x[2, 5] = 3e5
    w, b = draw(1, dim), draw(2, dim)
    op = gd.LayerNorm(dim, torch.float32, eps)
    y, _ = op.forward(x, w, b)
    assert torch.equal(y[0], b)  # no spread: the bias
    check_forward(x[1:], w, b, None, eps, y[1:], x[1:], "outliers")
    dx, *_ = op.backward(draw(3, 3, dim), x, w)
    assert bool(dx.isfinite().all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strides_offsets_and_outputs_in_place(kind):
    """Rows inside a wider buffer, starting off any alignment; outputs in the inputs' own buffers."""
    t, rows, dim = TYPES[kind], 5, 300
    wide = draw(1, rows, 333, dtype=t)
    x = wide[:, 7:7 + dim]
    r = draw(2, rows * 301 + 1, dtype=t)[1:].view(rows, 301)[:, :dim]
    w, b = draw(3, dim + 1, dtype=t)[1:], draw(6, dim + 1, dtype=t)[1:]
    op = gd.LayerNorm(dim, t)
    y, h = op.forward(x, w, b, r)
    check_forward(x, w, b, r, 1e-5, y, h, "strided")
    out = torch.full((rows, 310), -7.0, dtype=t, device="cuda")
    op.forward(x, w, b, r, out=out[:, 3:3 + dim])
    assert torch.equal(out[:, 3:3 + dim], y) and bool((out[:, :3] == -7).all() and (out[:, 3 + dim:] == -7).all())
    before = wide.clone()
    y2, h2 = op.forward(x, w, b, r, out=x, sum_out=r)  # y over x, the sum over the residual stream
    assert torch.equal(x, y) and torch.equal(r, h) and y2 is x and h2 is r
    assert torch.equal(wide[:, :7], before[:, :7]) and torch.equal(wide[:, 7 + dim:], before[:, 7 + dim:])
    dy, dsum = draw(4, rows, dim, dtype=t), draw(5, rows, dim, dtype=t)
    dx, dw, db = op.backward(dy, h, w, dsum=dsum)
    flat = torch.zeros(2 * dim + 9, device="cuda")
    dx2, *_ = op.backward(dy, h, w, dsum=dsum, dx=dsum, dweight=flat[3:3 + dim], dbias=flat[5 + dim:5 + 2 * dim])
    assert torch.equal(dx, dsum) and torch.equal(flat[3:3 + dim], dw) and torch.equal(flat[5 + dim:5 + 2 * dim], db)
    assert float(flat[:3].abs().sum() + flat[3 + dim:5 + dim].abs().sum() + flat[5 + 2 * dim:].abs().sum()) == 0
    assert op.backward(dy, h, w, dbias=False)[2] is None


@pytest.mark.parametrize("rows,dim", [(1, 5), (7, 60), (9, 60), (16, 500), (17, 500), (4, 2000), (5, 2000), (40, 96), (600, 700)])
def test_accumulate(rows, dim):
    """Up to a few rows the gradients over rows are written by the block that sums them, past them by a second launch."""
    x, dy, w = draw(1, rows, dim), draw(2, rows, dim), draw(3, dim)
    op = gd.LayerNorm(dim, torch.float32)
    dx, dw, db = op.backward(dy, x, w)
    flat = torch.full((2 * dim + 4,), 0.5, device="cuda")
    dx2, *_ = op.backward(dy, x, w, dweight=flat[1:1 + dim], dbias=flat[2 + dim:2 + 2 * dim], accumulate=True)
    assert torch.equal(dx, dx2) and float((flat[[0, 1 + dim, 2 * dim + 2, 2 * dim + 3]] - 0.5).abs().sum()) == 0
    for got, was in ((flat[1:1 + dim], dw), (flat[2 + dim:2 + 2 * dim], db)):
        total = d(was) + 0.5  # the gradient is rounded once more than the sum that was added, and the total once
        close(got, total, E * d(was).abs() + E * total.abs(), "accumulated")


def test_no_rows():
    dim = 96
    op, w = gd.LayerNorm(dim, torch.float32), draw(1, dim)
    none, total = torch.empty(0, dim, device="cuda"), draw(2, 2, dim)
    was = total.clone()
    assert op.forward(none, w)[0].shape == (0, dim)
    op.backward(none, none, w, dweight=total[0], dbias=total[1], accumulate=True)
    assert torch.equal(total, was)
    op.backward(none, none, w, dweight=total[0], dbias=total[1])
    assert float(total.abs().sum()) == 0


def test_rows_that_are_not_finite_stay_apart():
    dim = 128
    x, w, b = draw(1, 6, dim), draw(2, dim), draw(3, dim)
    clean = x.clone()
    x[0, 0], x[2, 5], x[4, 127] = math.nan, math.inf, -math.inf
    op = gd.LayerNorm(dim, torch.float32)
    y, want = op.forward(x, w, b)[0], op.forward(clean, w, b)[0]
    q, scale, _ = op.forward_int8(x, w, b)
    for row in range(6):
        if row % 2 == 0:
            assert bool(y[row].isnan().all()) and not bool(scale[row].isfinite())
        else:
            assert torch.equal(y[row], want[row]) and bool(scale[row].isfinite())


def test_another_stream_and_graph_replays():
    rows, dim = 300, 768
    x, w, b, dy = draw(1, rows, dim, dtype=torch.bfloat16), draw(2, dim, dtype=torch.bfloat16), draw(3, dim, dtype=torch.bfloat16), draw(4, rows, dim, dtype=torch.bfloat16)
    op = gd.LayerNorm(dim)
    y, h = op.forward(x, w, b)
    dx, dw, db = op.backward(dy, x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, _ = op.forward(x, w, b, stream=s)
    got = op.backward(dy, x, w, stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(a, c) for a, c in zip((dx, dw, db), got))
    out, gx, gw, gb = torch.empty_like(y), torch.empty_like(dx), torch.empty_like(dw), torch.empty_like(db)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(x, w, b, out=out)
        op.backward(dy, x, w, dx=gx, dweight=gw, dbias=gb)
    for seed in range(3):
        x.copy_(draw(10 + seed, rows, dim, dtype=torch.bfloat16))
        graph.replay()
        y, _ = op.forward(x, w, b)
        want = op.backward(dy, x, w)
        torch.cuda.synchronize()
        assert torch.equal(out, y) and all(torch.equal(a, c) for a, c in zip((gx, gw, gb), want))


def test_refusals():
    op = gd.LayerNorm(64)
    x, w = draw(1, 4, 64, dtype=torch.bfloat16), draw(2, 64, dtype=torch.bfloat16)
    for bad in (lambda: op.forward(x.float(), w), lambda: op.forward(x.cpu(), w), lambda: op.forward(x, w.float()),
                lambda: op.forward(x, w, w.float())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: op.forward(x[:, :63], w), lambda: op.forward(x, w[:63]), lambda: op.forward(x, w, w[:3]),
                lambda: op.forward(x.t(), w), lambda: op.forward(x, w, out=x.view(-1)[:0].view(0, 64)),
                lambda: op.backward(x, x, w, dx=x[:3]),
                lambda: op.backward(x, x.clone(), w, accumulate=True), lambda: op.backward(x.clone(), x, w, dx=x)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        op.forward(x, w, w.clone().requires_grad_())
    with torch.no_grad():
        op.forward(x, w, w.clone().requires_grad_())
    with pytest.raises(gd.GDError):
        gd.LayerNorm(32769)
    with pytest.raises(gd.GDError):
        gd.LayerNorm(64, eps=-1.0).forward(x, w)
