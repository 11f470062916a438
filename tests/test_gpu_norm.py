"""Root-mean-square norm, forward (in the type and in 8 bits) and backward, against the 64-bit definition."""
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


def draw(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def check_forward(x, w, r, eps, y, h, what):
    H, Y = plain.norm(d(x), d(w), d(r), eps)
    close(h, H, rounded(H, x.dtype) + E * H.abs(), what + " sum")
    # the sum, the factor, and two products: five roundings in 32 bits
    close(y, Y, rounded(Y, x.dtype) + 5 * E * Y.abs(), what)


# rows and widths: one, the edges of a vector, of a wave's and a block's share, past every register shape
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 8), (1, 64), (6, 500), (4, 512), (9, 513), (2, 1024), (3, 1025),
                                      (2, 2048), (2, 2056), (1, 4096), (3, 4100), (2, 8192), (2, 9001), (2, 16384),
                                      (1, 20000), (2, 32768)])
def test_forward_and_backward_over_sizes(kind, rows, dim):
    t, eps = TYPES[kind], 1e-5
    x, w = draw(1, rows, dim, dtype=t), (1 + draw(2, dim, scale=0.2)).to(t)
    op = gd.RMSNorm(dim, t, eps)
    for r in (None, draw(3, rows, dim, dtype=t, scale=2.0)):
        y, h = op.forward(x, w, r)
        check_forward(x, w, r, eps, y, h, f"{kind} {rows}x{dim}")
        assert r is not None or h is x
        q, scale, h8 = op.forward_int8(x, w, r)
        assert torch.equal(h8, h)
        Y = plain.norm(d(x), d(w), d(r), eps)[1]
        s = plain.quantise(Y)
        close(scale, s[:, 0], 8 * E * s[:, 0], "scale")
        close(d(q) * d(scale)[:, None], Y, 0.5 * s + 16 * E * s * 127, "int8")
        dy = draw(4, rows, dim, dtype=t, scale=0.5)
        dx, dw = op.backward(dy, h, w, dsum=r)
        DX, DW, size, wsize = plain.norm_back(d(dy), d(h), d(w), d(r), eps)
        close(dx, DX, rounded(DX, t) + 8 * E * size, "dx")
        close(dw, DW, 8 * E * wsize, "dweight")


@pytest.mark.parametrize("rows,dim", [(700, 40), (2500, 512), (1300, 640), (3000, 500), (600, 2000)])
def test_backward_over_many_rows(rows, dim):
    """More rows than partial sums: every thread adds several rows to its share of the weight's gradient."""
    x, dy, w = draw(1, rows, dim, dtype=torch.bfloat16), draw(2, rows, dim, dtype=torch.bfloat16), draw(3, dim, dtype=torch.bfloat16)
    op = gd.RMSNorm(dim)
    dx, dw = op.backward(dy, x, w)
    DX, DW, size, wsize = plain.norm_back(d(dy), d(x), d(w), None, 1e-6)
    close(dx, DX, rounded(DX, torch.bfloat16) + 8 * E * size, "dx")
    close(dw, DW, (8 + math.ceil(rows / 512)) * E * wsize, "dweight")


def test_gradients_against_differences():
    rows, dim, eps = 3, 24, 1e-3
    x, w, c = draw(1, rows, dim), draw(2, dim), draw(3, rows, dim)
    dx, dw = gd.RMSNorm(dim, torch.float32, eps).backward(c, x, w)
    loss = lambda a, b: float((plain.norm(a, b, None, eps)[1] * d(c)).sum())  # noqa: E731
    step = 1e-6
    for k in range(0, rows * dim, 5):
        lo, hi = d(x).clone(), d(x).clone()
        lo.view(-1)[k] -= step
        hi.view(-1)[k] += step
        assert abs((loss(hi, d(w)) - loss(lo, d(w))) / (2 * step) - float(dx.view(-1)[k])) < 2e-5
    for k in range(0, dim, 5):
        lo, hi = d(w).clone(), d(w).clone()
        lo[k] -= step
        hi[k] += step
        assert abs((loss(d(x), hi) - loss(d(x), lo)) / (2 * step) - float(dw[k])) < 2e-5


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strides_offsets_and_outputs_in_place(kind):
    """Rows inside a wider buffer, starting off any alignment; outputs in the inputs' own buffers."""
    t, rows, dim = TYPES[kind], 5, 300
    wide = draw(1, rows, 333, dtype=t)
    x = wide[:, 7:7 + dim]
    r = draw(2, rows * 301 + 1, dtype=t)[1:].view(rows, 301)[:, :dim]
    w = draw(3, dim + 1, dtype=t)[1:]
    op = gd.RMSNorm(dim, t)
    y, h = op.forward(x, w, r)
    check_forward(x, w, r, 1e-6, y, h, "strided")
    out = torch.full((rows, 310), -7.0, dtype=t, device="cuda")
    op.forward(x, w, r, out=out[:, 3:3 + dim])
    assert torch.equal(out[:, 3:3 + dim], y) and bool((out[:, :3] == -7).all() and (out[:, 3 + dim:] == -7).all())
    before = wide.clone()
    y2, h2 = op.forward(x, w, r, out=x, sum_out=r)  # y over x, the sum over the residual stream
    assert torch.equal(x, y) and torch.equal(r, h) and y2 is x and h2 is r
    assert torch.equal(wide[:, :7], before[:, :7]) and torch.equal(wide[:, 7 + dim:], before[:, 7 + dim:])
    dy, dsum = draw(4, rows, dim, dtype=t), draw(5, rows, dim, dtype=t)
    dx, dw = op.backward(dy, h, w, dsum=dsum)
    flat = torch.zeros(dim + 9, device="cuda")
    dx2, _ = op.backward(dy, h, w, dsum=dsum, dx=dsum, dweight=flat[3:3 + dim])
    assert torch.equal(dx, dsum) and torch.equal(flat[3:3 + dim], dw) and float(flat[:3].abs().sum() + flat[3 + dim:].abs().sum()) == 0


def test_accumulate_and_no_rows():
    dim = 96
    x, dy, w = draw(1, 40, dim), draw(2, 40, dim), draw(3, dim)
    op = gd.RMSNorm(dim, torch.float32)
    _, dw = op.backward(dy, x, w)
    total = dw.clone()
    op.backward(dy, x, w, dweight=total, accumulate=True)
    close(total, 2 * d(dw), 2 * E * d(dw).abs(), "accumulated")
    none = torch.empty(0, dim, device="cuda")
    y, h = op.forward(none, w)
    assert y.shape == (0, dim)
    op.backward(none, none, w, dweight=total, accumulate=True)
    close(total, 2 * d(dw), 2 * E * d(dw).abs(), "nothing added")
    op.backward(none, none, w, dweight=total)
    assert float(total.abs().sum()) == 0


@pytest.mark.parametrize("rows,dim", [(1, 5), (7, 60), (9, 60), (16, 500), (17, 500), (4, 2000), (5, 2000), (2, 8000), (3, 8000)])
def test_few_rows_accumulate(rows, dim):
    """Up to a few rows the weight's gradient is written by the block that sums it, past them by a second launch."""
    x, dy, w = draw(1, rows, dim), draw(2, rows, dim), draw(3, dim)
    op = gd.RMSNorm(dim, torch.float32)
    dx, dw = op.backward(dy, x, w)
    flat = torch.full((dim + 4,), 0.5, device="cuda")
    dx2, _ = op.backward(dy, x, w, dweight=flat[1:1 + dim], accumulate=True)
    assert torch.equal(dx, dx2) and bool((flat[:1] == 0.5).all() and (flat[1 + dim:] == 0.5).all())
    total = d(dw) + 0.5  # dw is rounded once more than the sum that was added, and the total once
    close(flat[1:1 + dim], total, E * d(dw).abs() + E * total.abs(), "accumulated")


def test_rows_of_zeros_and_of_values_that_are_not_finite():
    dim = 128
    x = draw(1, 5, dim)
    x[0] = 0
    x[2, 5] = math.inf
    x[3, 7] = math.nan
    w = torch.ones(dim, device="cuda")
    op = gd.RMSNorm(dim, torch.float32)
    y, _ = op.forward(x, w)
    assert bool((y[0] == 0).all()) and bool(y[3].isnan().all()) and bool(y[2, 5].isnan()) and bool((y[2, 6:] == 0).all())
    q, scale, _ = op.forward_int8(x, w)
    assert float(scale[0]) == 0 and bool((q[0] == 0).all())
    assert not bool(scale[2].isfinite()) and not bool(scale[3].isfinite())
    for i in (1, 4):  # rows beside them are as alone
        y1, _ = op.forward(x[i:i + 1], w)
        assert torch.equal(y1[0], y[i])
        q1, s1, _ = op.forward_int8(x[i:i + 1], w)
        assert torch.equal(q1[0], q[i]) and float(s1[0]) == float(scale[i])
    tiny = torch.full((1, dim), 1e-42, device="cuda")
    q, scale = gd.quantise_rows(tiny)
    assert bool((q == 0).all()) and float(scale[0]) < 1e-38


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,columns", [(1, 1), (5, 10), (3, 784), (2, 4096), (3, 5001), (1, 40000), (2, 131072)])
def test_quantise_rows(kind, rows, columns):
    x = draw(1, rows, columns + 3, dtype=TYPES[kind])[:, 1:1 + columns]
    q, scale = gd.quantise_rows(x)
    s = plain.quantise(d(x))
    close(scale, s[:, 0], 2 * E * s[:, 0], "scale")
    close(d(q) * d(scale)[:, None], d(x), 0.5 * s + 4 * E * s * 127, "codes")
    assert int(d(q).abs().max()) == 127


def test_other_streams_and_graphs():
    """On a stream of its own, and captured and replayed between other work, results stay the same."""
    dim = 1000
    x, w, r = draw(1, 50, dim, dtype=torch.bfloat16), draw(2, dim, dtype=torch.bfloat16), draw(3, 50, dim, dtype=torch.bfloat16)
    op = gd.RMSNorm(dim)
    y, h = op.forward(x, w, r)
    dx, dw = op.backward(x, h, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, h2 = op.forward(x, w, r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    graph = torch.cuda.CUDAGraph()
    out = [torch.empty_like(y), torch.empty_like(h), torch.empty_like(dx), torch.empty_like(dw)]
    with torch.cuda.graph(graph):
        op.forward(x, w, r, out=out[0], sum_out=out[1])
        op.backward(x, out[1], w, dx=out[2], dweight=out[3])
    for seed in range(3):
        x.copy_(draw(10 + seed, 50, dim, dtype=torch.bfloat16))
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        y, h = op.forward(x, w, r)
        dx, dw = op.backward(x, h, w)
        for a, b in zip(got, (y, h, dx, dw)):
            assert torch.equal(a, b)


def test_refusals():
    for dim in (0, 32769, 1 << 33):
        with pytest.raises(gd.GDError):
            gd.RMSNorm(dim)
    with pytest.raises(TypeError):
        gd.RMSNorm(8, torch.float64)
    op = gd.RMSNorm(64)
    x, w = draw(1, 4, 64, dtype=torch.bfloat16), draw(2, 64, dtype=torch.bfloat16)
    for bad in (x.float(), x.cpu()):
        with pytest.raises(TypeError):
            op.forward(bad, w)
    for bad in (x[:, :63], draw(1, 64, 4, dtype=torch.bfloat16).t(), x[:1].expand(4, 64)):
        with pytest.raises((ValueError, gd.GDError)):
            op.forward(bad, w)
    with pytest.raises(ValueError):
        op.forward(x, w[:63].contiguous())
    with pytest.raises(ValueError):
        op.forward(x, w, x[:3])
    with pytest.raises(ValueError):
        op.backward(x, x, w, accumulate=True)
    for eps in (-1.0, math.nan, math.inf):
        with pytest.raises(gd.GDError):
            gd.RMSNorm(64, eps=eps).forward(x, w)
