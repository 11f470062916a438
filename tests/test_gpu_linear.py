"""Linear layers, forward (in the type and with 8-bit operands) and backward, against the 64-bit definition."""
import math

import pytest
import torch

import plain_ops as plain
from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, ULP, close, d, rounded

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


def whole(seed, *shape, dtype=torch.float32, most=3):
    """Small whole numbers: sums of their products are exact in 32 bits, in any order."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype).cuda()


def check_forward(op, x, w, b, r, y, pre, what):
    t = op.dtype
    z, off = plain.product(d(x), d(w))
    if b is not None:
        z, off = z + d(b), off + E * (z.abs() + d(b).abs())
    if pre is not None:
        close(pre, z, off + rounded(z, t), what + " pre")
    a = plain.act(op.act, z)
    off = 1.2 * off + 16 * E * (z.abs() + a.abs())  # slopes are below 1.2; the functions are within a few ulps
    if r is not None:
        a = a + d(r)
        off = off + E * a.abs()
    close(y, a, off + rounded(a, t), what)


def check_backward(op, dy, x, w, pre, got, what):
    t = op.dtype
    dx, dw, db, dz = got
    want = d(dy) * plain.slope(op.act, d(pre)) if op.act != "none" else d(dy)
    close(dz, want, rounded(want, t) + 24 * E * d(dy).abs() * (1 + d(pre).abs() if pre is not None else 1), what + " dz")
    z = d(dz)  # the products take the rounded gradient
    if dx is not None:
        s, off = plain.product(z, d(w).t())
        close(dx, s, off + rounded(s, t), what + " dx")
    if dw is not None:
        s, off = plain.product(z.t(), d(x).t())
        close(dw, s, off + E * s.abs(), what + " dweight")
    if db is not None:
        s, off = plain.product(z.t(), torch.ones(1, z.shape[0], dtype=torch.float64))
        close(db, s[:, 0], off[:, 0] + E * s[:, 0].abs(), what + " dbias")


SIZES = [(1, 1, 1), (1, 8, 8), (2, 7, 9), (3, 64, 10), (1, 784, 512), (16, 500, 33), (15, 1024, 1000), (17, 65, 64),
         (33, 129, 127), (40, 784, 500), (64, 64, 64), (65, 1000, 130), (100, 10, 300), (257, 100, 65), (300, 511, 257)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_sizes(kind, rows, k, n):
    t = TYPES[kind]
    x, w = draw(1, rows, k, dtype=t), draw(2, n, k, dtype=t, scale=k ** -0.5)
    b, r, dy = draw(3, n, dtype=t), draw(4, rows, n, dtype=t), draw(5, rows, n, dtype=t)
    for act in ("none", "relu", "gelu", "silu"):
        op = gd.Linear(k, n, t, act, max_rows=rows)
        y, pre = op.forward(x, w, b, r, keep_pre=True)
        check_forward(op, x, w, b, r, y, pre, f"{kind} {act} {rows}x{k}x{n}")
        assert torch.equal(op.forward(x, w, b, r), y)
        got = op.backward(dy, x, w, pre, dbias=True)
        check_backward(op, dy, x, w, pre if act != "none" else None, got, f"{kind} {act} {rows}x{k}x{n}")
        if act == "none":
            assert got[3] is dy


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
# every tile of the three products, with whole and with ragged edges: most results of the largest tile, of the
# middle one, and of the smallest with and without a split of k
@pytest.mark.parametrize("rows,k,n", [(256 * 15, 128, 256 * 14), (256 * 14 + 33, 72, 256 * 15 - 40), (128, 256 * 15, 256 * 14),
                                      (100, 256 * 14 + 8, 256 * 15 - 9), (256 * 15, 256 * 14, 64), (128 * 15, 136, 128 * 14),
                                      (128 * 14 + 5, 200, 128 * 15 - 4), (64, 128 * 15, 128 * 14 + 4), (128 * 15 - 3, 128 * 14, 40),
                                      (64, 4096, 64), (90, 4100, 70), (4096, 64, 64), (5000, 70, 90), (70, 64, 4096),
                                      (60, 90, 5003), (10, 4096, 4096), (7, 8191, 33),
                                      # tiles of 192 and 128 rows beside 256, in each of the three products
                                      (64, 4096, 3000), (3000, 128, 4096), (3000, 4096, 128), (2990, 136, 4080),
                                      (2048, 128, 4096), (2048, 4096, 128), (128, 4096, 2048), (200, 4088, 2040)])
def test_tiles_are_exact_on_whole_numbers(kind, rows, k, n):
    """Sums below 2^24 of whole numbers are exact, so every result is the exact one, rounded once."""
    t = TYPES[kind]
    x, w, dy = whole(1, rows, k, dtype=t), whole(2, n, k, dtype=t), whole(3, rows, n, dtype=t)
    op = gd.Linear(k, n, t, max_rows=rows)
    f = lambda a: a.double()  # noqa: E731
    assert torch.equal(op.forward(x, w), (f(x) @ f(w).t()).to(t))
    dx, dw, db, _ = op.backward(dy, x, w, dbias=True)
    assert torch.equal(dx, (f(dy) @ f(w)).to(t))
    assert torch.equal(dw, (f(dy).t() @ f(x)).float())
    assert torch.equal(db, f(dy).sum(0).float())
    if kind != "f32":
        q, s = whole(4, rows, k, dtype=torch.int8, most=127), torch.full((rows,), 0.5, device="cuda")
        wq, ws = whole(5, n, k, dtype=torch.int8, most=127), torch.full((n,), 2.0 ** -12, device="cuda")
        want = (f(q) @ f(wq).t()).float() * 2.0 ** -13  # one rounding of the exact sum, then powers of two
        assert torch.equal(op.forward_int8(q, s, wq, ws), want.to(t))


def guarded(a, seed):
    """a inside a wider buffer of NaN, off any alignment."""
    lead, gap = seed % 5, 1 + seed % 7
    wide = torch.full((a.shape[0] + 2, a.shape[1] + lead + gap), math.nan, dtype=a.dtype, device="cuda")
    inner = wide[1:1 + a.shape[0], lead:lead + a.shape[1]]
    inner.copy_(a)
    return inner


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 7, 8, 9, 31, 33, 62, 65, 131, 257])
def test_ends_inside_a_vector(kind, k):
    """Rows and k that end anywhere in a vector: exact sums, and nothing read past the operands reaches them."""
    t, f = TYPES[kind], lambda a: a.double()  # noqa: E731
    for rows in (1, 2, 3, 5, 18, 66, 131):
        for n in (1, 2, 3, 6, 13, 67, 130):
            x, w, dy = (guarded(whole(i + k, *s, dtype=t), rows + n + i) for i, s in enumerate([(rows, k), (n, k), (rows, n)]))
            op = gd.Linear(k, n, t, max_rows=rows)
            assert torch.equal(op.forward(x, w), (f(x) @ f(w).t()).to(t)), (rows, n)
            dx, dw, db, _ = op.backward(dy, x, w, dbias=True)
            assert torch.equal(dx, (f(dy) @ f(w)).to(t)), (rows, n)
            assert torch.equal(dw, (f(dy).t() @ f(x)).float()) and torch.equal(db, f(dy).sum(0).float()), (rows, n)
            q, wq = whole(7, rows, k, dtype=torch.int8), whole(8, n, k, dtype=torch.int8)
            y = op.forward_int8(q, torch.ones(rows, device="cuda"), wq, torch.ones(n, device="cuda"))
            assert torch.equal(y, (f(q) @ f(wq).t()).to(t)), (rows, n)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,k,n", [(40, 96, 80), (37, 90, 75), (150, 301, 67)])
def test_gradients_that_are_not_finite_stay_in_their_rows(kind, rows, k, n):
    t, f = TYPES[kind], lambda a: a.double()  # noqa: E731
    x, w, dy = whole(1, rows, k, dtype=t), whole(2, n, k, dtype=t), whole(3, rows, n, dtype=t)
    op = gd.Linear(k, n, t, max_rows=rows)
    dx, dw = (f(dy) @ f(w)).to(t), (f(dy).t() @ f(x)).float()
    dy[rows - 1, n - 1] = math.nan  # the last of the last row, which loads past the end repeat
    gx, gw = op.backward(dy, x, w)[:2]
    assert torch.equal(gx[:-1], dx[:-1]) and bool(gx[-1].isnan().all())
    assert torch.equal(gw[:-1], dw[:-1]) and bool(gw[-1].isnan().all())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_large_ragged_products_are_exact(kind):
    """Sizes at which operands off any alignment are copied into padded rows first, forward too."""
    t, f, (rows, k, n) = TYPES[kind], lambda a: a.double(), (2101, 2203, 2201)  # noqa: E731
    x, w, dy = whole(1, rows, k, dtype=t), whole(2, n, k, dtype=t), whole(3, rows, n, dtype=t)
    op = gd.Linear(k, n, t, max_rows=rows)
    dx, dw, db, _ = op.backward(dy, x, w, dbias=True)
    assert torch.equal(op.forward(x, w), (f(x) @ f(w).t()).to(t)) and torch.equal(dx, (f(dy) @ f(w)).to(t))
    assert torch.equal(dw, (f(dy).t() @ f(x)).float()) and torch.equal(db, f(dy).sum(0).float())
    q, wq = whole(4, rows, k, dtype=torch.int8), whole(5, n, k, dtype=torch.int8)
    y = op.forward_int8(q, torch.ones(rows, device="cuda"), wq, torch.ones(n, device="cuda"))
    assert torch.equal(y, (f(q) @ f(wq).t()).to(t))


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_slopes_over_the_whole_range(kind, act):
    """Each slope from far below zero to far above, the steep part closely."""
    t, n = TYPES[kind], 1000
    pre = torch.cat([torch.linspace(-60, 60, 2 * n), torch.linspace(-6, 6, 3 * n), torch.tensor([0.0, -0.0] * (n // 2)),
                     torch.linspace(-3e4, 3e4, n), 10.0 ** torch.linspace(-30, 0, n)]).view(-1, n).to(t).cuda()
    x, w, dy = draw(1, pre.shape[0], 8, dtype=t), draw(2, n, 8, dtype=t), draw(3, *pre.shape, dtype=t)
    op = gd.Linear(8, n, t, act, max_rows=pre.shape[0])
    check_backward(op, dy, x, w, pre, op.backward(dy, x, w, pre, dbias=True), f"{kind} {act}")


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n", [(1, 784, 512), (5, 100, 7), (40, 1000, 300), (200, 4096, 130)])
def test_int8_with_everything_in_the_epilogue(kind, rows, k, n):
    t = TYPES[kind]
    x, w = draw(1, rows, k, dtype=t), draw(2, n, k, dtype=t, scale=k ** -0.5)
    b, r = draw(3, n, dtype=t), draw(4, rows, n, dtype=t)
    q, s = gd.quantise_rows(x)
    wq, ws = gd.quantise_rows(w)
    op = gd.Linear(k, n, t, "silu", max_rows=rows)
    y = op.forward_int8(q, s, wq, ws, b, r)
    z = (d(q) @ d(wq).t()) * d(s)[:, None] * d(ws)[None, :]
    off = 4 * E * z.abs() + E * d(b).abs()
    z = z + d(b)
    a = plain.act("silu", z) + d(r)
    close(y, a, 1.2 * off + 16 * E * (z.abs() + a.abs()) + rounded(a, t), "int8")
    # and near the layer in the type: each operand is off by at most half a 127th of its row's largest
    full = d(x) @ d(w).t()
    near = 0.5 / 127 * (d(x).abs().amax(1, keepdim=True) * d(w).abs().sum(1)[None, :]
                        + d(x).abs().sum(1, keepdim=True) * d(w).abs().amax(1)[None, :]) * 1.01
    close(z - d(b), full, near, "quantised product")


def test_long_sums_and_row_independence():
    """A single row gives the same result alone and among others where the form is the same; long k stays exact
    enough in 32 bits."""
    k, n = 16384, 48
    w = draw(2, n, k, dtype=torch.bfloat16)
    for rows in (1, 16, 30):
        x = draw(1, rows, k, dtype=torch.bfloat16)
        op = gd.Linear(k, n, torch.bfloat16, max_rows=rows)
        check_forward(op, x, w, None, None, op.forward(x, w), None, f"{rows} rows")
    x = draw(1, 16, k, dtype=torch.bfloat16)
    op = gd.Linear(k, n, torch.bfloat16, max_rows=16)
    assert torch.equal(op.forward(x, w)[3], op.forward(x[3:4], w)[0])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 40, 150])
def test_strides_offsets_and_outputs_in_place(kind, rows):
    """Operands inside wider buffers that start off any alignment (slices of flat parameters and gradients)."""
    t, k, n = TYPES[kind], 100, 77
    x = draw(1, rows, k + 9, dtype=t)[:, 3:3 + k]
    flat = draw(2, n * k + n + 5, dtype=t)
    w, b = flat[1:1 + n * k].view(n, k), flat[1 + n * k:1 + n * k + n]
    r = draw(3, rows, n + 3, dtype=t)[:, 2:2 + n]
    op = gd.Linear(k, n, t, "gelu", max_rows=rows)
    out, pre = torch.full((rows, n + 5), -7.0, dtype=t, device="cuda"), torch.full((rows, n + 4), -7.0, dtype=t, device="cuda")
    y, p = op.forward(x, w, b, r, out=out[:, 1:1 + n], keep_pre=pre[:, 3:3 + n])
    check_forward(op, x, w, b, r, y, p, "strided")
    assert float((out[:, 0] + 7).abs().sum() + (out[:, 1 + n:] + 7).abs().sum()) == 0
    assert float((pre[:, :3] + 7).abs().sum() + (pre[:, 3 + n:] + 7).abs().sum()) == 0
    want = y.clone()
    op.forward(x, w, b, r, out=r)
    assert torch.equal(r, want)
    grad = torch.full((n * k + n + 5,), -7.0, device="cuda")
    dy = draw(5, rows, n + 1, dtype=t)[:, 1:]
    got = op.backward(dy, x, w, p, dweight=grad[3:3 + n * k].view(n, k), dbias=grad[3 + n * k:3 + n * k + n])
    check_backward(op, dy, x, w, p, got, "strided")
    assert float((grad[:3] + 7).abs().sum() + (grad[3 + n * k + n:] + 7).abs().sum()) == 0
    again = op.backward(dy, x, w, p, dbias=True, dz=dy)  # dz over dy
    assert again[3] is dy and torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    wide = torch.full((n, k + 6), -7.0, device="cuda")
    op.backward(got[3], x, w, p, dz=torch.empty_like(got[3]), dweight=wide[:, 2:2 + k], need_dx=False)
    assert float((wide[:, :2] + 7).abs().sum() + (wide[:, 2 + k:] + 7).abs().sum()) == 0


@pytest.mark.parametrize("act", ["none", "relu"])
def test_accumulate_shared_weights_and_no_rows(act):
    """Gradients of a layer used twice add up; no rows give zeros, or add nothing."""
    k, n, t = 60, 30, torch.float32
    op = gd.Linear(k, n, t, act, max_rows=64)
    xs, dys, w = [whole(i, 64, k) for i in (1, 2)], [whole(i, 64, n) for i in (3, 4)], whole(5, n, k)
    pres = [op.forward(x, w, keep_pre=True)[1] for x in xs]
    parts = [op.backward(dy, x, w, p, dbias=True) for dy, x, p in zip(dys, xs, pres)]
    dw, db = parts[0][1].clone(), parts[0][2].clone()
    op.backward(dys[1], xs[1], w, pres[1], dweight=dw, dbias=db, accumulate=True)
    assert torch.equal(dw, parts[0][1] + parts[1][1]) and torch.equal(db, parts[0][2] + parts[1][2])
    none_x, none_y = torch.empty(0, k, device="cuda"), torch.empty(0, n, device="cuda")
    assert op.forward(none_x, w).shape == (0, n)
    kept = dw.clone()
    op.backward(none_y, none_x, w, none_y, dweight=dw, dbias=db, accumulate=True)
    assert torch.equal(dw, kept)
    dx, _, _, _ = op.backward(none_y, none_x, w, none_y, dweight=dw, dbias=db)
    assert dx.shape == (0, k) and float(dw.abs().sum() + db.abs().sum()) == 0


def test_gradients_against_differences():
    rows, k, n = 3, 12, 7
    x, w, b, c = draw(1, rows, k), draw(2, n, k), draw(3, n), draw(4, rows, n)
    for act in ("gelu", "silu", "none"):
        op = gd.Linear(k, n, torch.float32, act, max_rows=rows)
        _, pre = op.forward(x, w, b, keep_pre=True)
        dx, dw, db, _ = op.backward(c, x, w, pre, dbias=True)
        loss = lambda X, W, B: float((plain.act(act, X @ W.t() + B) * d(c)).sum())  # noqa: E731
        for at, grad in ((0, dx), (1, dw), (2, db)):
            for i in range(0, grad.numel(), 5):
                lo, hi = [d(v).clone() for v in (x, w, b)], [d(v).clone() for v in (x, w, b)]
                lo[at].view(-1)[i] -= 1e-6
                hi[at].view(-1)[i] += 1e-6
                assert abs((loss(*hi) - loss(*lo)) / 2e-6 - float(grad.view(-1)[i])) < 1e-4


@pytest.mark.parametrize("rows", [4, 100])
def test_values_that_are_not_finite_stay_in_their_row(rows):
    k, n = 200, 70
    x, w = draw(1, rows, k, dtype=torch.bfloat16), draw(2, n, k, dtype=torch.bfloat16)
    clean = gd.Linear(k, n, max_rows=rows).forward(x, w)
    x[1, 3], x[2, k - 1] = math.nan, math.inf
    for act in ("none", "relu", "gelu", "silu"):
        y = gd.Linear(k, n, act=act, max_rows=rows).forward(x, w)
        assert bool(y[1].isnan().all()) and not bool(y[2].isfinite().all())
        if act == "none":
            assert torch.equal(y[0], clean[0]) and torch.equal(y[3:], clean[3:])
    # float16 results past its range are infinities, as the type has it
    big = torch.full((rows, k), 60.0, dtype=torch.float16, device="cuda")
    assert bool(gd.Linear(k, n, torch.float16, max_rows=rows).forward(big, torch.full((n, k), 60.0, dtype=torch.float16, device="cuda")).isinf().all())


def test_extreme_inputs_of_activations():
    """Far tails: the activations and their slopes are 0 or 1 there, not NaN."""
    z = torch.tensor([[-1e30, -200.0, -89.0, -20.0, -0.0, 0.0, 20.0, 89.0, 200.0, 1e30]], device="cuda")
    eye = torch.eye(10, device="cuda")
    for act in ("relu", "gelu", "silu"):
        op = gd.Linear(10, 10, torch.float32, act, max_rows=1)
        y, pre = op.forward(z, eye, keep_pre=True)
        assert bool(y.isfinite().all()) and bool((y[0, 8:] == z[0, 8:]).all()) and float(y[0, :3].abs().max()) < 1e-30
        dz = op.backward(torch.ones_like(z), z, eye, pre)[3]
        assert bool(dz.isfinite().all()) and bool((dz[0, 7:] == 1).all()) and float(dz[0, :3].abs().max()) < 1e-30


def test_streams_graphs_and_shared_handles():
    """One handle for two layers, on another stream, and captured and replayed between other work."""
    k, n, rows = 500, 300, 60
    x, dy = draw(1, rows, k, dtype=torch.bfloat16), draw(2, rows, n, dtype=torch.bfloat16)
    ws = [draw(3 + i, n, k, dtype=torch.bfloat16) for i in range(2)]
    op = gd.Linear(k, n, act="silu", max_rows=rows)

    def work(**more):
        out = []
        for w in ws:
            y, pre = op.forward(x, w, keep_pre=True, **more)
            out += [y, pre, *[t for t in op.backward(dy, x, w, pre, dbias=True, **more)]]
        return out

    want = work()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = work(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for seed in range(3):
        x.copy_(draw(20 + seed, rows, k, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for a, b in zip(work(), got):
            assert torch.equal(a, b)


def test_refusals():
    for k, n, most in ((0, 4, 1), (4, 0, 1), (1 << 23, 4, 1), (4, 1 << 23, 1), (4, 4, 1 << 31), (1 << 33, 4, 1)):
        with pytest.raises(gd.GDError):
            gd.Linear(k, n, max_rows=most)
    with pytest.raises(ValueError):
        gd.Linear(4, 4, act="tanh")
    with pytest.raises(TypeError):
        gd.Linear(4, 4, torch.float64)
    k, n, t = 32, 24, torch.bfloat16
    op = gd.Linear(k, n, act="relu", max_rows=8)
    x, w, b, y = draw(1, 8, k, dtype=t), draw(2, n, k, dtype=t), draw(3, n, dtype=t), draw(4, 8, n, dtype=t)
    with pytest.raises(gd.GDError):  # more rows than planned
        op.forward(draw(1, 9, k, dtype=t), w)
    for args in ((x.float(), w), (x, w.cpu()), (x, w.half()), (x, w, b.float())):
        with pytest.raises(TypeError):
            op.forward(*args)
    for args in ((x[:, :31], w), (x, w[:23]), (x, w, b[:23].contiguous()), (x, w, b, y[:7]), (x, w.t().contiguous().t())):
        with pytest.raises(ValueError):
            op.forward(*args)
    with pytest.raises(ValueError):
        op.backward(y, x, w)  # no pre
    with pytest.raises(ValueError):
        op.backward(y, x, w, y, accumulate=True)
    with pytest.raises(TypeError):
        op.backward(y, x, w, y, dweight=torch.empty(n, k, dtype=t, device="cuda"))
    q, s = gd.quantise_rows(x)
    with pytest.raises(TypeError):
        op.forward_int8(x, s, q, s)
    with pytest.raises(TypeError):
        op.forward_int8(q, None, q[:1].expand(n, k).contiguous(), s)
    long = gd.Linear(131073, 1, max_rows=1)
    one = torch.ones(1, 131073, dtype=torch.int8, device="cuda")
    with pytest.raises(gd.GDError):
        long.forward_int8(one, torch.ones(1, device="cuda"), one, torch.ones(1, device="cuda"))
    with pytest.raises(ValueError):
        gd.quantise_rows(torch.empty(3, 0, device="cuda"))
    with pytest.raises(TypeError):
        gd.quantise_rows(torch.empty(3, 4, dtype=torch.float64, device="cuda"))
