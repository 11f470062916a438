"""Gated layers, forward (in the type and with 8-bit operands) and backward, against the 64-bit definition."""
import math

import pytest
import torch

import launch_stub
import plain_ops as plain
from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, close, d, rounded

gpu = pytest.mark.gpu


def draw(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def whole(seed, *shape, dtype=torch.float32, most=1):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype).cuda()


def sums(x, w, b):
    """Both sums and the allowance of forming them in 32 bits."""
    z, off = plain.product(d(x), d(w))
    return (z, off) if b is None else (z + d(b), off + E * (z.abs() + 2 * d(b).abs()))


def check_forward(op, x, w, b, y, pre, what, values=None):
    t, n = op.dtype, op.outf
    z, off = sums(x, w, b) if values is None else values
    if pre is not None:
        close(pre, z, off + rounded(z, t), what + " pre")
    g, u, og, ou = z[:, :n], z[:, n:], off[:, :n], off[:, n:]
    a = plain.act(op.act, g)
    oa = 1.2 * og + 16 * E * (g.abs() + a.abs())  # slopes are below 1.2; the functions are within a few ulps
    y64 = a * u
    close(y, y64, oa * (u.abs() + ou) + a.abs() * ou + E * y64.abs() + rounded(y64, t), what)


def check_backward(op, dy, x, w, pre, got, what):
    t, n = op.dtype, op.outf
    dx, dw, db, dz = got
    g, u, top = d(pre)[:, :n], d(pre)[:, n:], d(dy)
    want = torch.cat([top * u * plain.slope(op.act, g), top * plain.act(op.act, g)], 1)
    # the slope is within 24 roundings of values below 1.2 (1 + |g|), as the linear layer's; one more for the product dy u
    off = torch.cat([25 * E * (top * u).abs() * (1 + g.abs()), 17 * E * top.abs() * (g.abs() + plain.act(op.act, g).abs())], 1)
    close(dz, want, rounded(want, t) + off, what + " dz")
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


SIZES = [(1, 1, 1), (1, 8, 8), (2, 7, 9), (3, 64, 10), (1, 784, 512), (16, 500, 33), (15, 1024, 500), (17, 65, 64),
         (33, 129, 127), (40, 784, 250), (64, 64, 32), (65, 1000, 130), (100, 10, 300), (257, 100, 65), (300, 511, 257)]


@gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_sizes(kind, rows, k, n):
    t = TYPES[kind]
    x, w = draw(1, rows, k, dtype=t), draw(2, 2 * n, k, dtype=t, scale=k ** -0.5)
    b, dy = draw(3, 2 * n, dtype=t), draw(5, rows, n, dtype=t)
    for act in ("none", "relu", "gelu", "silu"):
        op = gd.GatedLinear(k, n, t, act, max_rows=rows)
        for bias in (b, None):
            y, pre = op.forward(x, w, bias, keep_pre=True)
            check_forward(op, x, w, bias, y, pre, f"{kind} {act} {rows}x{k}x{n}")
            assert torch.equal(op.forward(x, w, bias), y)
        got = op.backward(dy, x, w, pre, dbias=True)
        check_backward(op, dy, x, w, pre, got, f"{kind} {act} {rows}x{k}x{n}")


# (rows, in, results) of every tile, whole and ragged, with and without a split of k; single rows; k past a vector's end
TILES = [(256 * 15, 128, 128 * 14), (256 * 14 + 33, 72, 128 * 15 - 20), (128, 256 * 15, 128 * 14), (100, 256 * 14 + 8, 128 * 15 - 9),
         (128 * 15, 136, 64 * 14), (128 * 14 + 5, 200, 64 * 15 - 4), (64, 4096, 32), (90, 4100, 35), (5000, 70, 45),
         (60, 90, 2503), (10, 4096, 2048), (7, 8191, 17), (1, 4096, 4096), (64, 4096, 1500), (3000, 128, 2048), (2990, 136, 2040),
         (2048, 128, 2048), (128, 4096, 1024), (200, 4088, 1020)]


@gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n", TILES)
def test_tiles_are_exact_on_whole_numbers(kind, rows, k, n):
    """Sums and products of whole numbers below 2^24 are exact, so every result is the exact one, rounded once."""
    t = TYPES[kind]
    f = lambda a: a.double()  # noqa: E731
    x, w, dy = whole(1, rows, k, dtype=t), whole(2, 2 * n, k, dtype=t), whole(3, rows, n, dtype=t)
    z = f(x) @ f(w).t()
    assert float((z[:, :n] * z[:, n:]).abs().max()) < 2 ** 24
    op = gd.GatedLinear(k, n, t, "none", max_rows=rows)
    y, pre = op.forward(x, w, keep_pre=True)
    assert torch.equal(pre, z.to(t)) and torch.equal(y, (z[:, :n] * z[:, n:]).to(t))
    relu = gd.GatedLinear(k, n, t, "relu", max_rows=rows)
    assert torch.equal(relu.forward(x, w), (z[:, :n].clamp_min(0) * z[:, n:]).to(t))
    few = whole(6, rows, 2 * n, dtype=t, most=2)  # small inputs of the activation, so that sums over rows stay exact
    dx, dw, db, dz = op.backward(dy, x, w, few, dbias=True)
    want = torch.cat([f(dy) * f(few)[:, n:], f(dy) * f(few)[:, :n]], 1)
    assert torch.equal(f(dz), want) and torch.equal(dx, (want @ f(w)).to(t))
    assert torch.equal(dw, (want.t() @ f(x)).float()) and torch.equal(db, want.sum(0).float())
    q, s = whole(4, rows, k, dtype=torch.int8, most=2), torch.full((rows,), 0.5, device="cuda")
    wq, ws = whole(5, 2 * n, k, dtype=torch.int8, most=1), torch.full((2 * n,), 0.25, device="cuda")
    z = (f(q) @ f(wq).t()) * 0.125
    assert torch.equal(op.forward_int8(q, s, wq, ws), (z[:, :n] * z[:, n:]).to(t))


def guarded(a, seed):
    """a inside a wider buffer of NaN, off any alignment."""
    lead, gap = seed % 5, 1 + seed % 7
    wide = torch.full((a.shape[0] + 2, a.shape[1] + lead + gap), math.nan, dtype=a.dtype, device="cuda")
    inner = wide[1:1 + a.shape[0], lead:lead + a.shape[1]]
    inner.copy_(a)
    return inner


@gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("k", [1, 3, 5, 8, 9, 31, 65, 131])
def test_ends_inside_a_vector(kind, k):
    """Rows and k that end anywhere in a vector: exact sums, and nothing read past the operands reaches them."""
    t, f = TYPES[kind], lambda a: a.double()  # noqa: E731
    for rows in (1, 2, 5, 18, 66, 131):
        for n in (1, 3, 15, 17, 33, 67):
            x, w, dy, pre = (guarded(whole(i + k, *s, dtype=t), rows + n + i)
                             for i, s in enumerate([(rows, k), (2 * n, k), (rows, n), (rows, 2 * n)]))
            op = gd.GatedLinear(k, n, t, "none", max_rows=rows)
            z = f(x) @ f(w).t()
            out = torch.full((rows, n + 3), -9.0, dtype=t, device="cuda")
            kept = torch.full((rows, 2 * n + 3), -9.0, dtype=t, device="cuda")
            op.forward(x, w, out=out[:, 1:1 + n], keep_pre=kept[:, 2:2 + 2 * n])
            assert torch.equal(out[:, 1:1 + n], (z[:, :n] * z[:, n:]).to(t)) and torch.equal(kept[:, 2:2 + 2 * n], z.to(t)), (rows, n)
            assert bool((out[:, [0, n + 1, n + 2]] == -9).all() and (kept[:, [0, 1, 2 * n + 2]] == -9).all()), (rows, n)
            dx, dw, db, _ = op.backward(dy, x, w, pre, dbias=True)
            want = torch.cat([f(dy) * f(pre)[:, n:], f(dy) * f(pre)[:, :n]], 1)
            assert torch.equal(dx, (want @ f(w)).to(t)), (rows, n)
            assert torch.equal(dw, (want.t() @ f(x)).float()) and torch.equal(db, want.sum(0).float()), (rows, n)


STEP = {"f32": 32, "bf16": 64, "f16": 64, "int8": 128}  # k of a step
# results (units, rows) for which a tile is taken: its results in P's rows and Q's
SHAPES = {(64, 64): (36, 72), (128, 128): (752, 1504), (256, 128): (752, 3000), (256, 192): (1500, 2816), (256, 256): (1500, 4080)}
PIPES = [(kind, tile, direct, STEP[kind] * steps + (16 if kind == "int8" else 8), 1)
         for kind in ("bf16", "f16", "f32", "int8") for tile in SHAPES for direct in ((True, False) if kind != "f32" else (False,))
         if direct or tile[0] <= 128 for steps in (5, 8, 17)]
PIPES += [("bf16", (64, 64), True, 4104, 11), ("bf16", (64, 64), False, 4104, 11), ("f32", (128, 128), False, 4104, 3)]


def test_the_cases_take_these_tiles_and_steps(tmp_path):
    """So that other costs of the tiles cannot quietly leave one of them out."""
    launch_stub.run(f"PIPES, SHAPES, STEP = {PIPES!r}, {SHAPES!r}, {STEP!r}" + """
types = {"f32": ("f", 0), "bf16": ("DF16b", 1), "f16": ("DF16_", 2), "int8": ("a", 1)}
shape = {(64, 64): (2, 2, 2, 2, 4), (128, 128): (2, 2, 4, 4, 2), (256, 128): (2, 4, 8, 2, 2), (256, 192): (2, 4, 8, 3, 2), (256, 256): (2, 4, 8, 4, 2)}
for e, tile, direct, k, splits in PIPES:
    n, rows = SHAPES[tile]
    l = made("gated", k, n, types[e][1], 0, rows)
    off = 0 if direct or e == "f32" else 1 if e == "int8" else 2
    f = dict(rows=rows, x=P + off, weight=P, y=P, x_stride=k, weight_stride=k, y_stride=n)
    if e == "int8": f.update(x_scale=P, weight_scale=P)
    log = launches(lambda: G.gd_gated_forward(l, io(gd._GatedIO, **f), None))
    g, what = log[0], (e, tile, direct, k, log[0])
    assert g["name"] == ("k_gemm_fetch" if direct else "k_gemm") and len(log) == 1 + (splits > 1), what
    assert "NS_4TileI" + "".join(f"Li{x}E" for x in shape[tile]) + "EELb1E" in g["what"], what
    assert re.search(r"k_gemm(_fetch)?I" + types[e][0], g["what"]), what
    a = g["args"]
    assert (a["I"], a["J"], a["K"]) == (n, rows, k) and g["grid"][1] == splits, what
    assert g["grid"][0] == -(-2 * n // tile[0]) * -(-rows // tile[1]), what
    assert 2 * n % tile[0] and rows % tile[1] and k % STEP[e], what
    assert min(a["steps"], k // STEP[e]) >= 5, what  # whole steps of a share
    G.gd_gated_destroy(l)
""", tmp_path)


@gpu
@pytest.mark.parametrize("kind,tile,direct,k,splits", PIPES)
def test_pipelines(kind, tile, direct, k, splits):
    """Every tile with 5 to 17 whole steps of k and a rest: a load that comes too late shows as a wrong sum."""
    n, rows = SHAPES[tile]
    t = torch.int8 if kind == "int8" else TYPES[kind]
    off = int(not direct)
    x = whole(1, rows * k + off, dtype=t)[off:].view(rows, k)
    w = whole(2, 2 * n, k, dtype=t)
    z = x.double() @ w.double().t()
    op = gd.GatedLinear(k, n, torch.bfloat16 if kind == "int8" else t, "none", max_rows=rows)
    if kind == "int8":
        y = op.forward_int8(x, torch.ones(rows, device="cuda"), w, torch.ones(2 * n, device="cuda"))
    else:
        y = op.forward(x, w)
    assert torch.equal(y, (z[:, :n] * z[:, n:]).to(op.dtype))


@gpu
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_8_bit_operands(act):
    for rows, k, n in ((1, 100, 40), (16, 1024, 130), (70, 257, 65), (300, 1024, 512)):
        x, w, b = draw(1, rows, k), draw(2, 2 * n, k, scale=k ** -0.5), draw(3, 2 * n, dtype=torch.bfloat16)
        (q, s), (wq, ws) = gd.quantise_rows(x), gd.quantise_rows(w)
        op = gd.GatedLinear(k, n, torch.bfloat16, act, max_rows=rows)
        z = (d(q) @ d(wq).t()) * (d(s)[:, None] * d(ws)) + d(b)
        off = 4 * E * (z.abs() + d(b).abs())  # the exact sum's rounding, its two scales and the bias's sum
        check_forward(op, x, w, b, op.forward_int8(q, s, wq, ws, b), None, f"int8 {act} {rows}", (z, off))


@gpu
@pytest.mark.parametrize("act", ["relu", "gelu", "silu", "none"])
def test_gradients_against_differences(act):
    rows, k, n = 3, 10, 4
    x, w, b, c = draw(1, rows, k), draw(2, 2 * n, k), draw(3, 2 * n), draw(4, rows, n)
    op = gd.GatedLinear(k, n, torch.float32, act, max_rows=rows)
    _, pre = op.forward(x, w, b, keep_pre=True)
    dx, dw, db, _ = op.backward(c, x, w, pre, dbias=True)
    at = [d(x), d(w), d(b)]

    def loss(x, w, b):
        z = x @ w.t() + b
        return float((plain.act(act, z[:, :n]) * z[:, n:] * d(c)).sum())

    step = 1e-6
    for i, got in enumerate((dx, dw, db)):
        for j in range(at[i].numel()):
            ends = []
            for sign in (-1, 1):
                moved = [v.clone() for v in at]
                moved[i].view(-1)[j] += sign * step
                ends.append(loss(*moved))
            want = float(got.view(-1)[j])
            # differences err by about 1e-15 / step and step^2, the kernel by some 30 roundings of values below 100
            assert abs((ends[1] - ends[0]) / (2 * step) - want) < 2e-4 + 1e-5 * abs(want), (i, j)


@gpu
def test_outputs_that_are_given_and_what_is_left_out():
    rows, k, n = 50, 96, 40
    t = torch.bfloat16
    x, w, dy = draw(1, rows, k, dtype=t), draw(2, 2 * n, k, dtype=t), draw(3, rows, n, dtype=t)
    op = gd.GatedLinear(k, n, max_rows=rows)
    y, pre = op.forward(x, w, keep_pre=True)
    dx, dw, db, dz = op.backward(dy, x, w, pre, dbias=True)
    flat = torch.full((2 * n * k + 2 * n + 1,), 0.5, device="cuda")
    kept = pre.clone()
    got = op.backward(dy, x, w, kept, dz=kept, dweight=flat[:2 * n * k].view(2 * n, k), dbias=flat[2 * n * k:-1], accumulate=True)
    assert torch.equal(kept, dz) and torch.equal(got[0], dx) and float(flat[-1]) == 0.5
    close(flat[:2 * n * k], d(dw).flatten() + 0.5, E * d(dw).flatten().abs() + E * (d(dw).flatten() + 0.5).abs(), "accumulated")
    close(flat[2 * n * k:-1], d(db) + 0.5, E * d(db).abs() + E * (d(db) + 0.5).abs(), "accumulated bias")
    only = op.backward(dy, x, w, pre, need_dx=False)
    assert only[0] is None and torch.equal(only[1], dw) and only[2] is None
    only = op.backward(dy, x, w, pre, need_dweight=False)
    assert torch.equal(only[0], dx) and only[1] is None and torch.equal(only[3], dz)


@gpu
def test_relu_turns_units_off():
    """A unit that is off passes nothing, a gradient that is not finite neither."""
    op = gd.GatedLinear(2, 3, torch.float32, "relu", max_rows=2)
    pre = torch.tensor([[-1.0, 0.0, 2.0, 5.0, 6.0, 7.0]] * 2, device="cuda")
    dy = torch.tensor([[math.inf, math.nan, 2.0], [1.0, -math.inf, 3.0]], device="cuda")
    dz = op.backward(dy, draw(1, 2, 2), draw(2, 6, 2), pre)[3]
    assert torch.equal(dz, torch.tensor([[0, 0, 14.0, 0, 0, 4.0], [0, 0, 21.0, 0, 0, 6.0]], device="cuda"))


@gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_a_gate_that_is_nan_passes_nan(act, kind):
    """dz of what is gated is dy act(NaN), in the place of the NaN alone."""
    op = gd.GatedLinear(2, 11, kind, act, max_rows=2)
    pre, dy = draw(1, 2, 22, dtype=kind), draw(2, 2, 11, dtype=kind)
    pre[1, 9] = math.nan
    dz = op.backward(dy, draw(3, 2, 2, dtype=kind), draw(4, 22, 2, dtype=kind), pre)[3]
    gated = torch.zeros(2, 11, dtype=torch.bool, device="cuda")
    gated[1, 9] = True
    assert torch.equal(dz[:, 11:].isnan(), gated) and not bool((dz[:, :11].isnan() & ~gated).any())


@gpu
def test_no_rows_another_stream_and_graph_replays():
    rows, k, n = 300, 256, 192
    t = torch.bfloat16
    x, w, b, dy = draw(1, rows, k, dtype=t), draw(2, 2 * n, k, dtype=t), draw(3, 2 * n, dtype=t), draw(4, rows, n, dtype=t)
    op = gd.GatedLinear(k, n, max_rows=rows)
    none = x[:0]
    grad, gbias = torch.ones(2 * n, k, device="cuda"), torch.ones(2 * n, device="cuda")
    assert op.forward(none, w).shape == (0, n)
    op.backward(dy[:0], none, w, x.new_empty(0, 2 * n), dweight=grad, dbias=gbias, accumulate=True)
    assert bool((grad == 1).all() and (gbias == 1).all())
    op.backward(dy[:0], none, w, x.new_empty(0, 2 * n), dweight=grad, dbias=gbias)
    assert not bool(grad.any() or gbias.any())

    def everything(stream=None):
        y, pre = op.forward(x, w, b, keep_pre=True, stream=stream)
        return [y, pre, *op.backward(dy, x, w, pre, dbias=True, stream=stream), op.forward(x[:3], w, b, stream=stream)]

    want, s = everything(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = everything(s)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for seed in range(3):
        x.copy_(draw(10 + seed, rows, k, dtype=t))
        graph.replay()
        want = everything()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, got))


@gpu
def test_refusals():
    op = gd.GatedLinear(8, 4, torch.float32, max_rows=4)
    x, w, b = draw(1, 3, 8), draw(2, 8, 8), draw(3, 8)
    pre, dy = draw(4, 3, 8), draw(5, 3, 4)
    for bad in (lambda: op.forward(x.bfloat16(), w), lambda: op.forward(x, w.bfloat16()), lambda: op.forward(x, w, b.double()),
                lambda: op.forward(x.cpu(), w)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: op.forward(x[:, :7], w), lambda: op.forward(x, w[:4]), lambda: op.forward(x, w, b[:4]),
                lambda: op.forward(x, w, out=x[:, :4]), lambda: op.forward(x, w, keep_pre=x), lambda: op.backward(dy, x, w, pre[:, :4]),
                lambda: op.backward(dy, x, w, pre, accumulate=True), lambda: op.backward(dy, x, w, pre, dx=x),
                lambda: op.backward(pre[:, :4], x, w, draw(6, 3, 8), dz=pre)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: op.forward(draw(1, 5, 8), w), lambda: gd.GatedLinear(8, 0), lambda: gd.GatedLinear(8, (1 << 21) + 1)):
        with pytest.raises(gd.GDError):
            bad()
    with pytest.raises(ValueError):
        gd.GatedLinear(8, 4, act="tanh")
    with pytest.raises(RuntimeError):
        op.forward(x, w.clone().requires_grad_())
