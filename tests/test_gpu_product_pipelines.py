"""The matrix products where k is long enough for their loops to run in step: every tile in every form, through LDS
directly and through registers, k ending inside a step, rows and columns ending inside a tile.  Sums of small whole
numbers are exact, so a load that comes too late or a place overwritten too early shows as a wrong result."""
import pytest
import torch

import launch_stub
from paper_1704_05021_amd import gd

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# results i and j for which a tile is taken: the forward call's and the input's gradient, the weight's gradient
SIZES = {(64, 64): ((72, 72), (72, 72)), (128, 128): ((1504, 1504), (1504, 1504)), (256, 128): ((1504, 3000), (1504, 3000)),
         (256, 192): ((3000, 2816), None), (256, 256): ((3000, 4080), (3000, 3000))}
STEP = {"f32": 32, "bf16": 64, "f16": 64, "int8": 128}  # k of a step


def cases():
    """(form, operand type, result type, tile, direct, i, j, k, splits)"""
    out = []
    for kind in ("bf16", "f16", "f32"):
        for form in ("forward", "dx", "dw"):
            for tile, sizes in SIZES.items():
                ij = sizes[form == "dw"]
                for direct in ((True, False) if kind != "f32" else (False,)):
                    if ij is None or (not direct and tile[0] > 128):
                        continue
                    for steps in (5, 8, 17):
                        out.append((form, kind, kind, tile, direct, *ij, STEP[kind] * steps + 8, 1))
        for tile, sizes in SIZES.items():
            for direct in (True, False):
                if direct or tile[0] <= 128:
                    for steps in (5, 8):
                        out.append(("forward", "int8", kind, tile, direct, *sizes[0], STEP["int8"] * steps + 16, 1))
    # shares of k, each long enough
    for form in ("forward", "dx", "dw"):
        out.append((form, "f32", "f32", (128, 128), False, 1504, 1504, 4104, 3))
        out += [(form, "bf16", "bf16", (64, 64), direct, 72, 72, 4104, 11) for direct in (True, False)]
    return out


CASES = cases()
# both products of a backward call in one launch: rows, in, out
PAIRS = [(kind, direct, rows, 72, n) for kind in ("bf16", "f16", "f32") for direct in (True, False) for rows, n in ((392, 456), (648, 328))
         if direct <= (kind != "f32")]


def layer_of(form, i, j, k):
    """rows, in and out of the layer whose call this product is."""
    return {"forward": (j, k, i), "dx": (j, i, k), "dw": (k, i, j)}[form]


def test_the_cases_take_these_tiles_and_steps(tmp_path):
    """So that other costs of the tiles cannot quietly leave one of them out."""
    launch_stub.run(f"CASES, PAIRS, STEP = {CASES!r}, {PAIRS!r}, {STEP!r}" + """
types = {"f32": ("f", 0), "bf16": ("DF16b", 1), "f16": ("DF16_", 2), "int8": ("a", None)}
shape = {(64, 64): (2, 2, 2, 2, 4), (128, 128): (2, 2, 4, 4, 2), (256, 128): (2, 4, 8, 2, 2), (256, 192): (2, 4, 8, 3, 2), (256, 256): (2, 4, 8, 4, 2)}
def tile_name(t): return "NS_4TileI" + "".join(f"Li{x}E" for x in shape[t])
def backward(l, rows, k, n, off, **more):
    f = dict(rows=rows, dy=P + off, x=P, weight=P, dy_stride=n, x_stride=k, weight_stride=k, dx_stride=k, dweight_stride=k)
    return launches(lambda: G.gd_linear_backward(l, io(gd._LinearGrad, **f, **more), None))
for form, e, o, tile, direct, i, j, k, splits in CASES:
    rows, inf, outf = {"forward": (j, k, i), "dx": (j, i, k), "dw": (k, i, j)}[form]
    l = made("linear", inf, outf, types[o][1], 0, rows)
    off = 0 if direct else {"int8": 1, "f32": 0}.get(e, 2)
    if form == "forward":
        f = dict(rows=rows, x=P + off, weight=P, y=P, x_stride=k, weight_stride=k, y_stride=i)
        if e == "int8": f.update(x_scale=P, weight_scale=P)
        log = launches(lambda: G.gd_linear_forward(l, io(gd._LinearIO, **f), None))
    else:
        log = backward(l, rows, inf, outf, off, **({"dx": P} if form == "dx" else {"dweight": P}))
    g, what = log[0], (form, e, o, tile, direct, log[0])
    assert g["name"] == ("k_gemm_fetch" if direct else "k_gemm") and len(log) == 1 + (splits > 1), what
    assert tile_name(tile) in g["what"] and f"Lb{int(form != 'forward')}ELb{int(form == 'dw')}E" in g["what"], what
    assert re.search(r"k_gemm(_fetch)?I" + types[e][0], g["what"]), what
    a = g["args"]
    assert (a["I"], a["J"], a["K"]) == (i, j, k) and g["grid"][1] == splits, what
    assert i % tile[0] and j % tile[1] and k % STEP[e], what
    assert min(a["steps"], k // STEP[e]) >= 5, what  # whole steps of a share
    G.gd_linear_destroy(l)
for kind, direct, rows, k, n in PAIRS:
    l = made("linear", k, n, types[kind][1], 0, rows)
    log = backward(l, rows, k, n, 0 if direct or kind == "f32" else 2, dx=P, dweight=P)
    assert [x["name"] for x in log] == ["k_gemm_pair"] and f"k_gemm_pairI{types[kind][0]}Lb{int(direct)}E" in log[0]["what"], log
    assert min(rows, n) // STEP[kind] >= 5 and rows % STEP[kind] and n % STEP[kind]
    G.gd_linear_destroy(l)
""", tmp_path)


def whole(seed, rows, columns, kind, off=0):
    """Small whole numbers, `off` elements into their buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    most = 127 if kind is torch.int8 else 3
    flat = torch.randint(-most, most + 1, (rows * columns + off,), generator=g, device="cuda").to(kind)
    return flat[off:].view(rows, columns)


def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def exact(a, b):
    return a.double() @ b.double()


@pytest.mark.gpu
@pytest.mark.parametrize("form,e,o,tile,direct,i,j,k,splits", CASES)
def test_products(form, e, o, tile, direct, i, j, k, splits):
    need_gpu()
    rows, inf, outf = layer_of(form, i, j, k)
    op, t, off = gd.Linear(inf, outf, TYPES[o], max_rows=rows), TYPES[o], 0 if direct or e == "f32" else 1
    for seed in (1, 2):
        if e == "int8":
            q, wq = whole(seed, rows, inf, torch.int8, off), whole(seed + 9, outf, inf, torch.int8)
            s, ws = torch.full((rows,), 0.5, device="cuda"), torch.full((outf,), 2.0 ** -12, device="cuda")
            want = (exact(q, wq.t()).float() * 2.0 ** -13).to(t)  # one rounding of the exact sum, then powers of two
            call = lambda: op.forward_int8(q, s, wq, ws)  # noqa: E731
        elif form == "forward":
            x, w = whole(seed, rows, inf, t, off), whole(seed + 9, outf, inf, t)
            want, call = exact(x, w.t()).to(t), lambda: op.forward(x, w)
        elif form == "dx":
            dy, w = whole(seed, rows, outf, t, off), whole(seed + 9, outf, inf, t)
            want, call = exact(dy, w).to(t), lambda: op.backward(dy, None, w, need_dweight=False)[0]
        else:
            dy, x = whole(seed, rows, outf, t, off), whole(seed + 9, rows, inf, t)
            want, call = exact(dy.t(), x).float(), lambda: op.backward(dy, x, None, need_dx=False)[1]
        for _ in range(3):
            assert torch.equal(call(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,direct,rows,k,n", PAIRS)
def test_both_products_in_one_launch(kind, direct, rows, k, n):
    need_gpu()
    t = TYPES[kind]
    op = gd.Linear(k, n, t, max_rows=rows)
    for seed in (1, 2):
        dy, x, w = whole(seed, rows, n, t, 0 if direct or kind == "f32" else 1), whole(seed + 3, rows, k, t), whole(seed + 6, n, k, t)
        want = exact(dy, w).to(t), exact(dy.t(), x).float()
        for _ in range(3):
            dx, dw, _, _ = op.backward(dy, x, w)
            assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
