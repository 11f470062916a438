"""The norm's backward pass where every block takes several turns: rows past what the blocks hold at once, for every
shape of the kernel, with the last turn whole, partly filled and missing in some blocks."""
import math

import pytest
import torch

import launch_stub
import plain_ops as plain
from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, close, d, rounded

# rows, dim, and the kernel's waves a row and vectors a thread
CASES = [(8192, 500, 1, 1), (9003, 40, 1, 1), (5000, 512, 1, 1), (4096, 640, 2, 1), (6151, 1024, 2, 1), (3071, 1100, 4, 1),
         (2049, 2000, 4, 1), (1536, 4096, 8, 1), (1301, 2056, 8, 1), (600, 8192, 16, 1), (513, 5000, 16, 1), (770, 9001, 16, 2),
         (512, 16384, 16, 2), (530, 20000, 16, 4), (258, 32768, 16, 4)]


def rows_per_block(rows, dim):
    """At least this many rows go to some block, by the number of blocks that a launch may have."""
    waves = next(w for at, w in ((512, 1), (1024, 2), (2048, 4), (4096, 8), (1 << 20, 16)) if dim <= at)
    blocks = {1: 1024, 2: 1024, 4: 1024, 8: 512, 16: 256}[waves]
    return math.ceil(rows / blocks)


def test_the_cases_take_several_turns(tmp_path):
    launch_stub.run(f"CASES = {CASES!r}" + """
shapes = set()
for rows, dim, waves, v in CASES:
    for ty, name in ((0, "f"), (1, "DF16b"), (2, "DF16_")):
        n = made("norm", dim, ty)
        f = dict(rows=rows, dy=P, x=P, weight=P, dx=P, dweight=P, dy_stride=dim, x_stride=dim, dx_stride=dim, eps=1e-6)
        back, join = launches(lambda: G.gd_norm_backward(n, io(gd._NormGrad, **f), None))
        assert join["name"] == "k_sum_parts" and back["what"].startswith(f"_ZN2gd11k_norm_backI{name}Li{waves}ELi{v}EE"), back
        rows_a_turn = back["block"] // (waves * 64)
        turns = -(-rows // rows_a_turn)
        assert 1 < back["grid"][0] < turns, (rows, dim, back["grid"], turns)
        shapes.add((waves, v, turns % back["grid"][0] == 0))
        G.gd_norm_destroy(n)
# each shape with the same number of turns in every block, or with fewer in some; both for most
assert {s[:2] for s in shapes} == {(1, 1), (2, 1), (4, 1), (8, 1), (16, 1), (16, 2), (16, 4)}
assert {s[:2] for s in shapes if s[2]} >= {(1, 1), (2, 1), (8, 1), (16, 2)} and len({s[:2] for s in shapes if not s[2]}) == 7
""", tmp_path)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim,waves,vectors", CASES)
def test_backward(kind, rows, dim, waves, vectors):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    t, g = TYPES[kind], torch.Generator().manual_seed(rows + dim)
    draw = lambda *s: torch.randn(*s, generator=g).to(t).cuda()  # noqa: E731
    x, dy, dsum, w = draw(rows, dim), draw(rows, dim), draw(rows, dim), draw(dim)
    op = gd.RMSNorm(dim, t)
    dx, dw = op.backward(dy, x, w, dsum=dsum)
    DX, DW, size, wsize = plain.norm_back(d(dy), d(x), d(w), d(dsum), 1e-6)
    close(dx, DX, rounded(DX, t) + 8 * E * size, "dx")
    # a product, its factor and its share of the block's sum, which takes a rounding a row
    close(dw, DW, (8 + rows_per_block(rows, dim)) * E * wsize, "dweight")
    total, over = dw.clone(), dy.clone()
    dx2, _ = op.backward(over, x, w, dsum=dsum, dx=over, dweight=total, accumulate=True)  # dx over dy, rows ahead being read
    assert torch.equal(dx2, dx)
    # the sum that dw is rounded from is added in 64 bits: a rounding of dw and one of the total
    close(total, 2 * d(dw), 3.01 * E * d(dw).abs(), "accumulated")


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [(1 << 22) + 5, (1 << 23) - 4])
def test_forward_and_row_codes_of_more_rows_than_a_grid_holds(rows):
    """A block takes four rows of up to 512 elements; past 2^20 blocks they go round, the last turn partly filled."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    dim, eps = 5, 1e-6
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, r = (torch.randn(rows, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(dim, generator=g, device="cuda").bfloat16()
    op = gd.RMSNorm(dim, eps=eps)
    y, h = op.forward(x, w, r)
    H = x.double() + r.double()
    Y = H / torch.sqrt((H * H).mean(1, keepdim=True) + eps) * w.double()
    half = torch.finfo(torch.bfloat16).eps / 2
    assert bool(((h.double() - H).abs() <= (half + E) * H.abs() + 2.0 ** -133).all())
    assert bool(((y.double() - Y).abs() <= (half + 5 * E) * Y.abs() + 2.0 ** -133).all())
    q, scale, h8 = op.forward_int8(x, w, r)
    step = Y.abs().amax(1, keepdim=True) / 127
    assert torch.equal(h8, h) and bool(((scale.double() - step[:, 0]).abs() <= 8 * E * step[:, 0]).all())
    assert bool(((q.double() * scale.double()[:, None] - Y).abs() <= step * (0.5 + 16 * E * 127)).all())
    q, scale = gd.quantise_rows(x)
    big = x.float().abs().amax(1, keepdim=True)
    assert torch.equal(scale, torch.div(big, torch.full_like(big, 127.0))[:, 0])
    assert torch.equal(q, torch.round(x.float() * (127.0 * torch.div(torch.ones_like(big), big))).to(torch.int8))
