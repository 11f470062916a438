"""Large products of layers whose widths are whole 16-byte chunks, with operands that are not at 16-byte boundaries, as
slices of a flat buffer behind a ragged tensor are; and of 8-bit operands with k no multiple of 16.  Exact on whole
numbers, and what lies around the operands reaches no result."""
import math

import pytest
import torch

from paper_1704_05021_amd import gd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def whole(seed, rows, columns, kind, off, most=3):
    """Small whole numbers `off` elements into a buffer that holds NaN (127 in 8 bits) around them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * columns + off + 8,), 127 if kind is torch.int8 else math.nan, device="cuda").to(kind)
    inner = flat[off:off + rows * columns].view(rows, columns)
    inner.copy_(torch.randint(-most, most + 1, (rows, columns), generator=g, device="cuda"))
    return inner


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("at", [(1, 0, 0), (0, 1, 0), (0, 0, 3), (5, 7, 1)])
def test_16_bits(kind, at):
    """The input, the weight or the gradient off the boundary, or all of them."""
    rows, k, n = 2101, 2200, 2056
    x, w, dy = (whole(i, *s, kind, off) for i, s, off in ((1, (rows, k), at[0]), (2, (n, k), at[1]), (3, (rows, n), at[2])))
    f = lambda a: a.double()  # noqa: E731
    op = gd.Linear(k, n, kind, max_rows=rows)
    assert torch.equal(op.forward(x, w), (f(x) @ f(w).t()).to(kind))
    dx, dw, db, _ = op.backward(dy, x, w, dbias=True)
    assert torch.equal(dx, (f(dy) @ f(w)).to(kind)) and torch.equal(dw, (f(dy).t() @ f(x)).float())
    assert torch.equal(db, f(dy).sum(0).float())


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("k,at", [(2200, (0, 0)), (4088, (0, 0)), (2208, (1, 0)), (2208, (0, 9))])
def test_8_bits(kind, k, at):
    rows, n = 2101, 2056
    q, wq = whole(4, rows, k, torch.int8, at[0], 100), whole(5, n, k, torch.int8, at[1], 100)
    s, ws = torch.full((rows,), 0.5, device="cuda"), torch.full((n,), 2.0 ** -12, device="cuda")
    want = (q.double() @ wq.double().t()).float() * 2.0 ** -13
    assert torch.equal(gd.Linear(k, n, kind, max_rows=rows).forward_int8(q, s, wq, ws), want.to(kind))
