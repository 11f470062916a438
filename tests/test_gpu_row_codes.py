"""The codes of rows in 8 bits are those of the stated operations in binary32, bit for bit, the middles of two codes
included."""
import pytest
import torch

from paper_1704_05021_amd import gd

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def codes(x):
    """The definition on the CPU, each operation rounded to binary32."""
    x = x.cpu().float()
    big = x.abs().amax(1, keepdim=True)
    step = 127.0 * (torch.ones_like(big) / big)
    return torch.round(x * step).to(torch.int8), (big / 127.0)[:, 0]


def rows_with_middles(rows, columns, kind):
    """Normal rows whose every fourth value is half the row's largest: 63.5 of its steps, the middle of two codes."""
    g = torch.Generator().manual_seed(rows * 1000 + columns)
    x = torch.randn(rows, columns, generator=g).to(kind)
    half = x.abs().amax(1, keepdim=True) * 0.5
    x[:, 1::4] = torch.where(x[:, 1::4] < 0, -half, half)
    return x.cuda()


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("rows,columns", [(300, 100), (40, 4096), (20, 5001), (5, 40000)])
def test_rows(kind, rows, columns):
    x = rows_with_middles(rows, columns, TYPES[kind])
    q, scale = gd.quantise_rows(x)
    want, ws = codes(x)
    assert torch.equal(q.cpu(), want) and torch.equal(scale.cpu(), ws)


@pytest.mark.parametrize("rows,dim", [(200, 300), (50, 4096), (7, 9001)])
def test_norm(rows, dim):
    """The norm's codes are those of its own output in binary32."""
    x, r = rows_with_middles(rows, dim, torch.float32), rows_with_middles(rows, dim, torch.float32).flip(0)
    w = torch.ones(dim, device="cuda")
    op = gd.RMSNorm(dim, torch.float32)
    for residual in (None, r):
        y, _ = op.forward(x, w, residual)
        q, scale, _ = op.forward_int8(x, w, residual)
        want, ws = codes(y)
        assert torch.equal(q.cpu(), want) and torch.equal(scale.cpu(), ws)
