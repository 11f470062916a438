"""Alternatives of rows of which very many logits are above the bound that the threads' largest give: the scan that takes
the next largest each time, on finite rows."""
import pytest
import torch

from paper_1704_05021_amd import gd
from plain_ops import TYPES
from test_gpu_scores import check_scores, ids_of

pytestmark = pytest.mark.gpu

TOP = 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def piece_elements(rows, vocab):
    """Elements that a block takes of a row at a time: few long rows are cut."""
    pieces = min(512 // rows, vocab // 4096, 64, 1024 // TOP) if rows < 256 and vocab >= 8192 else 1
    each = (vocab + pieces - 1) // pieces
    return (each + 7) // 8 * 8


# one wave a row, four, eight, and rows in pieces
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(3, 1203), (3, 2048), (1030, 2100), (300, 9000), (260, 51_000), (2, 40_000), (1, 85_000)])
@pytest.mark.parametrize("low", [-50.0, -1e30])
def test_a_group_of_lanes_that_holds_only_low_logits(kind, rows, vocab, low):
    g = torch.Generator().manual_seed(7)
    x = torch.randn(rows, vocab, generator=g) * 3.0
    e = torch.arange(vocab) % piece_elements(rows, vocab)
    mine = e // 8 % 64 == 5  # what one of a wave's lanes reads of every turn
    x[:, mine] = low
    assert int((~mine).sum()) > 1024
    x, tokens = x.to(TYPES[kind]).cuda(), ids_of(1, vocab, rows)
    r = gd.TokenLogProbs(vocab, TYPES[kind], max_rows=rows).forward(x, tokens, top=TOP)
    check_scores(r, x, tokens, 1.0, TOP, f"{kind} {rows}x{vocab}")
