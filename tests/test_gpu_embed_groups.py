"""The embedding's gradient holds sums in 32 bits for groups of at most 32 rows: rows that a longer group would lose."""
import pytest
import torch

from paper_1704_05021_amd import gd
from plain_ops import E, close, d

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


# a word of 32 rows and fewer by a wave alone, of more by several; sorted, in units of 8, 16 and 32 rows, over several of them
@pytest.mark.parametrize("rows,dim", [(32, 8), (64, 8), (64, 200), (640, 8), (4096, 24), (4160, 8), (9984, 300), (12_800, 520), (32_000, 260)])
@pytest.mark.parametrize("lead", [0, 7])
def test_what_a_group_loses(rows, dim, lead):
    """One in 64 rows is 1, the others are 0.9 of half of its last place: added to it one by one in 32 bits they are lost.
    A group of 32 rows loses 31 of them at most, 27.9 E; one of 64 would lose 56.7 E.  Allowed are the 31 sums of a group, and
    a rounding each of its share, of the joined sum and of the product with the scale."""
    vocab = 5
    dy = torch.full((rows, dim), 0.9 * 2.0 ** -24)
    dy[lead::64] = 1.0
    tokens = torch.full((rows,), 3, device="cuda")
    if lead:
        tokens[:lead] = 1
    dw = gd.Embedding(vocab, dim, torch.float32, scale=1.5, max_rows=rows).backward(dy.cuda(), tokens)
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens.cpu(), d(dy) * 1.5)
    close(dw, want, 34 * E * want.abs(), f"{rows} {dim}")
