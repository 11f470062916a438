"""Both halves of a gated layer's dz where ReLU's gate is NaN, as the header has them."""
import math

import pytest
import torch

from paper_1704_05021_amd import gd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [5, 16])
def test_a_gate_that_is_nan_under_relu(kind, n):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    op = gd.GatedLinear(2, n, kind, "relu", max_rows=1)
    pre = torch.ones(1, 2 * n, dtype=kind, device="cuda")
    pre[0, :4] = torch.tensor([math.nan, 0.0, -1.0, -math.inf])
    for dy in (2.0, 0.0, math.inf, math.nan):
        dz = op.backward(torch.full((1, n), dy, dtype=kind, device="cuda"), pre[:, :2].contiguous(), pre.view(2 * n, 1).expand(2 * n, 2).contiguous(), pre)[3][0]
        assert not bool(dz[:4].any()) and bool(dz[n].isnan()) and not bool(dz[n + 1:n + 4].any()), dy
        want = torch.full((n - 4,), dy, dtype=kind, device="cuda")
        assert torch.equal(dz[4:n].nan_to_num(9.0), want.nan_to_num(9.0)) and torch.equal(dz[n + 4:].nan_to_num(9.0), want.nan_to_num(9.0))
