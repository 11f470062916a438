"""A step is skipped exactly when the norm that the caller gets is not finite: finite gradients can have one past
binary32's range."""
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


def once(bits, g, **more):
    """(norm, buffers before, buffers after) of a second step."""
    n = g.numel()
    opt = gd.AdamW([0, 500, n], bits=bits)
    first = torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda()
    p, copy, state = first.clone(), torch.zeros(n, dtype=torch.bfloat16, device="cuda"), opt.init_state()
    opt.step(p, first, state, 1, lr=1e-3, copy=copy)
    held = [t for t in (p, copy, state.m, state.v, state.m_unit, state.v_unit) if t is not None]
    before = [t.clone() for t in held]
    norm = opt.step(p, g, state, 2, lr=1e-3, copy=copy, **more)
    return float(norm), before, held


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1.0, math.inf])
def test_finite_gradients_with_a_norm_past_the_range(bits, kind, max_norm):
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[kind]
    g = torch.full((1234,), 1e38).to(t).cuda()  # norm about 3.5e39
    norm, before, after = once(bits, g, max_norm=max_norm)
    assert norm == math.inf
    for a, b in zip(before, after):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [1.0, -2.0 ** -40])
def test_the_last_norms_within_the_range_take_the_step(bits, scale):
    """Four elements of 2^126 have the norm 2^127; scaled, the same ones of up to the type's largest have a small one."""
    g = torch.zeros(1000, device="cuda")
    g[[0, 400, 600, 999]] = 2.0 ** 126 if scale == 1.0 else 3.4e38
    norm, before, after = once(bits, g, max_norm=1.0, grad_scale=scale)
    want = 2.0 ** 127 if scale == 1.0 else 2 * float(g[0]) * 2.0 ** -40
    assert abs(norm - want) <= 2.0 ** -22 * want
    assert all(bool(t.float().isfinite().all()) for t in after)
    assert not torch.equal(before[0], after[0]) and not torch.equal(before[2], after[2])
