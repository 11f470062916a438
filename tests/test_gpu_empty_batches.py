"""Batches of no rows through every call of the layers: empty results, no error."""
import pytest
import torch

import hip_stub
import test_operator_checks
from paper_1704_05021_amd import gd


def test_no_rows_need_no_scales(tmp_path):
    """An empty tensor's address may be NULL: with the weight's scales beside it, that is no missing scale."""
    hip_stub.run(f"ROOT, LIB = {hip_stub.ROOT!r}, {hip_stub.LIB!r}" + test_operator_checks.COMMON + """
l = made("linear", 64, 48, 1, 1, 100)
f = dict(rows=0, weight=P, weight_scale=P, x_stride=64, weight_stride=64, y_stride=48)
assert call("gd_linear_forward", l, io(gd._LinearIO, **f)) == (0, 0)
assert call("gd_linear_forward", l, io(gd._LinearIO, **but(f, rows=1, x=P, y=P)))[0] == 1
""", tmp_path)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(0,), (3, 0)])
def test_every_call(kind, shape):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    k, n = 24, 40
    draw = lambda *s: torch.randn(*s, device="cuda").to(kind)  # noqa: E731
    x, dy, w, gain, b = draw(*shape, k), draw(*shape, n), draw(n, k), draw(k), draw(n)
    norm, layer = gd.RMSNorm(k, kind), gd.Linear(k, n, kind, "gelu", max_rows=8)
    y, h = norm.forward(x, gain, x)
    q, scale, h8 = norm.forward_int8(x, gain, x)
    assert y.shape == h.shape == q.shape == h8.shape == x.shape and scale.shape == shape
    out, pre = layer.forward(x, w, b, keep_pre=True)
    wq, ws = gd.quantise_rows(w)
    q2, scale2 = gd.quantise_rows(x)
    assert q2.shape == x.shape and scale2.shape == shape
    out8 = layer.forward_int8(q, scale, wq, ws, b)
    assert out.shape == pre.shape == out8.shape == (*shape, n) and out8.dtype is kind
    dx, dw, db, dz = layer.backward(dy, x, w, pre, dbias=True)
    assert dx.shape == x.shape and dz.shape == dy.shape and float(dw.abs().sum() + db.abs().sum()) == 0
    dx, dgain = norm.backward(x, h, gain)
    assert dx.shape == x.shape and float(dgain.abs().sum()) == 0
