"""The example runs as it stands, and the README's layer example gives the gradients of its formulas."""
import importlib.util
import os
import re

import pytest
import torch

import plain_ops as plain
from plain_ops import close, d, rounded

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def test_workers_server_and_decoder():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, agree = example.main(report=lambda *_: None)
    assert losses[0] > 2.0 and losses[-1] < 0.7 * losses[0] and agree >= 0.85, (losses[0], losses[-1], agree)


def test_readme_layers():
    blocks = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), re.S)
    assert len(blocks) == 2
    env = {}
    torch.manual_seed(0)
    exec(compile(blocks[1], "README.md", "exec"), env)
    torch.cuda.synchronize()
    x, stream = d(env["x"]), d(env["stream0"])
    # the layers read the copy of the parameters as they were before the step
    o, was = env["offsets"], d(env["before"].bfloat16())
    g, w, b = was[:o[1]], was[o[1]:o[2]].view(env["hidden"], env["dim"]), was[o[2]:]
    h, y = plain.norm(x, g, stream, 1e-6)
    close(env["stream"], h, rounded(h, torch.bfloat16) * 1.001, "stream")
    z = d(env["y"]) @ w.t() + b
    close(env["out"], plain.act("gelu", z), 2 * rounded(plain.act("gelu", z), torch.bfloat16) + 1e-3, "out")
    assert torch.equal(env["grad"][env["offsets"][1]:env["offsets"][2]].view_as(env["weight"]), env["dw"])
    assert bool((env["params"] != env["before"]).any()) and torch.equal(env["copy"], env["params"].bfloat16())
