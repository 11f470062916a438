"""What 8-bit moments stand for: every code of both, decoded and as a step reads them, against the stated values."""
import numpy as np
import pytest
import torch

import plain_ops as plain
from paper_1704_05021_amd import gd
from plain_ops import E, close, d

pytestmark = pytest.mark.gpu

# blocks that end inside, an empty tensor, one that starts off a 16-byte boundary, chunks of 4,096 with and without a rest
LAYOUTS = {"block": [0, 256], "ragged": [0, 3, 3, 260, 517, 1541, 5640], "long": [0, 4096, 4096 + 9001]}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def state_of_codes(offsets, seed):
    """A state of arbitrary codes and units, and each element's block."""
    rng = np.random.default_rng(seed)
    n, spans = offsets[-1], plain.block_spans(offsets)
    m, v = rng.integers(-127, 128, n), rng.integers(0, 256, n)
    m[:min(n, 255)], v[:min(n, 256)] = np.arange(-127, 128)[:n], np.arange(256)[:n]  # all of them
    units = [torch.tensor(10.0 ** rng.uniform(-14, 1, len(spans)), dtype=torch.float32) for _ in range(2)]
    block = torch.cat([torch.full((b - a,), i) for i, (a, b) in enumerate(spans)])
    return torch.tensor(m), torch.tensor(v), *units, block


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_decode(layout):
    """unit * q * |q| and (unit * q^2)^2, each operation rounded to binary32 (q * |q| and q^2 are exact)."""
    off = LAYOUTS[layout]
    m, v, mu, vu, block = state_of_codes(off, 1)
    opt = gd.AdamW(off, bits=8)
    state = gd.AdamWState(m.to(torch.int8).cuda(), v.to(torch.uint8).cuda(), mu.cuda(), vu.cuda())
    assert opt.blocks == len(mu)
    mo, vo = opt.decode(state)
    root = vu[block] * (v * v).float()
    assert torch.equal(mo.cpu(), mu[block] * (m * m.abs()).float()) and torch.equal(vo.cpu(), root * root)


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_a_step_reads_the_same_values(layout):
    off, lr, betas, eps, step = LAYOUTS[layout], 1e-2, (0.9, 0.99), 1e-8, 7
    m, v, mu, vu, block = state_of_codes(off, 2)
    n = off[-1]
    M0 = d(mu)[block] * d(m) * d(m).abs()
    V0 = (d(vu)[block] * d(v) ** 2) ** 2
    g = torch.tensor(np.random.default_rng(3).standard_normal(n) * 1e-3, dtype=torch.float32)
    p = torch.tensor(np.random.default_rng(4).standard_normal(n), dtype=torch.float32)
    opt, q = gd.AdamW(off, bits=8), p.cuda()
    state = gd.AdamWState(m.to(torch.int8).cuda(), v.to(torch.uint8).cuda(), mu.cuda(), vu.cuda())
    opt.step(q, g.cuda(), state, step, lr=lr, betas=betas, eps=eps, weight_decay=0.0)
    P, M, V, U = plain.adamw(d(p), d(g), M0, V0, step, lr, betas, eps, 0.0, torch.ones(n, dtype=torch.float64))
    b1, b2 = betas
    # decoding rounds m once and v three times (its root once, squared, then the square); the rest as for 32-bit moments
    m_off = 4 * E * (b1 * M0).abs() + 4 * E * ((1 - b1) * d(g)).abs()
    v_off = 7 * E * (b2 * V0) + 6 * E * (1 - b2) * d(g) ** 2
    slack = m_off / M.abs().clamp_min(1e-300) + v_off / V.clamp_min(1e-300) + 8 * E
    close(q, P, 4 * E * d(p).abs() + 2 * E * P.abs() + torch.nan_to_num(slack * U.abs()), "params")
