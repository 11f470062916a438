"""AdamW over the tensors of a layout, moments in 32 and 8 bits, against the 64-bit definition."""
import math

import numpy as np
import pytest
import torch

import plain_ops as plain
from paper_1704_05021_amd import gd
from plain_ops import E, TYPES, close, d

pytestmark = pytest.mark.gpu

LAYOUTS = {
    "one": [0, 1],
    "block": [0, 256],
    "ragged": [0, 3, 3, 260, 517, 1541, 1542, 4096 + 1542],  # an empty tensor, blocks and chunks that end inside
    "mnist_small": list(np.cumsum([0, 784 * 64, 64, 64 * 48, 48, 480, 10])),
    "many": list(range(0, 2001, 5)),
}
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def draw(seed, n, scale=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, generator=g) * scale).to(dtype).cuda()


def spread_decay(offsets, decay):
    out = torch.empty(offsets[-1], dtype=torch.float64)
    for t, (a, b) in enumerate(zip(offsets, offsets[1:])):
        out[a:b] = decay[t]
    return out


def check_codes(code, unit, want, offsets, top, what):
    """Each block's unit, and each code at most half a step from the root it stands for."""
    code, unit = d(code), d(unit)
    spans = plain.block_spans(offsets)
    assert unit.numel() == len(spans)
    for k, (a, b) in enumerate(spans):
        big = max(float(want[a:b].abs().max()), 2.0 ** -100)
        assert abs(float(unit[k]) * top * top / big - 1) < 1e-6, f"{what}: unit of block {k}"
        root = torch.sqrt(want[a:b].abs() / (big / (top * top)))
        far = (code[a:b].abs() - root).abs()
        least = (code[a:b] == 1) & (root < 0.5)  # a second moment above 0 keeps code 1
        assert float(far[~least].max() if (~least).any() else 0) <= 0.5 + 1e-3, f"{what}: codes of block {k}"
        if top == 255:
            assert bool(((code[a:b] > 0) == (want[a:b] > 0)).all())
        else:
            assert not bool(least.any() and (root[least] < 0.49).any())
            assert bool((code[a:b] * want[a:b] >= 0).all())


def run_steps(offsets, bits, grad_type, copy_type, steps, max_norm=None, grad_scale=1.0, decay=None):
    n = offsets[-1]
    opt = gd.AdamW(offsets, bits=bits, decay=decay)
    state = opt.init_state()
    p = draw(1, n, 0.1)
    factor = spread_decay(offsets, decay or [1.0] * (len(offsets) - 1))
    copy = None if copy_type is None else torch.empty(n, dtype=copy_type, device="cuda")
    for t in range(1, steps + 1):
        g = draw(10 + t, n, 10.0 ** -(t % 3), grad_type)
        P0, G = d(p), d(g) * grad_scale
        M0, V0 = (d(x) for x in ((state.m, state.v) if bits == 32 else opt.decode(state)))
        norm = opt.step(p, g, state, t, max_norm=max_norm, grad_scale=grad_scale, copy=copy, **HYPER)
        ge = E
        if max_norm is not None:
            want = float(G.norm())
            assert abs(float(norm) - want) <= 2 * E * want
            if want > max_norm:
                G, ge = G * (max_norm / want), 3 * E
        else:
            assert norm is None
        P, M, V, U = plain.adamw(P0, G, M0, V0, t, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], factor)
        b1, b2 = HYPER["betas"]
        m_off = 3 * E * ((b1 * M0).abs() + ((1 - b1) * G).abs()) + ge * ((1 - b1) * G).abs()
        v_off = 4 * E * (b2 * V0 + (1 - b2) * G * G) + 2 * ge * (1 - b2) * G * G
        if bits == 32:
            close(state.m, M, m_off + 2.0 ** -149, "m")
            close(state.v, V, v_off + 2.0 ** -149, "v")
        else:
            check_codes(state.m, state.m_unit, M, offsets, 127.0, "m")
            check_codes(state.v, state.v_unit, V.sqrt(), offsets, 255.0, "v")
        # the update's relative error: the moments', a root, and five operations; then the parameter's three
        slack = (m_off / M.abs().clamp_min(1e-300)) + v_off / V.clamp_min(1e-300) + 8 * E
        close(p, P, 4 * E * P0.abs() + 2 * E * P.abs() + torch.nan_to_num(slack * U.abs()) + 1e-30, "params")
        if copy is not None:
            assert torch.equal(copy, p.to(copy_type))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_steps_over_layouts(layout, bits):
    run_steps(LAYOUTS[layout], bits, torch.float32, None, 3)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("copy", ["bf16", "f16"])
def test_types_clip_scale_and_decay(bits, grad, copy):
    off = LAYOUTS["ragged"]
    decay = [0.0, 1.0, 0.5, 1.0, 0.0, 2.0, 1.0]
    run_steps(off, bits, TYPES[grad], TYPES[copy], 2, max_norm=0.7, grad_scale=0.25, decay=decay)
    run_steps(off, bits, TYPES[grad], TYPES[copy], 1, max_norm=math.inf)


def test_8bit_state_follows_32bit_training():
    """On a quadratic, both kinds of state bring the parameters to the same place."""
    off = [0, 1000, 1700]
    target = draw(5, 1700)
    ends = []
    for bits in (32, 8):
        opt, p = gd.AdamW(off, bits=bits), torch.zeros(1700, device="cuda")
        state = opt.init_state()
        for t in range(1, 301):
            opt.step(p, p - target, state, t, lr=0.03, weight_decay=0.0)
        ends.append(float((p - target).abs().max()))
    assert ends[0] < 0.05 and ends[1] < 0.05, ends


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_skips_the_step(bits, bad):
    off = LAYOUTS["ragged"]
    n = off[-1]
    opt = gd.AdamW(off, bits=bits)
    state, p, copy = opt.init_state(), draw(1, n), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    opt.step(p, draw(2, n), state, 1, lr=1e-3)
    kept = [t.clone() for t in (p, state.m, state.v, copy)]
    g = draw(3, n)
    g[777] = bad
    norm = opt.step(p, g, state, 2, lr=1e-3, max_norm=1.0, copy=copy)
    assert not math.isfinite(float(norm))
    for a, b in zip(kept, (p, state.m, state.v, copy)):
        assert torch.equal(a, b)
    # without a norm the value goes where the formula takes it, and no further than its block
    opt.step(p, g, state, 2, lr=1e-3)
    m = opt.decode(state)[0] if bits == 8 else state.m
    assert not bool(m[777].isfinite()) and bool(m[:517].isfinite().all()) and bool(m[1541:].isfinite().all())
    assert bool(p[:777].isfinite().all())


def test_zero_and_tiny_gradients():
    """All-zero state stays zero under zero gradients; magnitudes near the type's lowest keep their order."""
    for bits in (32, 8):
        opt, p = gd.AdamW([0, 700], bits=bits), draw(1, 700)
        state, kept = opt.init_state(), p.clone()
        opt.step(p, torch.zeros(700, device="cuda"), state, 1, lr=1e-2, weight_decay=0.0)
        assert torch.equal(p, kept) and float(state.m.float().abs().sum() + state.v.float().abs().sum()) == 0
        g = torch.full((700,), 1e-18, device="cuda")
        opt.step(p, g, state, 2, lr=1e-2, weight_decay=0.0)
        assert bool(p.isfinite().all())


def test_tensors_do_not_share_blocks():
    """A tensor's 8-bit moments are those it has alone, whatever lies beside it."""
    g = torch.cat([draw(1, 300, 1e3), draw(2, 10, 1e-4), draw(3, 500, 1e3)])
    p = draw(4, 810)
    opt, alone = gd.AdamW([0, 300, 310, 810], bits=8), gd.AdamW([0, 10], bits=8)
    s, a, q = opt.init_state(), alone.init_state(), p[300:310].clone()
    opt.step(p, g, s, 1, lr=1e-2)
    alone.step(q, g[300:310].contiguous(), a, 1, lr=1e-2)
    assert torch.equal(s.m[300:310], a.m) and torch.equal(s.v[300:310], a.v) and torch.equal(p[300:310], q)
    assert float(s.m_unit[2]) == float(a.m_unit[0])


def test_streams_graphs_and_repeats():
    off = LAYOUTS["mnist_small"]
    n = off[-1]
    results = []
    for way in range(3):
        opt, p = gd.AdamW(off, bits=8), draw(1, n)
        state, g = opt.init_state(), draw(2, n)
        call = lambda **k: opt.step(p, g, state, 5, lr=1e-3, max_norm=1.0, **k)  # noqa: E731
        if way == 2:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
        for _ in range(3):
            if way == 0:
                call()
            elif way == 1:
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                call(stream=side)
                torch.cuda.current_stream().wait_stream(side)
            else:
                graph.replay()
                draw(3, 1000).sum().item()
        results.append([t.clone() for t in (p, state.m, state.v, state.m_unit, state.v_unit)])
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


def test_empty_layout_and_refusals():
    opt = gd.AdamW([0, 0, 0])
    nothing = torch.empty(0, device="cuda")
    assert float(opt.step(nothing, nothing, opt.init_state(), 1, lr=1e-3, max_norm=1.0)) == 0
    for off in ([1, 5], [0, 5, 3], [0, 2 ** 41]):
        with pytest.raises(gd.GDError):
            gd.AdamW(off)
    for decay in ([-1.0], [math.nan], [math.inf]):
        with pytest.raises(gd.GDError):
            gd.AdamW([0, 4], decay=decay)
    with pytest.raises(ValueError):
        gd.AdamW([0, 4], decay=[1.0, 1.0])
    with pytest.raises(ValueError):
        gd.AdamW([0, 4], bits=16)
    opt = gd.AdamW([0, 64])
    p, g, s = draw(1, 64), draw(2, 64), opt.init_state()
    kept = p.clone()
    for k in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=1e-3, betas=(1.0, 0.9)), dict(lr=1e-3, betas=(0.9, -0.1)),
              dict(lr=1e-3, eps=0.0), dict(lr=1e-3, weight_decay=-1.0), dict(lr=1e-3, grad_scale=math.inf)):
        with pytest.raises(gd.GDError):
            opt.step(p, g, s, 1, **k)
    for step in (0, -1):
        with pytest.raises(ValueError):
            opt.step(p, g, s, step, lr=1e-3)
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError):
            opt.step(p, g, s, 1, lr=1e-3, max_norm=bad)
    with pytest.raises(TypeError):
        opt.step(p, g.double(), s, 1, lr=1e-3)
    with pytest.raises(TypeError):
        opt.step(p, g, gd.AdamW([0, 64], bits=8).init_state(), 1, lr=1e-3)
    with pytest.raises(TypeError):
        opt.step(p, g, s, 1, lr=1e-3, copy=torch.empty(64, device="cuda"))
    with pytest.raises(ValueError):
        opt.step(p[:63], g, s, 1, lr=1e-3)
    with pytest.raises(ValueError):
        opt.decode(s)
    assert torch.equal(p, kept)
