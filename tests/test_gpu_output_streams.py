"""Outputs that a call on a given stream allocates: their memory is in no other stream's hands, before the call or after."""
import pytest
import torch

from paper_1704_05021_amd import gd

pytestmark = pytest.mark.gpu

ROWS, K, N = 512, 768, 1024


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gd.load()
    torch.cuda.set_device(0)


def flat(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


def calls():
    g = torch.Generator().manual_seed(1)
    draw = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    x, r, dy, w, gain = draw(ROWS, K), draw(ROWS, K), draw(ROWS, N), draw(N, K), draw(K)
    norm, layer = gd.RMSNorm(K), gd.Linear(K, N, act="silu", max_rows=ROWS)
    _, pre = layer.forward(x, w, keep_pre=True)
    q, s = gd.quantise_rows(x)
    wq, ws = gd.quantise_rows(w)
    opt = gd.AdamW([0, K * N], bits=8)
    state, flat_p = opt.init_state(), draw(K * N).float()
    opt.step(flat_p, flat_p, state, 1, lr=1e-3)
    keep = (norm, layer, opt)
    return {
        "norm": lambda **a: norm.forward(x, gain, r, **a),
        "norm_int8": lambda **a: norm.forward_int8(x, gain, r, **a),
        "norm_back": lambda **a: norm.backward(x, r, gain, **a),
        "linear": lambda **a: layer.forward(x, w, keep_pre=True, **a),
        "linear_int8": lambda **a: layer.forward_int8(q, s, wq, ws, **a),
        "linear_back": lambda **a: layer.backward(dy, x, w, pre, dbias=True, **a),
        "quantise": lambda **a: gd.quantise_rows(x, **a),
        "decode": lambda **a: opt.decode(state, **a),
    }, keep


@pytest.mark.parametrize("name", ["norm", "norm_int8", "norm_back", "linear", "linear_int8", "linear_back", "quantise", "decode"])
def test_memory_of_outputs(name):
    ways, _ = calls()
    call = ways[name]
    want = [t.clone() for t in flat(call())]
    a = torch.randn(4096, 4096, device="cuda")
    busy = lambda: [torch.mm(a, a, out=b) for _ in range(20)]  # noqa: E731  (milliseconds)
    b = torch.empty_like(a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())

    # memory that was given back, but that queued work of the current stream still writes
    busy()
    freed = [torch.empty_like(t) for t in want]
    for t in freed:
        t.fill_(3)
    places = {t.data_ptr() for t in freed}
    del freed, t
    got = call(stream=side)
    assert not places & {t.data_ptr() for t in flat(got)}
    torch.cuda.synchronize()
    for x, y in zip(flat(got), want):
        assert torch.equal(x, y)

    # outputs that the current stream's queued work reads are not given to the next call before that is done
    torch.cuda.current_stream().wait_stream(side)
    busy()
    copies = [t.clone() for t in flat(got)]
    places = {t.data_ptr() for t in flat(got)}
    del got
    again = call(stream=side)
    assert not places & {t.data_ptr() for t in flat(again)}
    torch.cuda.synchronize()
    for x, y, z in zip(copies, want, flat(again)):
        assert torch.equal(x, y) and torch.equal(z, y)
