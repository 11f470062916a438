"""The operators of a language model together: the example runs as it stands, and its flat gradient, written tensor by
tensor by the operators' backward passes, is that of the same network in 64 bits by autograd."""
import importlib.util
import math
import os

import pytest
import torch

from plain_ops import E, d

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def words():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("train_words", os.path.join(ROOT, "examples", "train_words.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_the_example_runs(words):
    losses, best = words.main(steps=6, report=lambda *_: None)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses)
    assert all(s.top_ids.shape == (1, 5) and bool((s.top_logp <= 0).all()) for s in best)


def reference(words, net, params, tokens, target, ids, teacher):
    """(loss, flat gradient) in 64 bits by autograd, from elementary operations."""
    flat = d(params).requires_grad_()
    table, blocks, (g, b, head) = net.views(flat)
    count = (target >= 0).sum()

    def norm(h, g, b):
        c = h - h.mean(1, keepdim=True)
        return c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * g + b

    stream, x = 0.0, table[tokens] * words.DIM ** 0.5
    for g1, b1, up, down, bias in blocks:
        stream = stream + x
        z = norm(stream, g1, b1) @ up.t()
        gate, u = z.chunk(2, 1)
        x = (gate / (1 + torch.exp(-gate)) * u) @ down.t() + bias
    logits = norm(stream + x, g, b) @ head.t()
    seen = target >= 0
    lp = logits - torch.logsumexp(logits, 1, keepdim=True)
    loss = -lp[seen].gather(1, target[seen][:, None]).sum()
    w = torch.softmax(teacher * words.HEAT, 1)
    lq = logits * words.HEAT
    lq = lq - torch.logsumexp(lq, 1, keepdim=True)
    loss = loss + (w * (torch.log(w) - lq.gather(1, ids)))[seen].sum()
    loss = loss / count
    loss.backward()
    return loss.detach(), flat.grad


def test_the_flat_gradient(words):
    torch.manual_seed(1)
    rows = 96
    net = words.Net(torch.float32, rows)
    params = words.initial(net) + 0.1 * torch.randn(net.offsets[-1], device="cuda") * words.DIM ** -0.5
    tokens, target = words.words(rows), words.words(rows)
    target[-7:] = -1
    ids = torch.rand(rows, words.VOCAB, device="cuda").topk(words.TOP, dim=1).indices
    teacher = torch.randn(rows, words.TOP, device="cuda") * 2
    weights, grad = net.views(params), torch.full_like(params, math.nan)
    logits, kept = net.forward(tokens, weights)
    loss, dlogits = net.losses(logits, target, ids, teacher)
    net.backward(tokens, dlogits, kept, weights, net.views(grad))
    want, flat = reference(words, net, params, tokens.cpu(), target.cpu(), ids.cpu(), d(teacher))
    assert abs(float(loss) - float(want)) < 200 * E * float(want)  # sums of some hundred roundings, each relative to less
    # tensor by tensor: errors of some 30 operations in a row, each of a few roundings, times a margin of ten
    for a, b, shape in zip(net.offsets, net.offsets[1:], net.shapes):
        got, right = d(grad)[a:b], flat[a:b]
        assert bool(got.isfinite().all()) and float((got - right).norm()) < 1000 * E * float(right.norm()), shape
    seen = torch.zeros(words.VOCAB, dtype=torch.bool)
    seen[tokens.cpu()] = True
    assert not bool(d(net.views(grad)[0])[~seen].any())


def test_the_step_in_a_graph(words):
    """Forward, losses and backward captured once and replayed on other batches give what the calls themselves give."""
    torch.manual_seed(2)
    net = words.Net()
    copy = words.initial(net).bfloat16()
    weights = net.views(copy)
    teacher = torch.randn(words.ROWS, words.TOP, device="cuda").bfloat16()
    ids = torch.rand(words.ROWS, words.VOCAB, device="cuda").topk(words.TOP, dim=1).indices
    tokens, target = words.words(words.ROWS), words.words(words.ROWS)
    share = torch.full((words.ROWS,), 1.0 / words.ROWS, device="cuda")

    def step(grad):
        logits, kept = net.forward(tokens, weights)
        scores, dl = net.score.forward_backward(logits, target, -share)
        loss, d2 = net.distill.forward_backward(logits, ids, teacher, share)
        net.backward(tokens, dl + d2, kept, weights, net.views(grad))
        return scores.logp, loss

    grads = [torch.empty(net.offsets[-1], device="cuda") for _ in range(2)]
    step(grads[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(grads[1])
    for _ in range(3):
        tokens.copy_(words.words(words.ROWS))
        target.copy_(words.words(words.ROWS))
        graph.replay()
        torch.cuda.synchronize()
        logp, loss = step(grads[0])
        torch.cuda.synchronize()
        assert torch.equal(grads[0], grads[1]) and torch.equal(logp, held[0]) and torch.equal(loss, held[1])


def test_readme_language_model():
    """The README's example runs, and its table's gradient is that of its loss in 64 bits, at bfloat16's precision."""
    import re

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    blocks = re.findall(r"```py\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), re.S)
    assert len(blocks) == 1
    env = {}
    torch.manual_seed(0)
    exec(compile(blocks[0], "README.md", "exec"), env)
    torch.cuda.synchronize()
    table, up, down, head = (d(env[k]).requires_grad_() for k in ("table", "up", "down", "head"))
    tokens, following = env["tokens"].cpu(), env["following"].cpu()
    h0 = table[tokens] * env["width"] ** 0.5
    c = h0 - h0.mean(1, keepdim=True)
    z = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) @ up.t()
    gate, u = z.chunk(2, 1)
    logits = (gate / (1 + torch.exp(-gate)) * u @ down.t() + h0) @ head.t()
    lp = torch.log_softmax(logits, 1)
    seen = following >= 0
    loss = -lp[seen].gather(1, following[seen][:, None]).sum() / 290
    loss.backward()
    # each of some ten results along the way is rounded to bfloat16, half a step of 2^-8, at random: together within 2^-5
    assert abs(float(env["loss"]) - float(loss.detach())) < 2.0 ** -8 * float(loss.detach())
    for k, want in (("dtable", table), ("dup", up), ("ddown", down), ("dhead", head)):
        assert float((d(env[k]) - want.grad).norm()) < 2.0 ** -5 * float(want.grad.norm()), k
    assert env["best"].top_ids.shape == (1, 5) and bool(env["apart"].isfinite().all())
