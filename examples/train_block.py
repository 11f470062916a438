"""Workers train a small pre-norm network whose gradients are dropped, a server takes AdamW steps, a decoder serves it.

Two workers (in turn, on one GPU) run residual blocks forward and backward; every weight's gradient is written where a
flat gradient has it.  Each worker compresses that gradient to 5% of its entries and pushes them; the server sums the
pushes, takes one AdamW step with 8-bit moments, clipped by the gradient's norm, and hands out the parameters rounded
to bfloat16, which the workers' layers read in place.  At the end single tokens go through the same network with 8-bit
weights and activations.

    python examples/train_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1704_05021_amd import gd  # noqa: E402

DIM, HIDDEN, CLASSES, BLOCKS, ROWS, WORKERS = 256, 512, 16, 2, 512, 2


class Net:
    """Blocks of norm, product with activation, product; the sum that is normalised is the residual stream."""

    def __init__(self):
        shapes = []
        for _ in range(BLOCKS):
            shapes += [(DIM,), (HIDDEN, DIM), (HIDDEN,), (DIM, HIDDEN), (DIM,)]  # norm, up and its bias, down and its bias
        self.shapes = shapes + [(DIM,), (CLASSES, DIM), (CLASSES,)]
        self.offsets = [0]
        for s in self.shapes:
            self.offsets.append(self.offsets[-1] + torch.Size(s).numel())
        # plans hold no weights: one serves every layer of its shape
        self.norm = gd.RMSNorm(DIM)
        self.up = gd.Linear(DIM, HIDDEN, act="silu", max_rows=ROWS)
        self.down = gd.Linear(HIDDEN, DIM, max_rows=ROWS)
        self.head = gd.Linear(DIM, CLASSES, max_rows=ROWS)

    def views(self, flat):
        """The tensors of a flat buffer, by block: [(norm, up, up's bias, down, down's bias), ..., (norm, head, bias)]."""
        v = [flat[a:b].view(s) for a, b, s in zip(self.offsets, self.offsets[1:], self.shapes)]
        return [v[5 * i:5 * i + 5] for i in range(BLOCKS)] + [v[5 * BLOCKS:]]

    def forward(self, x, weights):
        kept, stream = [], None
        for g, w1, b1, w2, b2 in weights[:-1]:
            y, stream = self.norm.forward(x, g, stream)
            a, pre = self.up.forward(y, w1, b1, keep_pre=True)
            kept.append((y, stream, a, pre))
            x = self.down.forward(a, w2, b2)
        g, w, b = weights[-1]
        y, stream = self.norm.forward(x, g, stream)
        return self.head.forward(y, w, b), kept + [(y, stream)]

    def backward(self, dlogits, kept, weights, grads):
        y, stream = kept[-1]
        g, w, _ = weights[-1]
        dg, dw, db = grads[-1]
        dy, *_ = self.head.backward(dlogits, y, w, dweight=dw, dbias=db)
        d, _ = self.norm.backward(dy, stream, g, dweight=dg)
        for (y, stream, a, pre), (g, w1, _, w2, _), (dg, dw1, db1, dw2, db2) in reversed(
                list(zip(kept[:-1], weights[:-1], grads[:-1]))):
            da, *_ = self.down.backward(d, a, w2, dweight=dw2, dbias=db2)
            dy, *_ = self.up.backward(da, y, w1, pre, dweight=dw1, dbias=db1)
            d, _ = self.norm.backward(dy, stream, g, dsum=d, dweight=dg)

    def serve(self, x, weights, quantised):
        """Logits of a few tokens with 8-bit products in the blocks."""
        stream = None
        for (g, _, b1, _, b2), (w1, s1, w2, s2) in zip(weights[:-1], quantised):
            q, scale, stream = self.norm.forward_int8(x, g, stream)
            q, scale = gd.quantise_rows(self.up.forward_int8(q, scale, w1, s1, b1))
            x = self.down.forward_int8(q, scale, w2, s2, b2)
        g, w, b = weights[-1]
        y, _ = self.norm.forward(x, g, stream)
        return self.head.forward(y, w, b)


def main(steps=150, drop=0.95, report=print):
    torch.manual_seed(0)
    net = Net()
    n = net.offsets[-1]
    # the server's: parameters, moments, the working copy the layers read
    params = torch.zeros(n, device="cuda")
    for s, v in zip(net.shapes, [params[a:b] for a, b in zip(net.offsets, net.offsets[1:])]):
        if len(s) == 2:
            v.normal_(0, s[1] ** -0.5)
    for block in net.views(params):
        block[0].fill_(1.0)
    copy = params.bfloat16()
    weights = net.views(copy)
    opt = gd.AdamW(net.offsets, bits=8, decay=[float(len(s) == 2) for s in net.shapes])
    state = opt.init_state()
    # a worker's: the flat gradient, what was not sent yet, the compressor's scratch
    comp = [gd.Compressor(net.offsets) for _ in range(WORKERS)]
    residual = [torch.zeros(n, device="cuda") for _ in range(WORKERS)]
    grad = torch.empty(n, device="cuda")
    grads = net.views(grad)

    teacher = torch.randn(DIM, CLASSES, device="cuda")
    draw = lambda rows: torch.randn(rows, DIM, device="cuda")  # noqa: E731
    losses = []
    for step in range(1, steps + 1):
        pushes, loss = [], 0.0
        for w in range(WORKERS):
            x = draw(ROWS)
            target = (x @ teacher).argmax(1)
            logits, kept = net.forward(x.bfloat16(), weights)
            p = torch.log_softmax(logits.float(), 1)
            loss = loss - p[torch.arange(ROWS, device="cuda"), target].mean() / WORKERS
            dlogits = p.exp()
            dlogits[torch.arange(ROWS, device="cuda"), target] -= 1.0
            net.backward((dlogits / ROWS).bfloat16(), kept, weights, grads)
            out = comp[w].compress(grad, residual[w], drop, per_tensor=True)
            pushes.append((out.idx[:out.k], out.val[:out.k]))
        total = torch.zeros(n, device="cuda")
        gd.apply_sparse(total, [i for i, _ in pushes], [v for _, v in pushes], lr=-1.0 / WORKERS)  # the pushes' mean
        opt.step(params, total, state, step, lr=2e-3, weight_decay=0.01, max_norm=1.0, copy=copy)
        losses.append(loss)
    losses = [float(v) for v in losses]
    report(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} after {steps} steps, {sum(i.numel() for i, _ in pushes)} of "
           f"{WORKERS * n} gradient entries sent a step")

    quantised = [(*gd.quantise_rows(w1), *gd.quantise_rows(w2)) for _, w1, _, w2, _ in weights[:-1]]
    x = draw(ROWS).bfloat16()
    full, _ = net.forward(x, weights)
    tokens = torch.cat([net.serve(x[i:i + 1], weights, quantised) for i in range(64)])
    agree = float((tokens.argmax(1) == full[:64].argmax(1)).float().mean())
    report(f"single tokens in 8 bits choose the same class as the batch in bfloat16: {100 * agree:.0f}%")
    return losses, agree


if __name__ == "__main__":
    main()
