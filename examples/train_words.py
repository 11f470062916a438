"""Workers train a small language model whose gradients are dropped, a server takes AdamW steps, a decoder serves it.

Tokens go through an embedding, residual blocks of layer norm, gated layer and product, a last norm and the output layer
over the vocabulary.  The loss is that of the next token and the distance to a teacher's top logits, each with its gradient
in one call; every weight's gradient is written where a flat gradient has it, the embedding's by sorted tokens.  Two
workers (in turn, on one GPU) compress that gradient and push it, the server sums the pushes and takes one AdamW step.  At
the end a decoder takes single tokens through the network with 8-bit weights and reads the likeliest next ones.

    python examples/train_words.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1704_05021_amd import gd  # noqa: E402

VOCAB, DIM, HIDDEN, BLOCKS, ROWS, TOP, WORKERS, HEAT = 2000, 128, 256, 2, 512, 16, 2, 0.5


class Net:
    """The model's plans, and where its tensors lie in a flat buffer; plans hold no weights."""

    def __init__(self, dtype=torch.bfloat16, rows=ROWS):
        shapes = [(VOCAB, DIM)]
        for _ in range(BLOCKS):  # norm and its bias, both projections, down and its bias
            shapes += [(DIM,), (DIM,), (2 * HIDDEN, DIM), (DIM, HIDDEN), (DIM,)]
        self.shapes = shapes + [(DIM,), (DIM,), (VOCAB, DIM)]
        self.offsets = [0]
        for s in self.shapes:
            self.offsets.append(self.offsets[-1] + torch.Size(s).numel())
        self.embed = gd.Embedding(VOCAB, DIM, dtype, scale=DIM ** 0.5, max_rows=rows)
        self.norm = gd.LayerNorm(DIM, dtype)
        self.gated = gd.GatedLinear(DIM, HIDDEN, dtype, act="silu", max_rows=rows)
        self.down = gd.Linear(HIDDEN, DIM, dtype, max_rows=rows)
        self.head = gd.Linear(DIM, VOCAB, dtype, max_rows=rows)
        self.score = gd.TokenLogProbs(VOCAB, dtype, max_rows=rows)
        self.distill = gd.Distill(VOCAB, dtype, scale=HEAT, max_rows=rows)

    def views(self, flat):
        """The tensors of a flat buffer: the embedding, the blocks', the last ones."""
        v = [flat[a:b].view(s) for a, b, s in zip(self.offsets, self.offsets[1:], self.shapes)]
        return v[0], [v[1 + 5 * i:6 + 5 * i] for i in range(BLOCKS)], v[-3:]

    def forward(self, tokens, weights):
        table, blocks, (g, b, head) = weights
        x, stream, kept = self.embed.forward(tokens, table), None, []
        for g1, b1, up, down, bias in blocks:
            y, stream = self.norm.forward(x, g1, b1, stream)
            a, pre = self.gated.forward(y, up, keep_pre=True)
            kept.append((y, stream, a, pre))
            x = self.down.forward(a, down, bias)
        y, stream = self.norm.forward(x, g, b, stream)
        return self.head.forward(y, head), kept + [(y, stream)]

    def losses(self, logits, target, ids, teacher):
        """(sum of both losses, its gradient): means over the tokens that are not padding."""
        count = (target >= 0).sum()
        share = (1.0 / count).expand(len(target)).float()
        scores, d = self.score.forward_backward(logits, target, -share)
        named = torch.where((target >= 0)[:, None], ids, -1)  # padding names nothing
        loss, d2 = self.distill.forward_backward(logits, named, teacher, share.contiguous())
        return ((loss - scores.logp) / count).sum(), d + d2

    def backward(self, tokens, dlogits, kept, weights, grads):
        _, blocks, (g, _, head) = weights
        dtable, dblocks, (dg, db, dhead) = grads
        y, stream = kept[-1]
        dy, *_ = self.head.backward(dlogits, y, head, dweight=dhead)
        d, *_ = self.norm.backward(dy, stream, g, dweight=dg, dbias=db)
        for (y, stream, a, pre), (g1, _, up, down, _), (dg1, db1, dup, ddown, dbias) in reversed(
                list(zip(kept[:-1], blocks, dblocks))):
            da, *_ = self.down.backward(d, a, down, dweight=ddown, dbias=dbias)
            dy, *_ = self.gated.backward(da, y, up, pre, dweight=dup)
            d, *_ = self.norm.backward(dy, stream, g1, dsum=d, dweight=dg1, dbias=db1)
        self.embed.backward(d, tokens, dweight=dtable)

    def serve(self, tokens, weights, quantised, top):
        """The likeliest next tokens of a few, with 8-bit products in the blocks."""
        table, blocks, (g, b, head) = weights
        x, stream = self.embed.forward(tokens, table), None
        for (g1, b1, _, _, bias), (up, us, down, ds) in zip(blocks, quantised):
            q, scale, stream = self.norm.forward_int8(x, g1, b1, stream)
            q, scale = gd.quantise_rows(self.gated.forward_int8(q, scale, up, us))
            x = self.down.forward_int8(q, scale, down, ds, bias)
        y, _ = self.norm.forward(x, g, b, stream)
        return self.score.forward(self.head.forward(y, head), tokens, top=top)


def initial(net):
    """Parameters in float32: gains of 1, biases of 0, weights that keep their inputs' size."""
    params = torch.zeros(net.offsets[-1], device="cuda")
    table, blocks, (g, _, head) = net.views(params)
    table.normal_(0, DIM ** -0.5)
    for w in [head] + [w for block in blocks for w in block[2:4]]:
        w.normal_(0, w.shape[1] ** -0.5)
    for gain in [g] + [block[0] for block in blocks]:
        gain.fill_(1.0)
    return params


def words(rows):
    """Tokens as text has them: the v-th word about as often as 1 / v."""
    u = torch.rand(rows, device="cuda").double()
    return torch.exp(u * torch.log(torch.tensor(VOCAB + 1.0, device="cuda"))).long().sub_(1).clamp_(0, VOCAB - 1)


def main(steps=100, drop=0.95, report=print):
    torch.manual_seed(0)
    net = Net()
    n = net.offsets[-1]
    params = initial(net)
    copy = params.bfloat16()
    weights = net.views(copy)
    opt = gd.AdamW(net.offsets, bits=8, decay=[float(len(s) == 2) for s in net.shapes])
    state = opt.init_state()
    comp = [gd.Compressor(net.offsets) for _ in range(WORKERS)]
    residual = [torch.zeros(n, device="cuda") for _ in range(WORKERS)]
    grad = torch.empty(n, device="cuda")
    grads = net.views(grad)

    follows = torch.randperm(VOCAB, device="cuda")            # the word that follows each
    table = torch.randn(VOCAB, VOCAB, device="cuda")          # what the teacher thinks of the others
    table[torch.arange(VOCAB, device="cuda"), follows] += 8.0
    teacher, ids = table.topk(TOP, dim=1)
    teacher = teacher.bfloat16()
    losses = []
    for step in range(1, steps + 1):
        pushes, loss = [], 0.0
        for w in range(WORKERS):
            tokens = words(ROWS)
            target = follows[tokens]
            target[-ROWS // 16:] = -1  # the batch's padding
            logits, kept = net.forward(tokens, weights)
            value, dlogits = net.losses(logits, target, ids[tokens], teacher[tokens])
            loss = loss + value / WORKERS
            net.backward(tokens, dlogits, kept, weights, grads)
            out = comp[w].compress(grad, residual[w], drop, per_tensor=True)
            pushes.append((out.idx[:out.k], out.val[:out.k]))
        total = torch.zeros(n, device="cuda")
        gd.apply_sparse(total, [i for i, _ in pushes], [v for _, v in pushes], lr=-1.0 / WORKERS)  # the pushes' mean
        opt.step(params, total, state, step, lr=3e-3, weight_decay=0.01, max_norm=1.0, copy=copy)
        losses.append(loss)
    losses = [float(v) for v in losses]
    report(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} after {steps} steps")

    quantised = [(*gd.quantise_rows(up), *gd.quantise_rows(down)) for _, _, up, down, _ in weights[1]]
    tokens = words(64)
    best = [net.serve(tokens[i:i + 1], weights, quantised, top=5) for i in range(64)]
    found = sum(int(follows[t] in s.top_ids) for t, s in zip(tokens, best))
    report(f"the next word is among the five that the decoder names for {found} of 64 words")
    return losses, best


if __name__ == "__main__":
    main()
