"""More operators around the compressor whose speed is tracked: the two ends of a language model and two parts of its blocks.

Below the layers a worker looks up embeddings (``gd.Embedding``) whose gradient goes into the flat gradient by sorted
tokens; its blocks have layer norms (``gd.LayerNorm``) and gated layers (``gd.GatedLinear``); above them stand the log
probabilities of given tokens (``gd.TokenLogProbs``, a training loss with its gradient, and a decoder's scores with the
top alternatives) and the loss against a teacher's top logits (``gd.Distill``).  Each case is one call as such a program
makes it; the plain form of each is elementary torch operations in 32 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS_NORM = 1e-5


def listed():
    return [
        # embedding: the tokens of a training batch, scaled by the root of the width
        {"name": "embed_batch", "do": "embed", "rows": 8192, "vocab": 32_000, "dim": 4096, "type": "bf16", "scale": 64.0},
        # its gradient for the NMT model's words and the tokens of a step: most rows of the flat gradient are zeros
        {"name": "embed_nmt_back", "do": "embed_back", "rows": 3000, "vocab": 85_000, "dim": 500, "type": "f32", "scale": 1.0},
        # layer norm: one token of a decoder of the NMT model's hidden width, the residual added, 8-bit output
        {"name": "layer_norm_token", "do": "norm", "rows": 1, "dim": 1024, "type": "bf16", "residual": True, "int8": True},
        # a training batch forward: the residual stream is added and kept
        {"name": "layer_norm_batch", "do": "norm", "rows": 8192, "dim": 4096, "type": "bf16", "residual": True, "int8": False},
        # the same backward, with the gradient that comes down the residual stream
        {"name": "layer_norm_batch_back", "do": "norm_back", "rows": 8192, "dim": 4096, "type": "bf16", "residual": True},
        # gated layer: one token of a decoder
        {"name": "gated_token", "do": "gated", "rows": 1, "in": 4096, "out": 8192, "type": "bf16", "act": "silu", "bias": False,
         "pre": False},
        # a training batch forward, the activation's inputs kept for the backward
        {"name": "gated_batch", "do": "gated", "rows": 4096, "in": 4096, "out": 8192, "type": "bf16", "act": "silu",
         "bias": False, "pre": True},
        # its backward: gradients of input and weights
        {"name": "gated_batch_back", "do": "gated_back", "rows": 4096, "in": 4096, "out": 8192, "type": "bf16", "act": "silu",
         "bias": False},
        # a decoder's step over the NMT model's words: the chosen token's score, entropy and the 8 best alternatives
        {"name": "logprob_token", "do": "logprob", "rows": 1, "vocab": 85_000, "type": "bf16", "top": 8, "masked": False},
        # the loss of a training step with its gradient, in one call: 3,000 tokens over the NMT model's words
        {"name": "logprob_train", "do": "logprob_train", "rows": 3000, "vocab": 85_000, "type": "bf16", "entropy": False},
        # a small validation batch against a teacher's 16 best logits, forward, in 32 bits
        {"name": "distill_valid", "do": "distill", "rows": 40, "vocab": 32_000, "top": 16, "type": "f32"},
        # a student's training step against 32 of them, loss and gradient in one call
        {"name": "distill_train", "do": "distill_train", "rows": 2000, "vocab": 32_000, "top": 32, "type": "bf16"},
    ]


def draw(rng):
    """One more case of these ranges: any operator and direction, sizes over their logarithm, odd ones among them."""
    def log(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n if rng.random() < 0.5 else max(lo, n - n % 64)

    do = rng.choice(["embed", "embed_back", "norm", "norm_back", "gated", "gated", "gated_back", "gated_int8", "logprob",
                     "logprob_train", "distill", "distill_train"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if do in ("embed", "embed_back"):
        return {"do": do, "rows": log(1, 16_384), "vocab": log(1000, 85_000), "dim": log(64, 1024), "type": kind,
                "scale": rng.choice([1.0, 16.0])}
    if do in ("norm", "norm_back"):
        case = {"do": do, "rows": log(1, 8192), "dim": log(64, 8192 if kind != "f32" else 4096), "type": kind,
                "residual": rng.random() < 0.6}
        return {**case, "int8": rng.random() < 0.4} if do == "norm" else case
    if do in ("gated", "gated_back", "gated_int8"):
        case = {"do": do, "rows": log(1, 4096), "in": log(128, 4096), "out": log(128, 4096), "type": rng.choice(["bf16", "bf16", "f16"]),
                "act": rng.choice(["silu", "silu", "gelu", "relu", "none"]), "bias": rng.random() < 0.4}
        return {**case, "pre": rng.random() < 0.5} if do == "gated" else case
    vocab = log(2000, 128_000)
    rows = min(log(1, 4096), 120_000_000 // vocab)
    case = {"do": do, "rows": rows, "vocab": vocab, "type": kind}
    if do == "logprob":
        return {**case, "rows": min(rows, 512), "top": rng.choice([0, 1, 5, 20, 64]), "masked": rng.random() < 0.4}
    if do == "logprob_train":
        return {**case, "entropy": rng.random() < 0.4}
    return {**case, "top": rng.choice([1, 8, 20, 64, 128])}


# ---- inputs ----


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    def words(vocab, *shape):
        """Token ids as text has them: the v-th word about as often as 1 / v."""
        return torch.exp(uniform(*shape).double() * math.log(vocab + 1)).long().sub_(1).clamp_(0, vocab - 1)

    do, kind, s = case["do"], TYPES[case["type"]], {"case": case}
    if do in ("embed", "embed_back"):
        rows, vocab, dim = case["rows"], case["vocab"], case["dim"]
        s["tokens"] = words(vocab, rows)
        s["tokens"][rows - rows // 32:] = -1  # the batch's padding
        if do == "embed":
            s["weight"] = normal(vocab, dim, scale=0.02, dtype=kind)
        else:
            s["dy"] = normal(rows, dim, scale=1e-3, dtype=kind)
            s["dweight"] = torch.empty(vocab, dim, device="cuda")  # a slice of the flat gradient
    elif do in ("norm", "norm_back"):
        shape = (case["rows"], case["dim"])
        s["x"] = normal(*shape, dtype=kind)
        s["weight"] = (1.0 + normal(case["dim"], scale=0.1)).to(kind)
        s["bias"] = normal(case["dim"], scale=0.1, dtype=kind)
        s["residual"] = (0.5 + normal(*shape, scale=2.0)).to(kind) if case["residual"] else None
        if do == "norm_back":
            s["dy"] = normal(*shape, scale=1e-3 if kind != torch.float16 else 1.0, dtype=kind)
            s["dweight"], s["dbias"] = (torch.empty(case["dim"], device="cuda") for _ in range(2))
    elif do.startswith("gated"):
        rows, k, n = case["rows"], case["in"], case["out"]
        s["x"] = normal(rows, k, dtype=kind)
        s["weight"] = normal(2 * n, k, scale=k ** -0.5, dtype=kind)  # the gate's rows, then those that it multiplies
        s["bias"] = normal(2 * n, scale=0.1, dtype=kind) if case["bias"] else None
        if do == "gated_back":
            s["dy"] = normal(rows, n, scale=1e-3 if kind != torch.float16 else 1.0, dtype=kind)
            s["pre"] = normal(rows, 2 * n, dtype=kind)
            s["dweight"] = torch.empty(2 * n, k, device="cuda")
            s["dbias"] = torch.empty(2 * n, device="cuda") if case["bias"] else None
        if do == "gated_int8":  # the weights of a served model are quantised once
            s["wq"], s["wscale"] = _quantise(s.pop("weight").float())
    else:
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = normal(rows, vocab, scale=2.5, dtype=kind)
        if do in ("logprob", "logprob_train"):
            s["tokens"] = words(vocab, rows)
            if case.get("masked"):  # what a grammar forbids at this step
                s["logits"].masked_fill_(uniform(rows, vocab) < 0.7, -math.inf)
                s["logits"].scatter_(1, s["tokens"][:, None], 1.0)
            if do == "logprob_train":
                s["tokens"][rows - rows // 32:] = -1  # padding: no loss
                s["dlogp"] = torch.full((rows,), -1.0 / rows, device="cuda")
                s["dentropy"] = torch.full((rows,), -0.01 / rows, device="cuda") if case["entropy"] else None
                if kind == torch.float16:  # scaled, as gradients in this type are
                    s["dlogp"] *= 1024.0 * rows
                    s["dentropy"] = None if s["dentropy"] is None else s["dentropy"] * (1024.0 * rows)
        else:  # the teacher's best words, and logits near the student's own
            s["ids"] = torch.rand(rows, vocab, generator=g, device="cuda").topk(case["top"], dim=1).indices
            s["teacher"] = normal(rows, case["top"], scale=1.5).add_(6.0)
            s["scale"] = 0.5  # a temperature of 2
            s["dloss"] = torch.full((rows,), (1.0 if kind != torch.float16 else 1024.0 * rows) / rows, device="cuda")
    if own:
        s["op"] = _handle(case, s)
    return s


def _handle(case, s):
    """What a user's program keeps of the framework: the operator's plan."""
    from paper_1704_05021_amd import gd

    do, kind = case["do"], TYPES[case["type"]]
    if do in ("embed", "embed_back"):
        return gd.Embedding(case["vocab"], case["dim"], kind, scale=case["scale"], max_rows=case["rows"])
    if do in ("norm", "norm_back"):
        return gd.LayerNorm(case["dim"], kind, eps=EPS_NORM)
    if do.startswith("gated"):
        return gd.GatedLinear(case["in"], case["out"], kind, act=case["act"], max_rows=case["rows"])
    if do.startswith("logprob"):
        return gd.TokenLogProbs(case["vocab"], kind, max_rows=case["rows"])
    return gd.Distill(case["vocab"], kind, scale=s["scale"], max_rows=case["rows"])


# ---- one pass ----


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, op, do = s["case"], s["op"], s["case"]["do"]
    if do == "embed":
        return {"y": op.forward(s["tokens"], s["weight"])}
    if do == "embed_back":
        return {"dweight": op.backward(s["dy"], s["tokens"], dweight=s["dweight"])}
    if do == "norm" and case["int8"]:
        q, scale, h = op.forward_int8(s["x"], s["weight"], s["bias"], s["residual"])
        return {"y": q * scale[:, None], "h": h}
    if do == "norm":
        y, h = op.forward(s["x"], s["weight"], s["bias"], s["residual"])
        return {"y": y, "h": h}
    if do == "norm_back":
        dx, dw, db = op.backward(s["dy"], s["x"], s["weight"], dsum=s["residual"], dweight=s["dweight"], dbias=s["dbias"])
        return {"dx": dx, "dweight": dw, "dbias": db}
    if do == "gated":
        if not case["pre"]:
            return {"y": op.forward(s["x"], s["weight"], s["bias"])}
        y, pre = op.forward(s["x"], s["weight"], s["bias"], keep_pre=True)
        return {"y": y, "pre": pre}
    if do == "gated_int8":
        from paper_1704_05021_amd import gd

        q, scale = gd.quantise_rows(s["x"])
        return {"y": op.forward_int8(q, scale, s["wq"], s["wscale"], s["bias"])}
    if do == "gated_back":
        dx, dw, db, dz = op.backward(s["dy"], s["x"], s["weight"], s["pre"], dweight=s["dweight"], dbias=s["dbias"])
        return {"dx": dx, "dweight": dw, "dbias": db, "dz": dz}
    if do == "logprob":
        r = op.forward(s["logits"], s["tokens"], top=case["top"])
        return {"logp": r.logp, "entropy": r.entropy, "top_logp": r.top_logp, "top_ids": r.top_ids}
    if do == "logprob_train":
        r, dlogits = op.forward_backward(s["logits"], s["tokens"], s["dlogp"], s["dentropy"])
        return {"logp": r.logp, "entropy": r.entropy if case["entropy"] else None, "dlogits": dlogits}
    if do == "distill":
        loss, _ = op.forward(s["logits"], s["ids"], s["teacher"])
        return {"loss": loss}
    loss, dlogits = op.forward_backward(s["logits"], s["ids"], s["teacher"], s["dloss"])
    return {"loss": loss, "dlogits": dlogits}


def _run_plain(s):
    case, do = s["case"], s["case"]["do"]
    kind = TYPES[case["type"]]
    if do == "embed":
        t = s["tokens"]
        y = s["weight"][t.clamp_min(0)].float() * case["scale"]
        return {"y": torch.where((t >= 0)[:, None], y, 0.0).to(kind)}
    if do == "embed_back":
        t = s["tokens"]
        d = torch.where((t >= 0)[:, None], s["dy"].float() * case["scale"], 0.0)
        s["dweight"].zero_().index_add_(0, t.clamp_min(0), d)
        return {"dweight": s["dweight"]}
    if do in ("norm", "norm_back"):
        x, w = s["x"].float(), s["weight"].float()
        if do == "norm":
            h = x if s["residual"] is None else x + s["residual"].float()
            c, rstd = _centred(h)
            y = c * rstd * w + s["bias"].float()
            if case["int8"]:
                q, scale = _quantise(y)
                y = q * scale[:, None]
            return {"y": y if case["int8"] else y.to(kind), "h": h.to(kind)}
        c, rstd = _centred(x)
        dy, xhat = s["dy"].float(), c * rstd
        a = dy * w
        dx = rstd * (a - a.mean(1, keepdim=True) - xhat * (a * xhat).mean(1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        s["dweight"].copy_((dy * xhat).sum(0))
        s["dbias"].copy_(dy.sum(0))
        return {"dx": dx.to(kind), "dweight": s["dweight"], "dbias": s["dbias"]}
    if do.startswith("gated"):
        n, x = case["out"], s["x"].float()
        if do == "gated_back":
            dy, g, u = s["dy"].float(), s["pre"][:, :n].float(), s["pre"][:, n:].float()
            dz = torch.cat([dy * u * _slope(case["act"], g), dy * _act(case["act"], g)], 1)
            dz = dz.to(kind)  # the gradient at both products is an output in the type, and what the others are taken with
            d = dz.float()
            torch.mm(d.t(), x, out=s["dweight"])
            if s["dbias"] is not None:
                s["dbias"].copy_(d.sum(0))
            return {"dx": (d @ s["weight"].float()).to(kind), "dweight": s["dweight"], "dbias": s["dbias"], "dz": dz}
        if do == "gated_int8":
            q, scale = _quantise(x)
            z = (q.float() @ s["wq"].float().t()) * (scale[:, None] * s["wscale"][None, :])
        else:
            z = x @ s["weight"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(case["act"], z[:, :n]) * z[:, n:]
        return {"y": y.to(kind), "pre": z.to(kind) if case.get("pre") else None}
    z = s["logits"].float() * s.get("scale", 1.0)
    most = z.amax(1, keepdim=True)
    e = torch.exp(z - most)
    total = e.sum(1, keepdim=True)
    if do in ("logprob", "logprob_train"):
        t = s["tokens"][:, None]
        lp = z - most - torch.log(total)
        logp = torch.where(t >= 0, lp.gather(1, t.clamp_min(0)), 0.0)[:, 0]
        p = e / total
        if do == "logprob" or case["entropy"]:
            entropy = -(p * torch.where(p > 0, lp, 0.0)).sum(1)
        if do == "logprob":
            k = case["top"]
            ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k] if k else None  # ties: the lower id first
            return {"logp": logp, "entropy": entropy, "top_logp": lp.gather(1, ids) if k else None, "top_ids": ids}
        g = torch.where(t >= 0, s["dlogp"][:, None], 0.0)
        d = p * -g
        d.scatter_add_(1, t.clamp_min(0), g)
        if case["entropy"]:
            d = d - s["dentropy"][:, None] * p * (lp + entropy[:, None])
        return {"logp": logp, "entropy": entropy if case["entropy"] else None, "dlogits": d.to(kind)}
    a = s["teacher"].float() * s["scale"]
    a = a - a.amax(1, keepdim=True)
    log_t = a - torch.log(torch.exp(a).sum(1, keepdim=True))
    t = torch.exp(log_t)
    loss = (t * (log_t - (z - most - torch.log(total)).gather(1, s["ids"]))).sum(1)
    if do == "distill":
        return {"loss": loss}
    d = e / total
    d.scatter_add_(1, s["ids"], -t)
    return {"loss": loss, "dlogits": (d * (s["dloss"] * s["scale"])[:, None]).to(kind)}


def _centred(h):
    """(h less its row's mean, the factor that gives it a variance of 1)."""
    mean = h.double().mean(1, keepdim=True)
    c = h.double() - mean
    return c.float(), torch.rsqrt(c.square().mean(1, keepdim=True) + EPS_NORM).float()


def _quantise(y):
    """Rows in 8 bits: whole numbers of a 127th of the row's largest magnitude."""
    big = y.abs().amax(1, keepdim=True)
    q = torch.round(y * torch.where(big > 0, 127.0 / big, 0.0))
    return q.to(torch.int8), (big / 127.0)[:, 0].contiguous()


def _act(act, z):
    if act == "relu":
        return z.clamp_min(0.0)
    if act == "gelu":
        return z * (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _slope(act, z):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * (torch.exp(-0.5 * (z * z)) / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


# ---- in 64 bits ----


def exact(case, seed):
    """The definitions in 64 bits, written apart from the forms above."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    up = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    do = case["do"]
    if do == "embed":
        seen = s["tokens"] >= 0
        y = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
        y[seen] = case["scale"] * up["weight"][s["tokens"][seen]]
        return {"y": y}
    if do == "embed_back":
        seen = s["tokens"] >= 0
        d = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
        return {"dweight": d.index_put_((s["tokens"][seen],), case["scale"] * up["dy"][seen], accumulate=True)}
    if do in ("norm", "norm_back"):
        h = up["x"] + up["residual"] if do == "norm" and case["residual"] else up["x"]
        var, mean = torch.var_mean(h, 1, keepdim=True, correction=0)
        inv = (var + EPS_NORM) ** -0.5
        hat = inv * (h - mean)
        if do == "norm":
            y = hat * up["weight"] + up["bias"]
            if case["int8"]:
                scale = y.abs().max(1, keepdim=True).values / 127
                y = scale * torch.round(y / scale)
            return {"y": y, "h": h}
        a, d = up["dy"] * up["weight"], case["dim"]
        dx = inv / d * (d * a - a.sum(1, keepdim=True) - hat * (a * hat).sum(1, keepdim=True))
        return {"dx": dx + up["residual"] if case["residual"] else dx, "dweight": torch.linalg.vecdot(up["dy"], hat, dim=0),
                "dbias": up["dy"].sum(0)}
    acts = {"none": lambda z: z, "relu": torch.relu, "silu": lambda z: z * torch.sigmoid(z),
            "gelu": lambda z: 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))}
    slopes = {"none": torch.ones_like, "relu": lambda z: torch.heaviside(z, torch.zeros_like(z)),
              "silu": lambda z: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z),
              "gelu": lambda z: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}
    if do == "gated_back":
        g, u = up["pre"].chunk(2, 1)
        dz = torch.cat([slopes[case["act"]](g) * u, acts[case["act"]](g)], 1) * up["dy"].repeat(1, 2)
        dz = dz.to(TYPES[case["type"]]).double()
        return {"dx": dz @ up["weight"], "dweight": dz.t() @ up["x"], "dbias": dz.sum(0) if case["bias"] else None, "dz": dz}
    if do in ("gated", "gated_int8"):
        if do == "gated":
            z = up["x"] @ up["weight"].t()
        else:
            scale = up["x"].abs().max(1, keepdim=True).values / 127
            z = (torch.round(up["x"] / scale) @ s["wq"].double().t()) * scale * up["wscale"]
        z = z + up["bias"] if case["bias"] else z
        g, u = z.chunk(2, 1)
        return {"y": u * acts[case["act"]](g), "pre": z if case.get("pre") else None}
    z = up["logits"] * s.get("scale", 1.0)
    lse = torch.logsumexp(z, 1, keepdim=True)
    if do in ("logprob", "logprob_train"):
        row = torch.arange(case["rows"], device="cuda")
        seen = s["tokens"] >= 0
        logp = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
        logp[seen] = z[row[seen], s["tokens"][seen]] - lse[seen, 0]
        p = torch.exp(z - lse)
        entropy = torch.special.entr(p).sum(1)
        if do == "logprob":
            k = case["top"]
            ids = torch.argsort(-z, dim=1, stable=True)[:, :k] if k else None
            return {"logp": logp, "entropy": entropy, "top_logp": torch.take_along_dim(z, ids, 1) - lse if k else None,
                    "top_ids": ids}
        one = torch.zeros_like(p)
        one[row[seen], s["tokens"][seen]] = 1.0
        d = up["dlogp"][:, None] * (one - p) * seen[:, None]
        if case["entropy"]:
            d += up["dentropy"][:, None] * (torch.special.entr(p) - p * entropy[:, None])
        return {"logp": logp, "entropy": entropy if case["entropy"] else None, "dlogits": d}
    t = torch.softmax(up["teacher"] * s["scale"], 1)
    loss = -(torch.special.entr(t).sum(1)) - (t * (torch.take_along_dim(z, s["ids"], 1) - lse)).sum(1)
    if do == "distill":
        return {"loss": loss}
    q = torch.exp(z - lse)
    q[torch.arange(case["rows"], device="cuda")[:, None], s["ids"]] -= t
    return {"loss": loss, "dlogits": s["scale"] * up["dloss"][:, None] * q}


# ---- what a pass cannot do without ----


def work(case):
    do, b = case["do"], {"f32": 4, "bf16": 2, "f16": 2}[case["type"]]
    if do in ("embed", "embed_back"):
        n = case["rows"] * case["dim"]
        if do == "embed":  # every row is read once and written once, at the most as many as there are words
            return {"bytes": (n + min(case["rows"], case["vocab"]) * case["dim"]) * b + 8 * case["rows"], "flops": n}
        return {"bytes": n * b + 8 * case["rows"] + 4 * case["vocab"] * case["dim"], "flops": 2 * n}
    if do in ("norm", "norm_back"):
        n, d = case["rows"] * case["dim"], case["dim"]
        if do == "norm":  # x, the residual and its sum where there is one, y (the values of the 8 bits)
            return {"bytes": n * (b + (2 * b if case["residual"] else 0) + (4 if case["int8"] else b)) + 2 * d * b, "flops": 8 * n}
        return {"bytes": n * b * (4 if case["residual"] else 3) + d * (b + 8), "flops": 16 * n}
    if do.startswith("gated"):
        m, k, n = case["rows"], case["in"], case["out"]
        bias = 2 * n * b if case["bias"] else 0
        if do == "gated_back":  # dy, both inputs of the product and their gradient; x, its gradient, the weights and theirs
            return {"bytes": 5 * m * n * b + (2 * m * k + 2 * n * k) * b + 8 * n * k + (8 * n if case["bias"] else 0),
                    "flops": 8 * m * n * k}
        weight = 2 * n * k * b if do == "gated" else 2 * n * k + 8 * n
        return {"bytes": m * k * b + weight + bias + m * n * b * (3 if case.get("pre") else 1), "flops": 4 * m * n * k}
    n = case["rows"] * case["vocab"]
    few = case["rows"] * (16 + 12 * case.get("top", 0))
    return {"bytes": n * b * (2 if do.endswith("train") else 1) + few, "flops": n * (10 if do.endswith("train") else 6)}
