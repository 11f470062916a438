"""The operators around the compressor whose speed is tracked: what makes a worker's gradient and what uses the server's.

A worker's layers (``gd.RMSNorm``, ``gd.Linear``) run forward and write their weights' gradients straight into the flat
gradient that the compressor takes; a server turns the summed gradient into new parameters (``gd.AdamW``).  Serving
runs the same layers on single tokens and on 8-bit weights.  Each case is one call as such a program makes it; the
plain form of each is elementary torch operations in 32 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256            # elements that share one scale of the 8-bit states
EPS_NORM = 1e-6
LR, BETAS, EPS, DECAY, STEP, MAX_NORM = 1e-3, (0.9, 0.999), 1e-8, 0.1, 1000, 1.0
TINY = 2.0 ** -100     # the least maximum that the 8-bit states resolve


def listed():
    return [
        # optimiser: the paper's MNIST network, every tensor in one call, where launches count
        {"name": "adamw_mnist", "do": "adamw", "net": "mlp", "widths": "784-512-512-10", "bits": 32, "grad": "f32",
         "clip": False, "copy": "none"},
        # a 20M-element network trained in mixed precision: clipped by its norm, a bfloat16 copy for the layers
        {"name": "adamw_mlp_20m_clip", "do": "adamw", "net": "mlp", "widths": "784-4096-4096-10", "bits": 32,
         "grad": "f32", "clip": True, "copy": "bf16"},
        # the benchmark's NMT-shaped set, 137M elements with mostly empty embedding rows, states in 8 bits
        {"name": "adamw_nmt_137m_8bit", "do": "adamw", "net": "nmt", "vocab": 85_000, "emb": 500, "hidden": 1024,
         "blocks": 6, "bits": 8, "grad": "f32", "clip": False, "copy": "none"},
        # norm: one token of a decoder, 8-bit output for the products behind it
        {"name": "norm_token_int8", "do": "norm", "rows": 1, "dim": 4096, "type": "bf16", "residual": True, "int8": True},
        # a training batch forward: the residual stream is added and kept
        {"name": "norm_batch", "do": "norm", "rows": 8192, "dim": 4096, "type": "bf16", "residual": True, "int8": False},
        # the same backward, with the gradient that comes down the residual stream
        {"name": "norm_batch_back", "do": "norm_back", "rows": 8192, "dim": 4096, "type": "bf16", "residual": True},
        # the NMT model's ragged width and tokens of a step, in 32 bits
        {"name": "norm_500_back", "do": "norm_back", "rows": 3000, "dim": 500, "type": "f32", "residual": False},
        # layer: one token of a decoder, a square projection with everything in its epilogue
        {"name": "linear_token", "do": "linear", "rows": 1, "in": 4096, "out": 4096, "type": "bf16", "act": "silu",
         "bias": True, "residual": True, "pre": False},
        # a training batch forward, the input of the activation kept for the backward
        {"name": "linear_batch", "do": "linear", "rows": 8192, "in": 4096, "out": 4096, "type": "bf16", "act": "gelu",
         "bias": True, "residual": False, "pre": True},
        # its backward: gradients of input, weights and bias
        {"name": "linear_batch_back", "do": "linear_back", "rows": 8192, "in": 4096, "out": 4096, "type": "bf16",
         "act": "relu", "bias": True},
        # the MNIST network's first layer at the paper's batch of 40, backward: small and ragged
        {"name": "linear_mnist_back", "do": "linear_back", "rows": 40, "in": 784, "out": 512, "type": "f16",
         "act": "relu", "bias": True},
        # a prompt through an 8-bit layer: the input is quantised by rows, then multiplied
        {"name": "linear_prompt_int8", "do": "linear_int8", "rows": 3000, "in": 4096, "out": 4096, "type": "bf16",
         "act": "none", "bias": False, "residual": True},
    ]


def draw(rng):
    """One more case of these ranges: any operator and direction, sizes over their logarithm, odd ones among them."""
    def log(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        n = n if rng.random() < 0.5 else max(lo, n - n % 64)
        return 3000 if n == 3072 else n  # 3,000: the tokens of an NMT step

    do = rng.choice(["adamw", "adamw", "norm", "norm_back", "linear", "linear", "linear_back", "linear_int8"])
    if do == "adamw":
        case = {"do": do, "bits": rng.choice([32, 8]), "grad": rng.choice(["f32", "f32", "bf16"]),
                "clip": rng.random() < 0.5, "copy": rng.choice(["none", "bf16", "f16"])}
        if rng.random() < 0.5:
            return {**case, "net": "mlp", "widths": "784-%d-%d-10" % (log(64, 4300), log(64, 4300))}
        return {**case, "net": "nmt", "vocab": log(2000, 80_000), "emb": log(64, 500), "hidden": log(96, 1024),
                "blocks": rng.randint(1, 6)}
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if do in ("norm", "norm_back"):
        case = {"do": do, "rows": log(1, 8192), "dim": log(64, 8192 if kind != "f32" else 4096), "type": kind,
                "residual": rng.random() < 0.6}
        return {**case, "int8": rng.random() < 0.4} if do == "norm" else case
    kind = rng.choice(["bf16", "bf16", "f16"])
    case = {"do": do, "rows": log(1, 8192), "in": log(128, 4096), "out": log(128, 4096), "type": kind,
            "act": rng.choice(["none", "relu", "gelu", "silu"]), "bias": rng.random() < 0.6}
    if do == "linear":
        return {**case, "residual": rng.random() < 0.5, "pre": rng.random() < 0.5}
    return {**case, "residual": rng.random() < 0.5} if do == "linear_int8" else case


def _shapes(case):
    """Tensor shapes of the case's network, in the order a flat gradient holds them."""
    if case["net"] == "mlp":
        a, b, c, d = (int(x) for x in case["widths"].split("-"))
        return [(a, b), (b,), (b, c), (c,), (c, d), (d,)]
    e, h = case["emb"], case["hidden"]
    return [(case["vocab"], e)] * 3 + [(h, e), (h,), (h, h), (h,)] * case["blocks"]


# ---- inputs ----


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    s = {"case": case}
    if case["do"] == "adamw":
        shapes = _shapes(case)
        off = [0]
        for shape in shapes:
            off.append(off[-1] + math.prod(shape))
        n = off[-1]
        grad, m, v = (torch.empty(n, device="cuda") for _ in range(3))
        for t, shape in enumerate(shapes):  # tensors on scales of their own; an embedding's unseen rows have no gradient
            a, b, k = off[t], off[t + 1], 10.0 ** (-4.0 + 0.25 * (t % 9))
            grad[a:b] = normal(b - a, scale=k)
            m[a:b] = normal(b - a, scale=0.3 * k)
            v[a:b] = normal(b - a, scale=k).square_().mul_(0.5).add_(0.3 * k * k)
            if case["net"] == "nmt" and t < 3:
                u = torch.rand(shape[0], 1, generator=g, device="cuda")
                grad[a:b].view(shape).mul_(u < 0.03)
                m[a:b].view(shape).mul_(u < 0.3)
                v[a:b].view(shape).mul_(u < 0.6)
        s["off"] = off
        s["decay"] = [1.0 if len(shape) > 1 else 0.0 for shape in shapes]
        s["params"] = normal(n, scale=0.02)
        s["grad"] = grad.to(TYPES[case["grad"]])
        s["copy"] = None if case["copy"] == "none" else s["params"].to(TYPES[case["copy"]])
        if case["bits"] == 8:
            block, count = _blocks(off)
            r, mu = _code(m.abs(), block, count, 127)
            rv, vu = _code(v.sqrt_(), block, count, 255)
            s["state"] = {"m": (r * m.sign()).to(torch.int8), "v": rv.to(torch.uint8), "m_unit": mu, "v_unit": vu}
            del block, r, rv
        else:
            s["state"] = {"m": m, "v": v, "m_unit": None, "v_unit": None}
    elif case["do"] in ("norm", "norm_back"):
        shape, kind = (case["rows"], case["dim"]), TYPES[case["type"]]
        s["x"] = normal(*shape, dtype=kind)
        s["weight"] = (1.0 + normal(case["dim"], scale=0.1)).to(kind)
        s["residual"] = normal(*shape, scale=2.0, dtype=kind) if case["residual"] else None
        if case["do"] == "norm_back":
            s["dy"] = normal(*shape, scale=1e-3, dtype=kind)
            s["dweight"] = torch.empty(case["dim"], device="cuda")  # a slice of the flat gradient
    else:
        rows, k, n, kind = case["rows"], case["in"], case["out"], TYPES[case["type"]]
        s["x"] = normal(rows, k, dtype=kind)
        s["weight"] = normal(n, k, scale=k ** -0.5, dtype=kind)
        s["bias"] = normal(n, scale=0.1, dtype=kind) if case["bias"] else None
        if case["do"] == "linear_back":
            s["dy"] = normal(rows, n, scale=1e-3 if kind != torch.float16 else 1.0, dtype=kind)
            s["pre"] = normal(rows, n, dtype=kind) if case["act"] != "none" else None
            s["dweight"] = torch.empty(n, k, device="cuda")  # slices of the flat gradient
            s["dbias"] = torch.empty(n, device="cuda") if case["bias"] else None
        else:
            s["residual"] = normal(rows, n, dtype=kind) if case["residual"] else None
        if case["do"] == "linear_int8":  # the weights of a served model are quantised once
            s["wq"], s["wscale"] = _quantise(s.pop("weight").float())
    if own:
        s["op"] = _handle(case, s)
    return s


def _handle(case, s):
    """What a user's program keeps of the framework: the layer's or the optimiser's plan, and its state."""
    from paper_1704_05021_amd import gd

    if case["do"] == "adamw":
        st = s["state"]
        s["state"] = gd.AdamWState(st["m"], st["v"], st["m_unit"], st["v_unit"])
        return gd.AdamW(s["off"], bits=case["bits"], decay=s["decay"])
    if case["do"] in ("norm", "norm_back"):
        return gd.RMSNorm(case["dim"], TYPES[case["type"]], eps=EPS_NORM)
    return gd.Linear(case["in"], case["out"], TYPES[case["type"]], act=case["act"], max_rows=case["rows"])


# ---- one pass ----


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, op = s["case"], s["op"]
    if case["do"] == "adamw":
        norm = op.step(s["params"], s["grad"], s["state"], STEP, lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY,
                       max_norm=MAX_NORM if case["clip"] else None, copy=s["copy"])
        m, v = (s["state"].m, s["state"].v) if case["bits"] == 32 else op.decode(s["state"])
        return {"params": s["params"], "m": m, "v": v, "copy": s["copy"], "norm": norm}
    if case["do"] == "norm" and case["int8"]:
        q, scale, h = op.forward_int8(s["x"], s["weight"], s["residual"])
        return {"y": q * scale[:, None], "h": h}
    if case["do"] == "norm":
        y, h = op.forward(s["x"], s["weight"], s["residual"])
        return {"y": y, "h": h}
    if case["do"] == "norm_back":
        dx, dw = op.backward(s["dy"], s["x"], s["weight"], dsum=s["residual"], dweight=s["dweight"])
        return {"dx": dx, "dweight": dw}
    if case["do"] == "linear":
        if not case["pre"]:
            return {"y": op.forward(s["x"], s["weight"], s["bias"], s["residual"])}
        y, pre = op.forward(s["x"], s["weight"], s["bias"], s["residual"], keep_pre=True)
        return {"y": y, "pre": pre}
    if case["do"] == "linear_int8":
        from paper_1704_05021_amd import gd

        q, scale = gd.quantise_rows(s["x"])
        return {"y": op.forward_int8(q, scale, s["wq"], s["wscale"], s["bias"], s["residual"])}
    dx, dw, db, dz = op.backward(s["dy"], s["x"], s["weight"], s["pre"], dweight=s["dweight"], dbias=s["dbias"])
    return {"dx": dx, "dweight": dw, "dbias": db, "dz": dz}


def _run_plain(s):
    case = s["case"]
    if case["do"] == "adamw":
        return _plain_adamw(s)
    kind = TYPES[case["type"]]
    x = s["x"].float()
    if case["do"] in ("norm", "norm_back"):
        w = s["weight"].float()
        if case["do"] == "norm":
            h = x if s["residual"] is None else x + s["residual"].float()
            y = h * _rstd(h) * w
            if case["int8"]:
                q, scale = _quantise(y)
                y = q * scale[:, None]
            return {"y": y if case["int8"] else y.to(kind), "h": h.to(kind)}
        dy, rstd = s["dy"].float(), _rstd(x)
        xhat, a = x * rstd, dy * w
        dx = rstd * (a - xhat * (a * xhat).mean(1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        s["dweight"].copy_((dy * xhat).sum(0))
        return {"dx": dx.to(kind), "dweight": s["dweight"]}
    if case["do"] == "linear_back":
        dz = s["dy"].float()
        if case["act"] != "none":
            dz = dz * _slope(case["act"], s["pre"].float())
        dz = dz.to(kind)  # the gradient at the activation's input is an output in the type, and what the products take
        d = dz.float()
        torch.mm(d.t(), x, out=s["dweight"])
        if s["dbias"] is not None:
            s["dbias"].copy_(d.sum(0))
        return {"dx": (d @ s["weight"].float()).to(kind), "dweight": s["dweight"], "dbias": s["dbias"], "dz": dz}
    if case["do"] == "linear_int8":
        q, scale = _quantise(x)
        z = (q.float() @ s["wq"].float().t()) * (scale[:, None] * s["wscale"][None, :])
    else:
        z = x @ s["weight"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(case["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(kind), "pre": z.to(kind) if case.get("pre") else None}


def _rstd(h):
    return torch.rsqrt(h.double().square().mean(1, keepdim=True) + EPS_NORM).float()


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
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * (torch.exp(-0.5 * (z * z)) / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _blocks(off):
    """(block of every element, number of blocks): blocks of 256 elements that start anew with each tensor."""
    start = torch.tensor(off[:-1], device="cuda")
    end = torch.tensor(off[1:], device="cuda")
    first = torch.cumsum((end - start + BLOCK - 1) // BLOCK, 0)
    at = torch.arange(off[-1], device="cuda")
    t = torch.bucketize(at, end, right=True)
    block = torch.div(at.sub_(start[t]), BLOCK, rounding_mode="floor")
    return block.add_((first - (end - start + BLOCK - 1) // BLOCK)[t]), int(sum((b - a + BLOCK - 1) // BLOCK for a, b in zip(off, off[1:])))


def _code(x, block, count, top):
    """(r, unit per block) of magnitudes x: x stands nearest to unit * r^2 in the root, r a whole number up to `top`."""
    big = torch.zeros(count, device="cuda").scatter_reduce_(0, block, x, "amax")
    unit = (big.clamp_min(TINY).double() / (top * top)).float()
    y = x * (1.0 / unit.double()).float()[block]
    r = torch.floor(y.sqrt() + 0.5)
    r = r + (y >= (r + 0.5).square()).float() - (y < (r - 0.5).clamp_min(0.0).square()).float()
    return r.clamp_(max=top), unit


def _plain_adamw(s):
    case, p, st = s["case"], s["params"], s["state"]
    g = s["grad"].float()
    norm = None
    if case["clip"]:
        norm = g.double().square().sum().sqrt()
        g = g * torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0).float()
        norm = norm.float().reshape(1)
    off = s["off"]
    small = case["bits"] == 8
    if small:
        block, count = _blocks(off)
        m = st["m"].float()
        m = st["m_unit"][block] * (m * m.abs())
        v = (st["v_unit"][block] * st["v"].float().square()).square_()
    else:
        m, v = st["m"], st["v"]
    m.mul_(BETAS[0]).add_(g * (1.0 - BETAS[0]))
    v.mul_(BETAS[1]).add_((g * g).mul_(1.0 - BETAS[1]))
    del g
    root = v.sqrt()
    upd = m / (root * (1.0 / math.sqrt(1.0 - BETAS[1] ** STEP)) + EPS)
    upd.mul_(LR / (1.0 - BETAS[0] ** STEP))
    t = torch.bucketize(torch.arange(off[-1], device="cuda"), torch.tensor(off[1:], device="cuda"), right=True)
    p.mul_((1.0 - (LR * DECAY) * torch.tensor(s["decay"], device="cuda"))[t]).sub_(upd)
    del upd, t
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if small:
        r, mu = _code(m.abs(), block, count, 127)
        st["m"].copy_(r * m.sign())
        st["m_unit"].copy_(mu)
        m = (mu[block] * r.square_()).mul_(m.sign())
        r, vu = _code(root, block, count, 255)
        r = torch.where(root > 0, r.clamp_min(1.0), r)
        st["v"].copy_(r)
        st["v_unit"].copy_(vu)
        v = (vu[block] * r.square_()).square_()
    return {"params": p, "m": m, "v": v, "copy": s["copy"], "norm": norm}


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
    if case["do"] == "adamw":
        off, st = s["off"], s["state"]
        sizes = [b - a for a, b in zip(off, off[1:])]
        lens = torch.tensor([min(BLOCK, n - i) for n in sizes for i in range(0, n, BLOCK)], device="cuda")
        spread = lambda u: torch.repeat_interleave(u, lens)  # noqa: E731
        g = up["grad"]
        norm = torch.linalg.vector_norm(g)
        if case["clip"]:
            g = g * min(1.0, MAX_NORM / float(norm))
        if case["bits"] == 8:
            m = spread(st["m_unit"].double()) * st["m"].double() * st["m"].double().abs()
            v = (spread(st["v_unit"].double()) * st["v"].double() ** 2) ** 2
        else:
            m, v = st["m"].double(), st["v"].double()
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
        del g
        mhat, vhat = m / (1 - BETAS[0] ** STEP), v / (1 - BETAS[1] ** STEP)
        wd = torch.repeat_interleave(torch.tensor(s["decay"], device="cuda", dtype=torch.float64) * DECAY,
                                     torch.tensor(sizes, device="cuda"))
        p = up["params"]
        p = p - LR * (mhat / (vhat.sqrt() + EPS) + wd * p)
        del mhat, vhat, wd
        if case["bits"] == 8:
            def held(x, top, least):
                ends = torch.cumsum(lens, 0)
                most = torch.segment_reduce(x, "max", lengths=lens, axis=0) if x.numel() < (1 << 24) else \
                    torch.zeros(len(lens), dtype=x.dtype, device="cuda").scatter_reduce_(
                        0, torch.bucketize(torch.arange(len(x), device="cuda"), ends, right=True), x, "amax")
                unit = spread(most.clamp_min(TINY) / top ** 2)
                r = (x / unit).sqrt().add_(0.5).floor_()
                return unit * torch.where(x > 0, r.clamp(least, top), r) ** 2

            m, v = held(m.abs(), 127, 0).mul_(m.sign()), held(v.sqrt(), 255, 1) ** 2
        return {"params": p, "m": m, "v": v, "copy": p if case["copy"] != "none" else None,
                "norm": norm.reshape(1) if case["clip"] else None}
    x = up["x"]
    if case["do"] in ("norm", "norm_back"):
        w = up["weight"]
        h = x + up["residual"] if case["do"] == "norm" and case["residual"] else x
        inv = (h.pow(2).sum(1, keepdim=True) / case["dim"] + EPS_NORM) ** -0.5
        if case["do"] == "norm":
            y = w * (h * inv)
            if case["int8"]:
                scale = y.abs().max(1, keepdim=True).values / 127
                y = scale * torch.round(y / scale)
            return {"y": y, "h": h}
        a = up["dy"] * w
        dx = inv * a - inv ** 3 * h * (a * h).sum(1, keepdim=True) / case["dim"]
        return {"dx": dx + up["residual"] if case["residual"] else dx, "dweight": (up["dy"] * h * inv).sum(0)}
    gelu = lambda z: 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))  # noqa: E731
    if case["do"] == "linear_back":
        dz, z = up["dy"], up["pre"]
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif case["act"] == "gelu":
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        elif case["act"] == "silu":
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        dz = dz.to(TYPES[case["type"]]).double()
        return {"dx": dz @ up["weight"], "dweight": dz.t() @ x, "dbias": dz.sum(0) if case["bias"] else None, "dz": dz}
    if case["do"] == "linear_int8":
        scale = x.abs().max(1, keepdim=True).values / 127
        z = (torch.round(x / scale) @ s["wq"].double().t()) * scale * up["wscale"]
    else:
        z = x @ up["weight"].t()
    z = z + up["bias"] if case["bias"] else z
    y = {"none": lambda: z, "relu": lambda: torch.relu(z), "gelu": lambda: gelu(z),
         "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
    return {"y": y + up["residual"] if case["residual"] else y, "pre": z if case.get("pre") else None}


# ---- what a pass cannot do without ----


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2, "none": 0}
    if case["do"] == "adamw":
        n = sum(math.prod(shape) for shape in _shapes(case))
        blocks = sum((math.prod(shape) + BLOCK - 1) // BLOCK for shape in _shapes(case))
        state = 16 * n if case["bits"] == 32 else 4 * n + 16 * blocks + 8 * n  # 8 bits: codes, units, the values returned
        return {"bytes": n * (8 + size[case["grad"]] + size[case["copy"]]) + state, "flops": 20 * n}
    b = size[case["type"]]
    if case["do"] in ("norm", "norm_back"):
        n, d = case["rows"] * case["dim"], case["dim"]
        if case["do"] == "norm":  # x, the residual and its sum where there is one, y (the values of the 8 bits)
            return {"bytes": n * (b + (2 * b if case["residual"] else 0) + (4 if case["int8"] else b)) + d * b, "flops": 6 * n}
        return {"bytes": n * b * (4 if case["residual"] else 3) + d * (b + 4), "flops": 12 * n}
    m, k, n = case["rows"], case["in"], case["out"]
    if case["do"] == "linear_back":
        held = m * n * b * (2 if case["act"] != "none" else 1)
        return {"bytes": held + m * n * b + (2 * m * k + n * k) * b + 4 * n * k + (4 * n if case["bias"] else 0),
                "flops": 4 * m * n * k}
    weight = n * k * b if case["do"] == "linear" else n * k + 4 * n
    out = m * n * b * (1 + bool(case["residual"]) + bool(case.get("pre")))
    return {"bytes": m * k * b + weight + out + (n * b if case["bias"] else 0), "flops": 2 * m * n * k}
