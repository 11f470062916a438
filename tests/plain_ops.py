"""Plain 64-bit definitions of the operators around the compressor, on the CPU, for the tests: written from the
formulas with numpy-like torch operations, and the rounding allowances the tests compare under."""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}  # half an ulp, relative: 2^-24, 2^-8, 2^-11
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}  # of the smallest ones
E = 2.0 ** -24  # one rounding of the 32-bit arithmetic inside


def d(t):
    return None if t is None else t.detach().cpu().double()


def close(got, want, allow, what):
    """Every |got - want| <= allow (a tensor or a number); equal infinities and NaN in the same places."""
    got, want = d(got).reshape(want.shape), d(want)
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    fine = want.isfinite()
    assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()]), f"{what}: infinities differ"
    off = ((got - want).abs() - allow)[fine]
    if off.numel():
        worst = int(off.argmax())
        assert off.max() <= 0, (f"{what}: {got[fine].flatten()[worst]} for {want[fine].flatten()[worst]}, "
                                f"{float(off.max())} past the allowance")


def rounded(want, dtype):
    """Allowance of one rounding to dtype."""
    return ULP[dtype] * want.abs() + LEAST[dtype]


def norm(x, weight, residual, eps):
    h = x if residual is None else x + residual
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * weight


def norm_back(dy, h, weight, dsum, eps):
    """(dx, dweight) and the sums of magnitudes that their roundings are relative to."""
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    xhat, a = h * r, dy * weight
    dx = r * (a - xhat * (a * xhat).mean(1, keepdim=True))
    size = r * (a.abs() + xhat.abs() * (a * xhat).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, size = dx + dsum, size + dsum.abs()
    return dx, (dy * xhat).sum(0), size, (dy * xhat).abs().sum(0)


def act(kind, z):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / math.sqrt(2.0)))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def slope(kind, z):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s + z * s * (1.0 - s)
    return torch.ones_like(z)


def product(a, b):
    """a b^T and the allowance of forming it in 32 bits: the roundings of K sums are independent, each half an
    ulp of a partial sum, and partial sums stay within a few times the 2-norm of the products; 16 times that."""
    s = a @ b.t()
    return s, 16.0 * E * math.sqrt(max(a.shape[1], 1)) * torch.sqrt((a * a) @ (b * b).t())


def quantise(y):
    """(scale, step) per row of the 8-bit form."""
    big = y.abs().amax(1, keepdim=True)
    return big / 127.0


BLOCK = 256


def block_spans(offsets):
    """(start, end) of every block of 256 elements, tensor by tensor."""
    return [(a, min(a + BLOCK, end)) for start, end in zip(offsets, offsets[1:]) for a in range(start, end, BLOCK)]


def adamw(p, g, m, v, step, lr, betas, eps, wd, decay):
    """One step on 64-bit vectors; decay is the weight decay's factor per element."""
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    upd = lr * (m / (1 - b1 ** step)) / (torch.sqrt(v / (1 - b2 ** step)) + eps)
    return p - lr * wd * decay * p - upd, m, v, upd
