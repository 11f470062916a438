"""Argument checks and launches of the layers' and the optimiser's C entry points, without a GPU: host code only, the
HIP calls recorded in place of made.  What is refused launches nothing; what is taken launches grids that a dispatch
holds (fewer than 2^32 threads)."""
import hip_stub

COMMON = """
import sys
sys.path.insert(0, ROOT)
from paper_1704_05021_amd import gd
gd.LIB_PATH = LIB
G = gd._lib()
h = vp()
P = 4096
def made(what, *args):
    h = vp()
    st = getattr(G, f"gd_{what}_create")(ctypes.byref(h), *args)
    assert st == 0 and h.value, (what, args, st)
    return h
def io(t, **fields):
    v = t()
    for k, x in fields.items(): setattr(v, k, x)
    return v
def call(name, h, v):
    before = get("g_launches")
    st = getattr(G, name)(h, v, None)
    n = get("g_launches") - before
    assert st == 0 or n == 0, (name, st, n)
    return st, n
def but(base, **change): return {**base, **change}
"""


def run(code, tmp_path):
    hip_stub.run(f"ROOT, LIB = {hip_stub.ROOT!r}, {hip_stub.LIB!r}" + COMMON + code, tmp_path)


def test_norm(tmp_path):
    run("""
for dim, ty in ((0, 1), (32769, 1), (8, 3), (8, -1)):
    assert G.gd_norm_create(ctypes.byref(h), dim, ty) == 1 and h.value is None
assert G.gd_norm_create(None, 8, 1) == 1
n = made("norm", 64, 1)
ok = dict(rows=5, x=P, weight=P, y=P, x_stride=64, y_stride=64, eps=1e-6)
assert call("gd_norm_forward", n, io(gd._NormIO, **ok)) == (0, 1)
assert call("gd_norm_forward", n, io(gd._NormIO, **but(ok, rows=0, x=None))) == (0, 0)
assert call("gd_norm_forward", n, io(gd._NormIO, **but(ok, rows=2**40))) == (0, 1)  # the grid goes round
for bad in (dict(x=None), dict(weight=None), dict(y=None), dict(x_stride=63), dict(y_stride=0), dict(eps=-1.0),
            dict(eps=float("nan")), dict(eps=float("inf")), dict(residual=P), dict(sum=P, sum_stride=63)):
    assert call("gd_norm_forward", n, io(gd._NormIO, **but(ok, **bad)))[0] == 1, bad
ok = dict(rows=5, dy=P, x=P, weight=P, dx=P, dweight=P, dy_stride=64, x_stride=64, dx_stride=64, eps=1e-6)
assert call("gd_norm_backward", n, io(gd._NormGrad, **ok)) == (0, 1)  # few rows: one block
assert call("gd_norm_backward", n, io(gd._NormGrad, **but(ok, rows=2**20))) == (0, 2)
assert call("gd_norm_backward", n, io(gd._NormGrad, **but(ok, dweight=None))) == (0, 1)
assert call("gd_norm_backward", n, io(gd._NormGrad, **but(ok, rows=0, dy=None))) == (0, 1)  # zeros
assert call("gd_norm_backward", n, io(gd._NormGrad, **but(ok, rows=0, accumulate=1))) == (0, 0)
for bad in (dict(dy=None), dict(x=None), dict(weight=None), dict(dx=None), dict(dx_stride=1), dict(dsum=P)):
    assert call("gd_norm_backward", n, io(gd._NormGrad, **but(ok, **bad)))[0] == 1, bad
assert G.gd_norm_forward(None, io(gd._NormIO), None) == 1
assert G.gd_norm_forward(n, None, None) == 1
frees = get("g_frees"); G.gd_norm_destroy(n); assert get("g_frees") > frees
G.gd_norm_destroy(None)
for args, want in (((P, 1, 3, 0, 8, P, 8, P), 1), ((P, 3, 3, 8, 8, P, 8, P), 1), ((None, 1, 3, 8, 8, P, 8, P), 1), ((P, 1, 3, 8, 7, P, 8, P), 1),
                   ((P, 1, 3, 8, 8, P, 7, P), 1), ((P, 1, 3, 8, 8, P, 8, None), 1), ((None, 1, 0, 8, 8, None, 8, None), 0), ((P, 1, 3, 8, 8, P, 8, P), 0)):
    assert G.gd_quantise_rows(*args, None) == want, args
""", tmp_path)


def test_adamw(tmp_path):
    run("""
def create(off, state=0, decay=None):
    o = (u64 * len(off))(*off)
    dk = None if decay is None else (ctypes.c_float * len(decay))(*decay)
    return G.gd_adamw_create(ctypes.byref(h), o, len(off) - 1, state, dk)
for off, st in (([0, 5, 3], 2), ([1, 5], 2), ([0, 2**40 + 1], 2)):
    assert create(off) == st, off
assert create([0, 4], 2) == 1 and create([0, 4], 0, [float("nan")]) == 1 and create([0, 4], 0, [-1.0]) == 1
assert G.gd_adamw_create(ctypes.byref(h), None, 1, 0, None) == 1 and G.gd_adamw_create(None, None, 1, 0, None) == 1
assert G.gd_adamw_create(ctypes.byref(h), (u64 * 1)(0), 0, 0, None) == 1
off = (u64 * 4)(0, 300, 300, 10000)
for state, blocks in ((0, 2 + 38), (1, 2 + 38)):
    o = made("adamw", off, 3, state, None)
    assert G.gd_adamw_blocks(o) == blocks
    ok = dict(params=P, grad=P, m=P, v=P, m_unit=P, v_unit=P, copy_type=1, step=1, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8,
              weight_decay=0.1, grad_scale=1.0)
    assert call("gd_adamw_step", o, io(gd._AdamWIO, **ok)) == (0, 1)
    assert call("gd_adamw_step", o, io(gd._AdamWIO, **but(ok, max_norm=1.0))) == (0, 3)
    inf, nan = float("inf"), float("nan")
    for bad in (dict(params=None), dict(grad=None), dict(m=None), dict(v=None), dict(step=0), dict(lr=-1.0), dict(lr=nan),
                dict(lr=inf), dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=nan), dict(eps=0.0), dict(eps=1e-39), dict(eps=nan), dict(weight_decay=-1.0),
                dict(max_norm=-1.0), dict(max_norm=nan), dict(grad_scale=inf), dict(grad_type=3), dict(copy=P, copy_type=0),
                dict(copy=P, copy_type=7)) + ((dict(m_unit=None), dict(v_unit=None)) if state else ()):
        assert call("gd_adamw_step", o, io(gd._AdamWIO, **but(ok, **bad)))[0] == 1, bad
    st = G.gd_adamw_decode(o, P, P, P, P, P, P, None)
    assert st == (0 if state else 1)
    if state:
        assert G.gd_adamw_decode(o, P, P, None, P, P, P, None) == 1
    G.gd_adamw_destroy(o)
assert G.gd_adamw_blocks(None) == 0
e = made("adamw", (u64 * 2)(0, 0), 1, 0, None)
assert call("gd_adamw_step", e, io(gd._AdamWIO, **but(ok, params=None, grad=None, m=None, v=None)))[0] == 0
""", tmp_path)


def test_linear(tmp_path):
    run("""
for k, n, ty, act, rows in ((0, 4, 1, 0, 1), (4, 0, 1, 0, 1), (2**22 + 1, 4, 1, 0, 1), (4, 4, 3, 0, 1), (4, 4, 1, 4, 1), (4, 4, 1, -1, 1), (4, 4, 1, 0, 2**31)):
    assert G.gd_linear_create(ctypes.byref(h), k, n, ty, act, rows) == 1, (k, n)
    assert h.value is None
class Dim(ctypes.Structure): _fields_ = [("x", u32), ("y", u32), ("z", u32)]
for ty in (0, 1, 2):
    for k, n in ((64, 48), (65, 47), (4096, 4096), (4095, 10)):
        l = made("linear", k, n, ty, 1, 2**31 - 1)
        for rows in (1, 16, 17, 100, 5000, 2**20):
            f = dict(rows=rows, x=P, weight=P, y=P, x_stride=k, weight_stride=k, y_stride=n)
            st, launches = call("gd_linear_forward", l, io(gd._LinearIO, **f))
            assert st == 0 and 1 <= launches <= 4, (ty, k, n, rows, launches)
            assert Dim.in_dll(S, "g_grid").x < 2**22
            b = dict(rows=rows, dy=P, x=P, weight=P, pre=P, dz=P, dx=P, dweight=P, dbias=P, dy_stride=n, x_stride=k,
                     weight_stride=k, pre_stride=n, dz_stride=n, dx_stride=k, dweight_stride=k)
            st, launches = call("gd_linear_backward", l, io(gd._LinearGrad, **b))
            assert st == 0 and 2 <= launches <= 10, (ty, k, n, rows, launches)
        G.gd_linear_destroy(l)
l = made("linear", 64, 48, 1, 1, 100)
f = dict(rows=20, x=P, weight=P, y=P, x_stride=64, weight_stride=64, y_stride=48)
assert call("gd_linear_forward", l, io(gd._LinearIO, **f))[0] == 0
assert call("gd_linear_forward", l, io(gd._LinearIO, **but(f, rows=0, x=None, y=None))) == (0, 0)
for bad in (dict(rows=101), dict(x=None), dict(weight=None), dict(y=None), dict(x_stride=63), dict(weight_stride=0), dict(y_stride=47),
            dict(x_stride=2**22 + 1), dict(x_scale=P), dict(weight_scale=P), dict(residual=P), dict(pre=P, pre_stride=1)):
    assert call("gd_linear_forward", l, io(gd._LinearIO, **but(f, **bad)))[0] == 1, bad
assert call("gd_linear_forward", l, io(gd._LinearIO, **but(f, x_scale=P, weight_scale=P)))[0] == 0
b = dict(rows=20, dy=P, x=P, weight=P, pre=P, dz=P, dx=P, dweight=P, dbias=P, dy_stride=48, x_stride=64, weight_stride=64,
         pre_stride=48, dz_stride=48, dx_stride=64, dweight_stride=64)
assert call("gd_linear_backward", l, io(gd._LinearGrad, **b))[0] == 0
for bad in (dict(rows=101), dict(dy=None), dict(x=None), dict(weight=None), dict(pre=None), dict(dz=None), dict(dy_stride=47),
            dict(x_stride=1), dict(weight_stride=63), dict(pre_stride=0), dict(dz_stride=47), dict(dx_stride=63), dict(dweight_stride=63)):
    assert call("gd_linear_backward", l, io(gd._LinearGrad, **but(b, **bad)))[0] == 1, bad
assert call("gd_linear_backward", l, io(gd._LinearGrad, **but(b, rows=0, accumulate=1))) == (0, 0)
long = made("linear", 131073, 8, 1, 0, 4)
g = dict(rows=2, x=P, weight=P, y=P, x_scale=P, weight_scale=P, x_stride=131073, weight_stride=131073, y_stride=8)
assert call("gd_linear_forward", long, io(gd._LinearIO, **g))[0] == 2
assert G.gd_linear_forward(None, io(gd._LinearIO, **f), None) == 1 and G.gd_linear_backward(l, None, None) == 1
""", tmp_path)


def test_out_of_memory_is_an_error_and_leaks_nothing(tmp_path):
    run("""
put("g_other_capture", 1)  # the stub then refuses allocations
before = get("g_allocs"), get("g_frees")
assert G.gd_norm_create(ctypes.byref(h), 8, 1) == 5 and G.gd_linear_create(ctypes.byref(h), 8, 8, 1, 0, 8) == 5
assert G.gd_adamw_create(ctypes.byref(h), (u64 * 2)(0, 8), 1, 1, None) == 5
assert h.value is None and get("g_allocs") - before[0] == get("g_frees") - before[1]
""", tmp_path)
