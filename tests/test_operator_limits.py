"""Sizes at and past the stated limits of the layers' and the optimiser's C entry points, without a GPU (see hip_stub)."""
import hip_stub
import test_operator_checks


def run(code, tmp_path):
    hip_stub.run(f"ROOT, LIB = {hip_stub.ROOT!r}, {hip_stub.LIB!r}" + test_operator_checks.COMMON + code, tmp_path)


def test_adamw_layouts_are_counted_before_their_table_is_made(tmp_path):
    """2^40 elements are 2^32 blocks, as many as have numbers; their table of gigabytes is what this process cannot
    hold.  One block more is no layout, which is known without a table."""
    run("""
import resource
def create(off, state): return G.gd_adamw_create(ctypes.byref(h), (u64 * len(off))(*off), len(off) - 1, state, None)
pages = int(open("/proc/self/statm").read().split()[0])
resource.setrlimit(resource.RLIMIT_AS, (pages * 4096 + (1 << 30),) * 2)
for state in (0, 1):
    assert create([0, 2**40], state) == 5  # GD_ERR_OOM
    for off in ([0, 1, 2**40], [0, 2**39 + 1, 2**40], [0, 2**40 + 1], [0, 2**41]):
        assert create(off, state) == 2, off  # GD_ERR_LAYOUT
    assert create([0, 1, 2**24], state) == 0 and G.gd_adamw_blocks(h) == 1 + 2**16
""", tmp_path)


def test_linear_calls_of_the_most_rows(tmp_path):
    """Every number of rows that a handle takes is launched, or refused before anything is: no call ends halfway."""
    run("""
def fits(a, b): return -(-a // 128) * -(-b // 128) < 2**24
for ty in (0, 1, 2):
    for k, n in ((1, 1), (8, 8), (100, 1), (1, 100), (64, 64), (129, 1), (1, 129), (300, 40), (1, 1000), (1000, 8)):
        l = made("linear", k, n, ty, 1, 2**31 - 1)
        for rows in (2**31 - 1, 2**31 - 127, 2**31 - 128, 2**31 - 4096, 2**30 + 1, 2**30 - 128, 2**29, 2**24 + 3):
            f = dict(rows=rows, x=P, weight=P, y=P, x_stride=k, weight_stride=k, y_stride=n)
            for scales in ({}, dict(x_scale=P, weight_scale=P)):
                st, launches = call("gd_linear_forward", l, io(gd._LinearIO, **but(f, **scales)))
                assert (st, launches > 0) == ((0, True) if fits(n, rows) else (2, False)), (ty, k, n, rows, st)
            b = dict(rows=rows, dy=P, x=P, weight=P, pre=P, dz=P, dx=P, dweight=P, dbias=P, dy_stride=n, x_stride=k,
                     weight_stride=k, pre_stride=n, dz_stride=n, dx_stride=k, dweight_stride=k)
            st, launches = call("gd_linear_backward", l, io(gd._LinearGrad, **b))
            assert (st, launches > 0) == ((0, True) if fits(k, rows) else (2, False)), (ty, k, n, rows, st)
            assert call("gd_linear_backward", l, io(gd._LinearGrad, **but(b, dx=None)))[0] == 0
        G.gd_linear_destroy(l)
wide = made("linear", 2**22, 2**22, 1, 0, 8)
b = dict(rows=8, dy=P, x=P, weight=P, dx=P, dy_stride=2**22, x_stride=2**22, weight_stride=2**22, dx_stride=2**22, dweight_stride=2**22)
assert call("gd_linear_backward", wide, io(gd._LinearGrad, **b))[0] == 0
assert call("gd_linear_backward", wide, io(gd._LinearGrad, **but(b, dweight=P)))[0] == 2
""", tmp_path)
