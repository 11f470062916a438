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
