"""hip_stub with a record of what is launched: each kernel's name, grid and block, and the first bytes of a product's
arguments.  Child code calls launches(call) for the records of one call's launches in order, each a dict with "name"
(the kernel's), "what" (the mangled name, template arguments and all), "grid", "block" and, for products, "args"."""
import hip_stub
import test_operator_checks

RECORD = r"""
#include <stdint.h>
#include <string.h>
typedef struct { uint32_t x, y, z; } size3;
typedef struct { const char* name; size3 grid, block; unsigned char args[64]; } launch_t;
launch_t g_log[64];
int g_logged;
static struct { const void* f; const char* name; } kernels[8192];
static int num_kernels;
void __hipRegisterFunction(void** modules, const void* f, char* device, const char* name, unsigned limit, void* tid,
                           void* bid, void* block, void* grid, int* wave) {
    if (num_kernels < 8192) { kernels[num_kernels].f = f; kernels[num_kernels].name = name; ++num_kernels; }
}
static void record(const void* f, size3 grid, size3 block, void** args) {
    launch_t* l = &g_log[g_logged++ % 64];
    l->name = "";
    for (int i = 0; i < num_kernels; ++i)
        if (kernels[i].f == f) l->name = kernels[i].name;
    l->grid = grid; l->block = block;
    if (strstr(l->name, "GemmArgs")) memcpy(l->args, args[0], sizeof l->args);
}
"""

CHILD = r"""
import re, struct
class Size3(ctypes.Structure): _fields_ = [("x", u32), ("y", u32), ("z", u32)]
class Launch(ctypes.Structure): _fields_ = [("name", ctypes.c_char_p), ("grid", Size3), ("block", Size3), ("args", ctypes.c_ubyte * 64)]
def launches(call):
    first = get("g_logged")
    assert call() == 0
    log = (Launch * 64).in_dll(S, "g_log")
    out = []
    for i in range(first, get("g_logged")):
        l = log[i % 64]
        what = l.name.decode()
        one = {"name": re.match(r"_ZN2gd\d+(k_[a-z_]+?)(I|E)", what)[1], "what": what, "grid": (l.grid.x, l.grid.y), "block": l.block.x}
        if "GemmArgs" in what:  # the operands' addresses and strides, then these
            one["args"] = dict(zip(("I", "J", "K", "tiles_i", "tiles_j", "steps"), struct.unpack("6I", bytes(l.args)[32:56])))
        out.append(one)
    return out
"""


def run(code, tmp_path):
    kept = hip_stub.STUB
    before = "g_grid = grid; ++g_launches; return 0;"
    assert before in kept
    hip_stub.STUB = RECORD + kept.replace(before, "size3 a = {grid.x, grid.y, grid.z}, b = {block.x, block.y, block.z}; "
                                                  "record(f, a, b, args); " + before)
    try:
        hip_stub.run(f"ROOT, LIB = {hip_stub.ROOT!r}, {hip_stub.LIB!r}" + test_operator_checks.COMMON + CHILD + code, tmp_path)
    finally:
        hip_stub.STUB = kept
