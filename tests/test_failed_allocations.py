"""A create that runs out of memory reports it and leaves no error behind for the next call, here or in the caller's
program (without a GPU: hip_stub, whose runtime holds the last error until it is read)."""
import hip_stub
import test_operator_checks

HELD = (("int hipGetLastError(void) { return 0; }", "int g_error; int hipGetLastError(void) { int e = g_error; g_error = 0; return e; }"),
        ("++g_refused; return 900;", "++g_refused; g_error = 900; return 900;"))


def test_the_next_call_is_not_told(tmp_path, monkeypatch):
    stub = hip_stub.STUB
    for old, new in HELD:
        assert old in stub
        stub = stub.replace(old, new)
    monkeypatch.setattr(hip_stub, "STUB", stub)
    hip_stub.run(f"ROOT, LIB = {hip_stub.ROOT!r}, {hip_stub.LIB!r}" + test_operator_checks.COMMON + """
n, l, o = made("norm", 8, 1), made("linear", 8, 8, 1, 0, 64), made("adamw", (u64 * 2)(0, 8), 1, 0, None)
calls = {
    "norm": lambda: G.gd_norm_forward(n, io(gd._NormIO, rows=2, x=P, weight=P, y=P, x_stride=8, y_stride=8), None),
    "linear": lambda: G.gd_linear_forward(l, io(gd._LinearIO, rows=2, x=P, weight=P, y=P, x_stride=8, weight_stride=8, y_stride=8), None),
    "adamw": lambda: G.gd_adamw_step(o, io(gd._AdamWIO, params=P, grad=P, m=P, v=P, step=1, lr=1e-3, eps=1e-8, grad_scale=1.0), None),
    "quantise": lambda: G.gd_quantise_rows(P, 1, 2, 8, 8, P, 8, P, None),
}
creates = {
    "norm": lambda: G.gd_norm_create(ctypes.byref(h), 8, 1),
    "linear": lambda: G.gd_linear_create(ctypes.byref(h), 8, 8, 1, 0, 64),
    "adamw": lambda: G.gd_adamw_create(ctypes.byref(h), (u64 * 2)(0, 8), 1, 1, None),
    "compressor": lambda: L.gd_create(ctypes.byref(h), (u64 * 2)(0, 8), 1),
}
for create in creates:
    for call in calls:
        assert calls[call]() == 0, call
        put("g_other_capture", 1)  # the stub then refuses allocations
        assert creates[create]() == 5 and h.value is None, create
        put("g_other_capture", 0)
        assert get("g_error") == 0, create  # nothing for a launch of the caller's own to find
        assert calls[call]() == 0, (create, call)
""", tmp_path)
