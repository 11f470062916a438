"""Argument checks and launches of the C entry points of a language model's operators (embedding, layer norm, gated layer,
log probabilities, distillation), without a GPU: host code only, the HIP calls recorded in place of made.  What is refused
launches nothing; what is taken launches grids that a dispatch holds (fewer than 2^32 threads)."""
import hip_stub
import launch_stub
from test_operator_checks import COMMON

GRIDS = """
class Dim(ctypes.Structure): _fields_ = [("x", u32), ("y", u32), ("z", u32)]
nan, inf = float("nan"), float("inf")
def refused(create, *bad):
    for args in bad:
        assert getattr(G, create)(ctypes.byref(h), *args) == 1 and h.value is None, args
    assert getattr(G, create)(None, *bad[0]) == 1
"""


def run(code, tmp_path):
    hip_stub.run(f"ROOT, LIB = {hip_stub.ROOT!r}, {hip_stub.LIB!r}" + COMMON + GRIDS + code, tmp_path)


def test_layer_norm(tmp_path):
    run("""
refused("gd_layernorm_create", (0, 1), (32769, 1), (8, 3), (8, -1))
for dim in (1, 7, 8, 64, 512, 513, 4096, 4100, 8192, 16384, 32768):
    n = made("layernorm", dim, 1)
    ok = dict(rows=5, x=P, weight=P, y=P, x_stride=dim, y_stride=dim, eps=1e-6)
    assert call("gd_layernorm_forward", n, io(gd._LayerNormIO, **ok)) == (0, 1)
    assert call("gd_layernorm_forward", n, io(gd._LayerNormIO, **but(ok, rows=2**40))) == (0, 1)  # the grid goes round
    assert Dim.in_dll(S, "g_grid").x <= 2**20
    G.gd_layernorm_destroy(n)
n = made("layernorm", 64, 1)
ok = dict(rows=5, x=P, weight=P, y=P, x_stride=64, y_stride=64, eps=1e-6)
assert call("gd_layernorm_forward", n, io(gd._LayerNormIO, **but(ok, rows=0, x=None))) == (0, 0)
for more in (dict(bias=P), dict(residual=P, residual_stride=64, sum=P, sum_stride=64), dict(y_scale=P), dict(eps=0.0)):
    assert call("gd_layernorm_forward", n, io(gd._LayerNormIO, **but(ok, **more))) == (0, 1)
for bad in (dict(x=None), dict(weight=None), dict(y=None), dict(x_stride=63), dict(y_stride=0), dict(eps=-1.0), dict(eps=nan),
            dict(eps=inf), dict(residual=P), dict(sum=P, sum_stride=63)):
    assert call("gd_layernorm_forward", n, io(gd._LayerNormIO, **but(ok, **bad)))[0] == 1, bad
ok = dict(rows=5, dy=P, x=P, weight=P, dx=P, dweight=P, dbias=P, dy_stride=64, x_stride=64, dx_stride=64, eps=1e-6)
assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **ok)) == (0, 1)  # few rows: one block
assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **but(ok, rows=2**20))) == (0, 2)
assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **but(ok, rows=2**20, dbias=None))) == (0, 2)
assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **but(ok, rows=2**20, dweight=None, dbias=None))) == (0, 1)
assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **but(ok, rows=0, dy=None))) == (0, 1)  # zeros
assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **but(ok, rows=0, accumulate=1))) == (0, 0)
for bad in (dict(dy=None), dict(x=None), dict(weight=None), dict(dx=None), dict(dx_stride=1), dict(dsum=P), dict(eps=nan)):
    assert call("gd_layernorm_backward", n, io(gd._LayerNormGrad, **but(ok, **bad)))[0] == 1, bad
assert G.gd_layernorm_forward(None, io(gd._LayerNormIO), None) == 1 and G.gd_layernorm_forward(n, None, None) == 1
assert G.gd_layernorm_backward(None, io(gd._LayerNormGrad), None) == 1 and G.gd_layernorm_backward(n, None, None) == 1
frees = get("g_frees"); G.gd_layernorm_destroy(n); assert get("g_frees") > frees
G.gd_layernorm_destroy(None)
""", tmp_path)


def test_embedding(tmp_path):
    run("""
refused("gd_embed_create", (0, 8, 1, 4), (2**31, 8, 1, 4), (8, 0, 1, 4), (8, 2**20 + 1, 1, 4), (8, 8, 3, 4), (8, 8, 1, 2**24 + 1))
for ty in (0, 1, 2):
    for dim in (1, 64, 100, 500, 513, 4096, 2**20):
        e = made("embed", 2**31 - 1, dim, ty, 2**24 if dim <= 4096 else 64)
        f = dict(rows=2**50, tokens=P, weight=P, y=P, weight_stride=dim, y_stride=dim, scale=1.0, index=1)
        assert call("gd_embed_forward", e, io(gd._EmbedIO, **f)) == (0, 1)  # the grid goes round
        assert Dim.in_dll(S, "g_grid").x <= 2**20
        for rows, accumulate in ((1, 1), (1, 0), (8, 1), (9, 1), (4096, 1), (4096, 0), (4097, 1), (4097, 0), (2**24, 1), (2**24, 0)):
            if rows > 64 and dim > 4096: continue
            # in one launch where rows are few and short; zeros of more blocks than a launch holds go round in the sorted form
            few = rows <= 4096 and -(-dim // (256 if ty == 0 else 512)) <= 16 and (accumulate or -(-(2**31 - 1) // max(16384 // dim, 1)) <= 2**22)
            slices = -(-dim // (256 if ty == 0 else 512))
            unit = next((u for u in (32, 16) if -(-rows // u) * slices >= 768), 8)
            launches = 1 if few else 1 + (rows > 4096) + 1 + (rows > unit)
            b = dict(rows=rows, tokens=P, dy=P, dweight=P, dy_stride=dim, dweight_stride=dim, scale=1.0, index=0, accumulate=accumulate)
            assert call("gd_embed_backward", e, io(gd._EmbedGrad, **b)) == (0, launches), (dim, rows)
            assert Dim.in_dll(S, "g_grid").x * 1024 < 2**32
        G.gd_embed_destroy(e)
e = made("embed", 100, 8, 1, 50)
f = dict(rows=60, tokens=P, weight=P, y=P, weight_stride=8, y_stride=8, scale=2.0, index=0)
assert call("gd_embed_forward", e, io(gd._EmbedIO, **f)) == (0, 1)
assert call("gd_embed_forward", e, io(gd._EmbedIO, **but(f, rows=0, tokens=None, y=None))) == (0, 0)
for bad in (dict(tokens=None), dict(weight=None), dict(y=None), dict(weight_stride=7), dict(y_stride=0), dict(scale=inf), dict(scale=nan),
            dict(index=2), dict(index=-1)):
    assert call("gd_embed_forward", e, io(gd._EmbedIO, **but(f, **bad)))[0] == 1, bad
b = dict(rows=50, tokens=P, dy=P, dweight=P, dy_stride=8, dweight_stride=8, scale=1.0, index=1)
assert call("gd_embed_backward", e, io(gd._EmbedGrad, **b)) == (0, 1)
assert call("gd_embed_backward", e, io(gd._EmbedGrad, **but(b, rows=0, tokens=None, dy=None))) == (0, 1)  # zeros
assert call("gd_embed_backward", e, io(gd._EmbedGrad, **but(b, rows=0, accumulate=1))) == (0, 0)
for bad in (dict(rows=51), dict(tokens=None), dict(dy=None), dict(dweight=None), dict(dy_stride=7), dict(dweight_stride=7),
            dict(scale=nan), dict(index=5)):
    assert call("gd_embed_backward", e, io(gd._EmbedGrad, **but(b, **bad)))[0] == 1, bad
assert G.gd_embed_forward(None, io(gd._EmbedIO), None) == 1 and G.gd_embed_backward(e, None, None) == 1
frees = get("g_frees"); G.gd_embed_destroy(e); assert get("g_frees") == frees + 3
G.gd_embed_destroy(None)
""", tmp_path)


def test_units_of_the_embedding_fit_the_scratch():
    """No number of rows makes more units than a plan of this many rows or more has room for."""
    for slices in (1, 2, 3, 5, 8, 33, 100, 767, 768, 1000, 4096):
        def units(rows):
            return -(-rows // next((u for u in (32, 16) if -(-rows // u) * slices >= 768), 8))
        most = 0
        for rows in [*range(1, 3000), *range(3000, 60_000, 37), 2**24 - 1, 2**24]:
            most = max(most, units(rows))
            assert most <= max(min(-(-rows // 8), 1536 // slices), -(-rows // 32)), (slices, rows)


def test_gated_layer(tmp_path):
    run("""
refused("gd_gated_create", (0, 4, 1, 0, 1), (4, 0, 1, 0, 1), (2**22 + 1, 4, 1, 0, 1), (4, 2**21 + 1, 1, 0, 1), (4, 4, 3, 0, 1), (4, 4, 1, 4, 1),
        (4, 4, 1, -1, 1), (4, 4, 1, 0, 2**31))
for ty in (0, 1, 2):
    for k, n in ((64, 24), (65, 23), (4096, 2048), (4095, 5)):
        l = made("gated", k, n, ty, 3, 2**31 - 1)
        for rows in (1, 16, 17, 100, 5000, 2**20):
            f = dict(rows=rows, x=P, weight=P, y=P, pre=P, x_stride=k, weight_stride=k, y_stride=n, pre_stride=2 * n)
            st, launches = call("gd_gated_forward", l, io(gd._GatedIO, **f))
            assert st == 0 and 1 <= launches <= 4, (ty, k, n, rows, launches)
            assert Dim.in_dll(S, "g_grid").x < 2**22
            b = dict(rows=rows, dy=P, x=P, weight=P, pre=P, dz=P, dx=P, dweight=P, dbias=P, dy_stride=n, x_stride=k, weight_stride=k,
                     pre_stride=2 * n, dz_stride=2 * n, dx_stride=k, dweight_stride=k)
            st, launches = call("gd_gated_backward", l, io(gd._GatedGrad, **b))
            assert st == 0 and 2 <= launches <= 10, (ty, k, n, rows, launches)
        G.gd_gated_destroy(l)
l = made("gated", 64, 24, 1, 1, 100)
f = dict(rows=20, x=P, weight=P, y=P, x_stride=64, weight_stride=64, y_stride=24)
assert call("gd_gated_forward", l, io(gd._GatedIO, **f))[0] == 0
assert call("gd_gated_forward", l, io(gd._GatedIO, **but(f, rows=0, x=None, y=None))) == (0, 0)
for bad in (dict(rows=101), dict(x=None), dict(weight=None), dict(y=None), dict(x_stride=63), dict(weight_stride=0), dict(y_stride=23),
            dict(x_stride=2**22 + 1), dict(x_scale=P), dict(weight_scale=P), dict(pre=P, pre_stride=47)):
    assert call("gd_gated_forward", l, io(gd._GatedIO, **but(f, **bad)))[0] == 1, bad
assert call("gd_gated_forward", l, io(gd._GatedIO, **but(f, x_scale=P, weight_scale=P)))[0] == 0
b = dict(rows=20, dy=P, x=P, weight=P, pre=P, dz=P, dx=P, dweight=P, dbias=P, dy_stride=24, x_stride=64, weight_stride=64,
         pre_stride=48, dz_stride=48, dx_stride=64, dweight_stride=64)
assert call("gd_gated_backward", l, io(gd._GatedGrad, **b))[0] == 0
for bad in (dict(rows=101), dict(dy=None), dict(x=None), dict(weight=None), dict(pre=None), dict(dz=None), dict(dy_stride=23), dict(x_stride=1),
            dict(weight_stride=63), dict(pre_stride=47), dict(dz_stride=47), dict(dx_stride=63), dict(dweight_stride=63)):
    assert call("gd_gated_backward", l, io(gd._GatedGrad, **but(b, **bad)))[0] == 1, bad
assert call("gd_gated_backward", l, io(gd._GatedGrad, **but(b, rows=0, accumulate=1))) == (0, 0)
assert call("gd_gated_backward", l, io(gd._GatedGrad, **but(b, rows=0)))[0] == 0  # zeros
# as many results as a dispatch holds tiles of, and one tile more
wide = made("gated", 8, 2**21, 1, 0, 2**31 - 1)
g = dict(rows=(2**24 // 2**15 - 1) * 128, x=P, weight=P, y=P, x_stride=8, weight_stride=8, y_stride=2**21)
assert call("gd_gated_forward", wide, io(gd._GatedIO, **g))[0] == 0
assert call("gd_gated_forward", wide, io(gd._GatedIO, **but(g, rows=g["rows"] + 129))) == (2, 0)
long = made("gated", 131073, 8, 1, 0, 4)
g = dict(rows=2, x=P, weight=P, y=P, x_scale=P, weight_scale=P, x_stride=131073, weight_stride=131073, y_stride=8)
assert call("gd_gated_forward", long, io(gd._GatedIO, **g)) == (2, 0)
assert G.gd_gated_forward(None, io(gd._GatedIO, **f), None) == 1 and G.gd_gated_backward(l, None, None) == 1
G.gd_gated_destroy(None)
""", tmp_path)


def test_scores(tmp_path):
    run("""
for what in ("logprob", "distill"):
    refused(f"gd_{what}_create", (0, 1, 4), (2**31, 1, 4), (8, 3, 4), (8, -1, 4), (8, 1, 2**31))
V = 9000
l, d = made("logprob", V, 1, 2**31 - 1), made("distill", V, 1, 2**31 - 1)
f = dict(rows=300, logits=P, tokens=P, logp=P, stride=V, scale=1.0, index=1)
g = dict(rows=300, logits=P, tokens=P, dlogp=P, dlogits=P, stride=V, dlogits_stride=V, scale=1.0, index=0)
t = dict(rows=300, logits=P, ids=P, teacher=P, loss=P, stride=V, ids_stride=7, teacher_stride=7, scale=1.0, top=7, index=1, teacher_type=2)
u = dict(rows=300, logits=P, ids=P, teacher=P, dloss=P, dlogits=P, stride=V, ids_stride=7, teacher_stride=7, dlogits_stride=V, scale=1.0, top=7,
         index=0, teacher_type=0)
calls = (("gd_logprob_forward", l, gd._LogProbIO, f, 2), ("gd_logprob_backward", l, gd._LogProbGrad, g, 3), ("gd_distill_forward", d, gd._DistillIO, t, 2),
         ("gd_distill_backward", d, gd._DistillGrad, u, 3))
for name, hd, kind, ok, few in calls:
    assert call(name, hd, io(kind, **ok)) == (0, 1)
    assert call(name, hd, io(kind, **but(ok, rows=0, logits=None))) == (0, 0)
    for rows in (1, 2, 100, 255):  # in pieces: their sums, joined, and the gradient behind them
        assert call(name, hd, io(kind, **but(ok, rows=rows))) == (0, few), (name, rows)
    assert call(name, hd, io(kind, **but(ok, rows=2**22 + 1))) == (0, 2)  # a launch holds 2^22 rows
    assert Dim.in_dll(S, "g_grid").x == 1
    assert call(name, hd, io(kind, **but(ok, rows=2**31 - 1)))[0] == 0
    for bad in (dict(logits=None), dict(stride=V - 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=inf), dict(scale=nan), dict(index=2), dict(index=-1)):
        assert call(name, hd, io(kind, **but(ok, **bad)))[0] == 1, (name, bad)
    assert getattr(G, name)(None, io(kind, **ok), None) == 1 and getattr(G, name)(hd, None, None) == 1
for bad in (dict(tokens=None), dict(top=1), dict(top=1, top_logp=P), dict(top=65, top_logp=P, top_id=P)):
    assert call("gd_logprob_forward", l, io(gd._LogProbIO, **but(f, **bad)))[0] == 1, bad
for rows, launches in ((300, 1), (1, 2)):
    assert call("gd_logprob_forward", l, io(gd._LogProbIO, **but(f, rows=rows, top=64, top_logp=P, top_id=P, entropy=P, stats=P))) == (0, launches)
for bad in (dict(tokens=None), dict(dlogp=None), dict(dlogits=None), dict(dlogits_stride=V - 1), dict(stats=P, logp_out=P), dict(stats=P, entropy_out=P),
            dict(stats=P, dentropy=P)):
    assert call("gd_logprob_backward", l, io(gd._LogProbGrad, **but(g, **bad)))[0] == 1, bad
assert call("gd_logprob_backward", l, io(gd._LogProbGrad, **but(g, rows=1, stats=P, dentropy=P, entropy=P))) == (0, 1)
for bad in (dict(ids=None), dict(teacher=None), dict(top=0), dict(top=257, ids_stride=300, teacher_stride=300), dict(ids_stride=6), dict(teacher_stride=6),
            dict(teacher_type=3)):
    assert call("gd_distill_forward", d, io(gd._DistillIO, **but(t, **bad)))[0] == 1, bad
    assert call("gd_distill_backward", d, io(gd._DistillGrad, **but(u, **bad)))[0] == 1, bad
for bad in (dict(dloss=None), dict(dlogits=None), dict(dlogits_stride=V - 1), dict(stats=P, loss_out=P)):
    assert call("gd_distill_backward", d, io(gd._DistillGrad, **but(u, **bad)))[0] == 1, bad
small = made("logprob", 5, 0, 10)
assert call("gd_logprob_forward", small, io(gd._LogProbIO, **but(f, rows=11, stride=5)))[0] == 1
assert call("gd_logprob_forward", small, io(gd._LogProbIO, **but(f, rows=10, stride=5, top=6, top_logp=P, top_id=P)))[0] == 1
assert call("gd_logprob_forward", small, io(gd._LogProbIO, **but(f, rows=10, stride=5, top=5, top_logp=P, top_id=P))) == (0, 1)
for what, hd in (("logprob", l), ("distill", d), ("logprob", small)):
    frees = get("g_frees"); getattr(G, f"gd_{what}_destroy")(hd); assert get("g_frees") > frees
    getattr(G, f"gd_{what}_destroy")(None)
""", tmp_path)


def test_pieces_cover_a_row_and_fit_the_scratch(tmp_path):
    """The kernel's own numbers of rows in pieces: every element in one, no more pieces than a wave joins, than the scratch
    holds or than the list of alternatives has room for."""
    launch_stub.run("""
import struct
for vocab in (8191, 8192, 8193, 9001, 20000, 32001, 85000, 100003, 2**20 + 5, 2**31 - 1):
    for rows in (1, 2, 3, 5, 16, 63, 64, 100, 255, 256):
        for top in (0, 1, 8, 64):
            l = made("logprob", vocab, 1, 300)
            f = dict(rows=rows, logits=P, tokens=P, logp=P, top_logp=P, top_id=P, stride=vocab, scale=1.0, index=1, top=top)
            log = launches(lambda: G.gd_logprob_forward(l, io(gd._LogProbIO, **f), None))
            blocks, name = log[0]["grid"][0], log[0]["what"]
            waves = int(re.search(r"Li(\\d+)ELi\\dELb0E", name)[1])
            a_block = 4 if waves == 1 else 1
            units = blocks * a_block
            assert (len(log) == 2) == (rows < 256 and vocab >= 8192), (vocab, rows, top)
            if len(log) == 1:
                assert rows <= units < rows + a_block
                continue
            assert log[1]["name"] == "k_score_join" and log[1]["grid"] == (rows, 1)
            pieces = units // rows if a_block == 1 else None
            if pieces:
                assert pieces * rows == units <= 512 and pieces <= 64 and pieces * top <= 1024 and pieces * 4096 <= vocab + 8 * pieces
            G.gd_logprob_destroy(l)
""", tmp_path)


def test_out_of_memory_is_an_error_and_leaks_nothing(tmp_path):
    run("""
put("g_other_capture", 1)  # the stub then refuses allocations
before = get("g_allocs"), get("g_frees")
assert G.gd_layernorm_create(ctypes.byref(h), 8, 1) == 5 and G.gd_embed_create(ctypes.byref(h), 8, 8, 1, 8) == 5
assert G.gd_gated_create(ctypes.byref(h), 8, 8, 1, 0, 8) == 5 and G.gd_logprob_create(ctypes.byref(h), 8, 1, 8) == 5
assert G.gd_distill_create(ctypes.byref(h), 8, 1, 8) == 5
assert h.value is None and get("g_allocs") - before[0] == get("g_frees") - before[1]
""", tmp_path)
