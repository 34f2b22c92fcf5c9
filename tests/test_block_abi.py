"""C ABI of the block operators without a GPU: every declared function is there, and
wrong arguments come back as a status before anything is launched."""

import ctypes

import pytest

import paper_2410_17243_amd as infcl
from paper_2410_17243_amd import block
from paper_2410_17243_amd.tower import _View

A = 1 << 20  # an aligned address that no call below reaches
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return block._load()


def test_exports_every_declared_function(lib):
    names = infcl.header_functions(infcl.BLOCK_HEADER_PATH)
    assert len(names) == 15
    for n in names:
        assert hasattr(lib, n), n


ROTARY = dict(n=5, heads=4, turned=3, hd=64, dt=0, paired=0, back=0, axes=2, pdt=0, sections=(8, 24), ps=2)


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(heads=0), INVALID), (dict(turned=5), INVALID), (dict(turned=-1), INVALID), (dict(hd=0), INVALID),
    (dict(dt=3), INVALID), (dict(paired=2), INVALID), (dict(back=2), INVALID), (dict(axes=0), INVALID), (dict(axes=5), INVALID),
    (dict(axes=3), INVALID), (dict(pdt=2), INVALID), (dict(ps=-1), INVALID), (dict(sections=(8, 25)), INVALID),
    (dict(sections=(1 << 30, 1 << 30)), INVALID), (dict(hd=68), UNSUPPORTED), (dict(hd=1032), UNSUPPORTED), (dict(heads=4097), UNSUPPORTED),
    (dict(n=(1 << 31) + 1), UNSUPPORTED), (dict(n=0, x=None, out=None, pos=None, freqs=None), OK), (dict(x=None), INVALID),
    (dict(x=(A + 8, 256, 64)), INVALID), (dict(x=(A, 32, 64)), INVALID), (dict(out=(A, 256, 64)), INVALID),
    (dict(x=(A, 260, 64)), UNSUPPORTED), (dict(x=(A, 256, 4)), UNSUPPORTED), (dict(pos=None), INVALID), (dict(pos=A + 2), INVALID),
    (dict(freqs=A + 1), INVALID), (dict(n=1 << 27, heads=4096), UNSUPPORTED),  # more workgroups than a launch has
])
def test_rotary(lib, kw, want):
    a = ROTARY | dict(x=(A, 256, 64), out=(2 * A, 256, 64), pos=A, freqs=A) | kw
    s = block._Rotary(a["n"], a["heads"], a["turned"], a["hd"], a["dt"], a["paired"], a["back"], a["axes"], a["pdt"],
                      (ctypes.c_int32 * 4)(*a["sections"]), a["ps"])
    view = [_View(*(a[k] or (None, 256, 64))) for k in ("x", "out")]
    assert lib.infcl_rotary(ctypes.byref(s), *view, a["pos"], a["freqs"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(d=0), INVALID), (dict(dt=7), INVALID), (dict(stride=8), INVALID), (dict(x=None), INVALID),
    (dict(out=A + 8), INVALID), (dict(drop=(None, 0, 0, 0, 1.1)), INVALID), (dict(drop=(None, 0, 0, 0, float("nan"))), INVALID),
    (dict(drop=(None, 0, -1, 0, 0.1)), INVALID), (dict(drop=(A + 4, 0, 0, 0, 0.1)), INVALID), (dict(d=12), UNSUPPORTED),
    (dict(stride=20), UNSUPPORTED), (dict(n=1 << 40), UNSUPPORTED), (dict(drop=(None, 0, 1 << 61, 0, 0.1)), UNSUPPORTED),
    (dict(n=0, x=None, out=None), OK),
])
def test_dropout(lib, kw, want):
    a = dict(x=A, stride=16, n=3, d=16, dt=0, drop=(None, 0, 0, 0, 0.1), out=A) | kw
    assert lib.infcl_dropout(a["x"], a["stride"], a["n"], a["d"], a["dt"], block._Drop(*a["drop"]), a["out"], None) == want


def _norm(kw):
    a = dict(n=3, d=16, dt=0, wdt=0, norm=0, eps=1e-5, alpha=1.0, drop=(None, 0, 0, 0, 0.0), xs=16, ys=16, gate=A, post_w=A,
             post_b=A, pre_w=A, pre_b=A) | kw
    a["drop"] = block._Drop(*a["drop"])
    return block._AddNorm(*a.values())


NORMS = [
    (dict(n=-1), {}, INVALID), (dict(dt=5), {}, INVALID), (dict(wdt=4), {}, INVALID), (dict(norm=2), {}, INVALID),
    (dict(eps=-1.0), {}, INVALID), (dict(eps=float("nan")), {}, INVALID), (dict(alpha=float("inf")), {}, INVALID),
    (dict(post_w=None), {}, INVALID), (dict(pre_w=None), {}, INVALID), (dict(gate=A + 8), {}, INVALID), (dict(xs=8), {}, INVALID),
    (dict(ys=8), {}, INVALID), (dict(d=12), {}, UNSUPPORTED), (dict(d=8200, xs=8200, ys=8200), {}, UNSUPPORTED), (dict(wdt=2), {}, UNSUPPORTED),
    (dict(xs=20), {}, UNSUPPORTED), (dict(ys=20), {}, UNSUPPORTED), ({}, dict(x=None), INVALID), ({}, dict(y=None), INVALID),
    ({}, dict(y=A + 2), INVALID), (dict(gate=None, post_w=None, post_b=None, alpha=0.5), dict(y=None), INVALID),
    (dict(gate=None, post_w=None, post_b=None, drop=(None, 0, 0, 0, 0.5)), dict(y=None), INVALID),
    (dict(n=0), dict(x=None, y=None, h=None, z=None, stats=None), OK),
]


@pytest.mark.parametrize("kw,rows,want", NORMS + [({}, dict(h=None), INVALID), ({}, dict(z=A + 4), INVALID), ({}, dict(stats=A + 4), INVALID)])
def test_add_norm_forward(lib, kw, rows, want):
    r = dict(x=A, y=A, h=A, z=A, stats=None) | rows
    assert lib.infcl_add_norm_fwd(ctypes.byref(_norm(kw)), r["x"], r["y"], r["h"], r["z"], r["stats"], None) == want


@pytest.mark.parametrize("kw,rows,want", [n for n in NORMS if n[2] != OK] + [
    ({}, dict(stats=None), INVALID), ({}, dict(ws=A + 16), INVALID), ({}, dict(n=64), WORKSPACE), ({}, dict(dh=A + 2), INVALID),
    ({}, dict(dhs=8), INVALID), ({}, dict(dzs=20), UNSUPPORTED), (dict(gate=None), {}, INVALID), (dict(post_b=None), {}, INVALID),
    (dict(pre_w=None, pre_b=None), {}, INVALID),
])
def test_add_norm_backward(lib, kw, rows, want):
    r = dict(x=A, y=A, stats=A, dh=A, dz=A, dhs=16, dzs=16, ws=A, n=BIG) | rows
    g = block._AddNormGrads(r["dh"], r["dz"], r["dhs"], r["dzs"], A, A, A, A, A, A, A)
    assert lib.infcl_add_norm_bwd(ctypes.byref(_norm(kw)), r["x"], r["y"], r["stats"], ctypes.byref(g), r["ws"], r["n"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(dt=4), INVALID), (dict(stride=8), INVALID), (dict(e=None), INVALID), (dict(qt=None), INVALID),
    (dict(q=None, e=None, qt=None, et=None, cs=None), INVALID), (dict(x=A + 8), INVALID), (dict(q=A + 8), INVALID), (dict(ws=None), INVALID),
    (dict(wsb=32), WORKSPACE), (dict(d=12), UNSUPPORTED), (dict(stride=20), UNSUPPORTED), (dict(n=(1 << 27) + 1), UNSUPPORTED),
    (dict(n=0, x=None, q=None, e=None, cs=None), OK),
])
def test_fp8_pack(lib, kw, want):
    a = dict(x=A, stride=16, n=3, d=16, dt=0, q=A, e=A, qt=A, et=A, cs=A, ws=A, wsb=BIG) | kw
    assert lib.infcl_fp8_pack(a["x"], a["stride"], a["n"], a["d"], a["dt"], a["q"], a["e"], a["qt"], a["et"], a["cs"], a["ws"],
                              a["wsb"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), INVALID), (dict(dt=9), INVALID), (dict(q=A + 4), INVALID), (dict(out=None), INVALID), (dict(rows=0, q=None, out=None), OK),
    (dict(rows=1 << 28), UNSUPPORTED),
])
def test_fp8_unpack(lib, kw, want):
    a = dict(q=A, e=A, rows=3, k=5, dt=0, out=A) | kw
    assert lib.infcl_fp8_unpack(a["q"], a["e"], a["rows"], a["k"], a["dt"], a["out"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(m=0), INVALID), (dict(k=-1), INVALID), (dict(dt=8), INVALID), (dict(dt=1), UNSUPPORTED),
    (dict(k=(1 << 23) + 1), UNSUPPORTED), (dict(n=1 << 28), UNSUPPORTED), (dict(n=1 << 26, m=1 << 20), UNSUPPORTED), (dict(a=A + 8), INVALID),
    (dict(be=None), INVALID), (dict(out=A + 2), INVALID), (dict(bias=A + 2), INVALID), (dict(m=(1 << 24) + 1), UNSUPPORTED), (dict(ws=None), INVALID), (dict(wsb=0), WORKSPACE),
    (dict(n=0, a=None, ae=None, out=None), OK),
])
def test_fp8_matmul(lib, kw, want):
    a = dict(a=A, ae=A, n=3, b=A, be=A, m=8, k=4096, bias=None, dt=0, out=A, ws=A, wsb=BIG) | kw
    assert lib.infcl_fp8_matmul(a["a"], a["ae"], a["n"], a["b"], a["be"], a["m"], a["k"], a["bias"], a["dt"], a["out"], a["ws"],
                                a["wsb"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(k=0, stride=8), INVALID), (dict(stride=8), INVALID), (dict(dt=1), UNSUPPORTED), (dict(k=4092), UNSUPPORTED),
    (dict(stride=4100), UNSUPPORTED), (dict(x=A + 8), INVALID), (dict(w=None), INVALID), (dict(we=None), INVALID), (dict(out=None), INVALID),
    (dict(ws=A + 16), INVALID), (dict(wsb=4096), WORKSPACE), (dict(n=0, x=None, out=None), OK),
])
def test_fp8_linear(lib, kw, want):
    a = dict(x=A, stride=4096, n=40, k=4096, w=A, we=A, m=8, bias=None, dt=0, out=A, ws=A, wsb=BIG) | kw
    assert lib.infcl_fp8_linear(a["x"], a["stride"], a["n"], a["k"], a["w"], a["we"], a["m"], a["bias"], a["dt"], a["out"], a["ws"],
                                a["wsb"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(k=0), INVALID), (dict(keeps=4), INVALID), (dict(dt=9), INVALID), (dict(xs=8), INVALID), (dict(ws=8), INVALID),
    (dict(x=A + 2), INVALID), (dict(w=None), INVALID), (dict(b=A + 2), INVALID), (dict(kept=None), INVALID), (dict(space=A + 16), INVALID),
    (dict(out=A + 8), INVALID), (dict(bytes=256), WORKSPACE), (dict(k=12), UNSUPPORTED), (dict(m=12), UNSUPPORTED), (dict(dt=1), UNSUPPORTED),
    (dict(xs=20), UNSUPPORTED), (dict(ws=20), UNSUPPORTED), (dict(n=(1 << 23) + 1), UNSUPPORTED),
])
def test_fp8_layer_forward(lib, kw, want):
    a = dict(x=A, xs=16, n=3, k=16, w=A, ws=16, m=8, b=A, dt=0, keeps=3, out=A, kept=A, space=A, bytes=BIG) | kw
    assert lib.infcl_fp8_layer_fwd(a["x"], a["xs"], a["n"], a["k"], a["w"], a["ws"], a["m"], a["b"], a["dt"], a["keeps"], a["out"],
                                   a["kept"], a["space"], a["bytes"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), INVALID), (dict(keeps=-1), INVALID), (dict(dys=4), INVALID), (dict(keeps=1), INVALID), (dict(keeps=2), INVALID),
    (dict(dy=A + 2), INVALID), (dict(dx=A + 2), INVALID), (dict(dw=A + 2), INVALID), (dict(db=A + 2), INVALID), (dict(kept=None), INVALID),
    (dict(space=None), INVALID), (dict(bytes=256), WORKSPACE), (dict(dt=1), UNSUPPORTED), (dict(dys=12), UNSUPPORTED),
    (dict(dx=None, dw=None, db=None, dy=None), OK),
])
def test_fp8_layer_backward(lib, kw, want):
    a = dict(dy=A, dys=8, n=3, k=16, m=8, dt=0, keeps=3, kept=A, dx=A, dw=A, db=A, space=A, bytes=BIG) | kw
    assert lib.infcl_fp8_layer_bwd(a["dy"], a["dys"], a["n"], a["k"], a["m"], a["dt"], a["keeps"], a["kept"], a["dx"], a["dw"], a["db"],
                                   a["space"], a["bytes"], None) == want


@pytest.mark.parametrize("n,k,m,keeps,want", [
    (1 << 27, 8, 8, 0, OK), ((1 << 27) + 1, 8, 8, 0, UNSUPPORTED), (1 << 26, 8, 64, 1, OK), (1 << 23, 8, 8, 3, OK),
    ((1 << 23) + 1, 8, 8, 2, UNSUPPORTED), ((1 << 23) + 1, 8, 8, 3, UNSUPPORTED), (8, 8, 1 << 23, 3, OK), (8, 8, (1 << 23) + 8, 0, UNSUPPORTED),
    (8, 1 << 23, 8, 3, OK), (8, (1 << 23) + 8, 8, 0, UNSUPPORTED), (1 << 27, 8, 2048, 0, UNSUPPORTED),
])
def test_fp8_layer_sizes(lib, n, k, m, keeps, want):
    """The limits are those of the products that there are; what is not kept for has no room."""
    sizes = [ctypes.c_size_t(0) for _ in range(3)]
    assert lib.infcl_fp8_layer_sizes(n, k, m, keeps, *(ctypes.byref(s) for s in sizes)) == want
    if want == OK:
        sums = ctypes.c_size_t(0)
        assert lib.infcl_fp8_pack_workspace(n, m, ctypes.byref(sums)) == OK
        assert (sizes[0].value > 0) == (keeps > 0) and sizes[1].value >= 128 * (n + m)
        assert sizes[2].value >= 128 * n + sums.value if keeps & 1 else keeps or sizes[2].value == sums.value


def test_workspaces(lib):
    def size(name, *a):
        n = ctypes.c_size_t(0)
        assert getattr(lib, name)(*a, ctypes.byref(n)) == OK
        assert getattr(lib, name)(*a, None) == INVALID
        return n.value
    assert size("infcl_fp8_pack_workspace", 1000, 64) == 8 * 64 * 4
    assert size("infcl_fp8_matmul_workspace", 1 << 16, 1 << 12, 1024) == 0  # tiles fill the chip
    assert size("infcl_fp8_matmul_workspace", 16, 16, 1 << 16) > 0          # one tile, a long contraction: parts
    assert size("infcl_fp8_linear_workspace", 16, 4096, 4096) == 0          # one launch
    assert size("infcl_fp8_linear_workspace", 17, 4096, 4096) >= 17 * (4096 + 32)
    n = ctypes.c_size_t(0)
    assert lib.infcl_add_norm_bwd_workspace(ctypes.byref(_norm({})), ctypes.byref(n)) == OK and n.value == 5 * 16 * 4 + 192
    assert lib.infcl_add_norm_bwd_workspace(ctypes.byref(_norm(dict(n=1 << 30))), ctypes.byref(n)) == OK and n.value < 1 << 20
    assert lib.infcl_add_norm_bwd_workspace(ctypes.byref(_norm({})), None) == INVALID
