"""C ABI of the text tower's operators without a GPU: every declared function is
there, and wrong arguments come back as a status before anything is launched."""

import ctypes

import pytest

import paper_2410_17243_amd as infcl
from paper_2410_17243_amd import tower

A = 1 << 20  # an aligned address that no call below reaches
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return tower._load()


def test_exports_every_declared_function(lib):
    names = infcl.header_functions(infcl.TOWER_HEADER_PATH)
    assert len(names) == 12
    for n in names:
        assert hasattr(lib, n), n


@pytest.mark.parametrize("kw,want", [
    (dict(tb=2), INVALID), (dict(n=-1), INVALID), (dict(vocab=0), INVALID), (dict(dt=3), INVALID), (dict(tok=None), INVALID),
    (dict(tok=A + 4), INVALID), (dict(table=A + 8), INVALID), (dict(out=None), INVALID), (dict(d=12), UNSUPPORTED),
    (dict(d=6, dt=1), UNSUPPORTED), (dict(n=1 << 31), UNSUPPORTED), (dict(n=0, tok=None, table=None, out=None), OK),
])
def test_embed_fwd(lib, kw, want):
    a = dict(tok=A, tb=8, n=5, table=A, vocab=9, d=16, dt=0, out=A) | kw
    assert lib.infcl_embed_fwd(a["tok"], a["tb"], a["n"], a["table"], a["vocab"], a["d"], a["dt"], 1.0, a["out"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(tb=0), INVALID), (dict(g=4), INVALID), (dict(g=2), UNSUPPORTED), (dict(dt=1, g=0), UNSUPPORTED),
    (dict(dout=A + 2), INVALID), (dict(dw=None), INVALID), (dict(ws=A + 16), INVALID), (dict(wsb=64), WORKSPACE),
    (dict(d=4), UNSUPPORTED), (dict(vocab=1 << 31), UNSUPPORTED),
])
def test_embed_bwd(lib, kw, want):
    a = dict(tok=A, tb=4, n=5, dout=A, vocab=9, d=16, dt=0, dw=A, g=1, ws=A, wsb=BIG) | kw
    assert lib.infcl_embed_bwd(a["tok"], a["tb"], a["n"], a["dout"], a["vocab"], a["d"], a["dt"], 1.0, a["dw"], a["g"],
                               a["ws"], a["wsb"], None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), INVALID), (dict(stride=8), INVALID), (dict(stride=20), UNSUPPORTED), (dict(d=12, stride=16), UNSUPPORTED),
    (dict(q=A + 8), INVALID), (dict(e=None), INVALID), (dict(dt=9), INVALID), (dict(n=0, x=None, q=None, e=None), OK),
])
def test_ckpt8_pack(lib, kw, want):
    a = dict(x=A, stride=16, n=3, d=16, dt=0, q=A, e=A) | kw
    assert lib.infcl_ckpt8_pack(a["x"], a["stride"], a["n"], a["d"], a["dt"], a["q"], a["e"], None) == want


@pytest.mark.parametrize("act,want", [(0, INVALID), (3, INVALID), (-1, INVALID)])
def test_activations(lib, act, want):
    assert lib.infcl_ckpt8_act_fwd(A, 16, 3, 16, 0, act, A, A, A, None) == want
    assert lib.infcl_ckpt8_act_bwd(A, 16, A, A, 3, 16, 0, act, A, None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dt=1), UNSUPPORTED), (dict(g=2), UNSUPPORTED), (dict(g=7), INVALID), (dict(act=5), INVALID), (dict(m=12), INVALID),
    (dict(m=12, stride=16), UNSUPPORTED), (dict(dw=A + 4), INVALID), (dict(wsb=16), WORKSPACE), (dict(ws=None), INVALID),
    (dict(stride=1 << 25), UNSUPPORTED),
])
def test_ckpt8_wgrad(lib, kw, want):
    a = dict(dy=A, stride=8, q=A, e=A, n=3, d=16, m=8, dt=0, act=0, dw=A, g=1, ws=A, wsb=BIG) | kw
    assert lib.infcl_ckpt8_wgrad(a["dy"], a["stride"], a["q"], a["e"], a["n"], a["d"], a["m"], a["dt"], a["act"], a["dw"],
                                 a["g"], a["ws"], a["wsb"], None) == want


SHAPE = dict(tq=20, tk=30, nseq=2, heads=4, kv=2, hd=64, dt=0, causal=1, mq=9, mk=9, scale=0.125)


def _shape(kw):
    return tower._Shape(*(SHAPE | kw).values())


@pytest.mark.parametrize("kw,want", [
    (dict(heads=3), INVALID), (dict(kv=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(causal=2), INVALID), (dict(dt=5), INVALID), (dict(mq=-1), INVALID), (dict(tq=-1), INVALID), (dict(dt=1), UNSUPPORTED),
    (dict(hd=12), UNSUPPORTED), (dict(hd=136), UNSUPPORTED), (dict(tk=1 << 31), UNSUPPORTED), ({}, OK), (dict(nseq=0), OK),
])
def test_attn_shapes(lib, kw, want):
    f, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.infcl_attn_workspace(ctypes.byref(_shape(kw)), ctypes.byref(f), ctypes.byref(b)) == want
    assert lib.infcl_attn_workspace(ctypes.byref(_shape(kw)), None, None) == (want if want != OK else INVALID)


@pytest.mark.parametrize("bad,want", [
    (dict(q=(None, 256, 64)), INVALID), (dict(q=(A + 8, 256, 64)), INVALID), (dict(k=(A, 32, 64)), INVALID),
    (dict(v=(A, 260, 64)), UNSUPPORTED), (dict(out=(A, 1 << 24, 64)), UNSUPPORTED), (dict(cu_q=None), INVALID),
    (dict(len_k=A + 2), INVALID),
])
def test_attn_views(lib, bad, want):
    a = dict(q=(A, 256, 64), k=(A, 128, 64), v=(A, 128, 64), cu_q=A, cu_k=A, len_k=None, out=(A, 256, 64)) | bad
    view = {n: tower._View(*a[n]) for n in ("q", "k", "v", "out")}
    assert lib.infcl_attn_fwd(ctypes.byref(_shape({})), view["q"], view["k"], view["v"], a["cu_q"], a["cu_k"], a["len_k"],
                              view["out"], None, A, BIG, None) == want


def test_attn_backward_wants_its_workspace_and_lse(lib):
    q, k = tower._View(A, 256, 64), tower._View(A, 128, 64)
    call = lambda lse, n: lib.infcl_attn_bwd(ctypes.byref(_shape({})), q, k, k, A, A, q, lse, q, q, k, k, A, n, None)  # noqa: E731
    assert call(None, BIG) == INVALID and call(A, 16) == WORKSPACE


def test_workspaces_are_what_the_parts_need(lib):
    """Few queries over many keys: fp32 sums and two statistics a row and part;
    sequences that fill the chip: none."""
    def fwd(**kw):
        f = ctypes.c_size_t(0)
        assert lib.infcl_attn_workspace(ctypes.byref(_shape(kw)), ctypes.byref(f), None) == OK
        return f.value
    one = fwd(tq=1, tk=100000, nseq=1, mq=1, mk=100000)
    assert one % 256 == 0 and 0 < one <= 2048 * 4 * (64 + 2) * 4 + 512
    assert fwd(tq=1 << 20, tk=1 << 20, nseq=8192, mq=128, mk=128) == 0


def test_token_counts_that_the_sort_would_take_too_long_for(lib):
    n = ctypes.c_size_t(0)
    assert lib.infcl_embed_bwd_workspace(1 << 26, 100, 8, ctypes.byref(n)) == OK
    assert lib.infcl_embed_bwd_workspace((1 << 26) + 1, 100, 8, ctypes.byref(n)) == UNSUPPORTED


@pytest.mark.parametrize("kw,want", [
    # a launch has at most 2^32 - 1 work-items: 64 for each sequence (and the rows past them) and key head
    (dict(nseq=(1 << 25) // 16 * 2 - 1, heads=16, kv=16), UNSUPPORTED), (dict(nseq=(1 << 25) // 16 * 2 - 2, heads=16, kv=16), OK),
    (dict(nseq=1 << 14, heads=4096, kv=4096), UNSUPPORTED), (dict(nseq=(1 << 14) - 2, heads=4096, kv=4096), OK),
    # many short sequences and a long one: no more tiles at once than that, not a refusal
    (dict(nseq=1 << 20, tq=1 << 24, tk=1 << 24, mq=1 << 20, mk=1 << 20, heads=16, kv=16), OK),
])
def test_launches_stay_within_the_work_items_there_are(lib, kw, want):
    f, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.infcl_attn_workspace(ctypes.byref(_shape(kw)), ctypes.byref(f), ctypes.byref(b)) == want
