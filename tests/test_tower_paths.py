"""Every form that the host's plans choose between, reached by sizes that the plans
are asked about first: attention's backward sweeps in parts, many pairs of sequence
and key head with several tiles each, lengths longer than said in the split forms,
and the weight gradient's large tiles."""

import ctypes

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import tower
from paper_2410_17243_amd import tower as binding

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # one rounding to nearest
F32 = 2.0 ** -15  # (scores off by less than 2^-17, exponentials and sums of fp32)
TINY = {"bf16": 1e-30, "f16": 2.0 ** -25}


def _up(x):
    return (x + 255) // 256 * 256


def _cu(lens):
    return [0] + torch.tensor(lens).cumsum(0).tolist()


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda") if isinstance(x, list) else x.cuda()


# lengths of queries, of keys, heads, kv heads, head_dim, said lengths (q, k), parts of
# the backward sweeps over queries and over keys
SPLIT = [
    ([520, 300], [520, 300], 4, 1, 80, (520, 520), (4, 2)),
    ([520, 300], [520, 300], 4, 1, 128, (520, 520), (4, 2)),
    ([1100, 0, 400], [1100, 0, 400], 4, 2, 64, (1100, 1100), (4, 4)),
    ([700], [700], 3, 3, 40, (700, 700), (1, 2)),
    ([600, 40], [300, 900], 6, 2, 64, (600, 900), (3, 3)),
    ([900, 700], [900, 700], 4, 1, 72, (520, 520), (4, 2)),       # longer than said
    ([90, 60], [1500, 1400], 8, 8, 128, (90, 1500), (1, 5)),      # a prefix: few queries, many keys
]


@pytest.mark.parametrize("lens_q,lens_k,heads,kv,hd,said,parts", SPLIT)
def test_the_split_cases_are_cut_as_they_say(lens_q, lens_k, heads, kv, hd, said, parts):
    tq, tk = sum(lens_q), sum(lens_k)
    b = ctypes.c_size_t(0)
    shape = binding._Shape(tq, tk, len(lens_q), heads, kv, hd, infcl.INFCL_F16, 1, *said, hd ** -0.5)
    assert binding._load().infcl_attn_workspace(ctypes.byref(shape), None, ctypes.byref(b)) == 0
    dkv, dq = (2 * parts[0] * tk * kv * hd * 4 if parts[0] > 1 else 0), (parts[1] * tq * heads * hd * 4 if parts[1] > 1 else 0)
    assert b.value == _up(_up(2 * ((tq + 95) // 64 * 64) * heads * 4) + max(dkv, dq))


def _attention(lens_q, lens_k, heads, kv, hd, dtype, causal, said):
    cu_q, cu_k, e = _cu(lens_q), _cu(lens_k), EPS[dtype]
    g = torch.Generator().manual_seed(sum(lens_q) + hd)
    mk = lambda t, h: torch.randn((t, h, hd), generator=g).to(DT[dtype])  # noqa: E731
    q, k, v, do = mk(cu_q[-1], heads), mk(cu_k[-1], kv), mk(cu_k[-1], kv), mk(cu_q[-1], heads)
    r = tower.attention(q, k, v, cu_q, cu_k, causal, hd ** -0.5, do)
    a, off = [_dev(t) for t in (q, k, v)], (_dev(cu_q), said[0], _dev(cu_k), said[1])
    out, lse = infcl.packed_attn_fwd(*a, *off, causal=causal)
    grads = infcl.packed_attn_bwd(*a, out, lse, _dev(do), *off, causal=causal)
    for name, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        tol = (e + F32) * r[name + "_abs"] + e * r[name].abs() + TINY[dtype]
        if name in ("dq", "dk"):  # (D comes from out as rounded)
            tol = tol + (e + F32) * r[name + "_dlt"]
        got = got.cpu().double()
        assert torch.isfinite(got).all(), name
        assert ((got - r[name]).abs() <= tol).all(), (name, float(((got - r[name]).abs() - tol).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens_q,lens_k,heads,kv,hd,said,parts", SPLIT)
def test_backward_in_parts(lens_q, lens_k, heads, kv, hd, said, parts, causal, dtype):
    _attention(lens_q, lens_k, heads, kv, hd, dtype, causal, said)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("most,n,heads,kv,hd,dtype", [(300, 20, 4, 4, 64, "bf16"), (300, 20, 8, 4, 128, "f16"),
                                                     (100, 23, 4, 4, 64, "f16"), (120, 33, 2, 2, 80, "bf16")])
def test_many_pairs_with_several_tiles_each(most, n, heads, kv, hd, dtype, causal):
    """64 pairs of sequence and key head or more (84, 84, 96 and 68 with the rows past
    the last one): their order of tiles is another, with pairs that eight do not divide."""
    lens = torch.randint(most // 3, most + 1, (n,), generator=torch.Generator().manual_seed(n)).tolist()
    lens[3] = most
    _attention(lens, lens, heads, kv, hd, dtype, causal, (most, most))


# n, d, m, type, activation, gradient's type, parts of the tokens
LARGE = [
    (43713, 264, 520, "bf16", "none", "f32", 42), (43713, 264, 520, "f16", "gelu", "f16", 42),
    (1861, 3848, 2056, "bf16", "quick_gelu", "bf16", 1), (1861, 3848, 2056, "f16", "none", "f32", 1),
    (25001, 1000, 520, "bf16", "gelu", "bf16", 21),
]


@pytest.mark.parametrize("n,d,m,dtype,act,grad,parts", LARGE)
def test_the_large_tiles_are_reached(n, d, m, dtype, act, grad, parts):
    """Tiles of 256 x 256 from 8192 pairs of tile and stage of 32 tokens on; the parts
    are those of 256 workgroups (512 with the small tiles)."""
    tiles, stages = -(-m // 256) * -(-d // 256), -(-n // 32)
    assert tiles * stages >= 8192
    b = ctypes.c_size_t(0)
    assert binding._load().infcl_ckpt8_wgrad_workspace(n, d, m, ctypes.byref(b)) == 0
    assert b.value == _up(n * d * 2) + (_up(parts * m * d * 4) if parts > 1 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,m,dtype,act,grad,parts", LARGE)
def test_weight_gradient_with_large_tiles(n, d, m, dtype, act, grad, parts):
    g = torch.Generator().manual_seed(n + d)
    x, dy = torch.randn((n, d), generator=g).to(DT[dtype]), torch.randn((n, m), generator=g).to(DT[dtype])
    kept = infcl.ckpt8_pack(x.cuda())
    wide = torch.full((n, m + 16), float("nan"), dtype=DT[dtype])
    wide[:, 8:8 + m] = dy
    dw = infcl.ckpt8_wgrad(wide.cuda()[:, 8:8 + m], kept, act, DT[grad])
    f = tower.act(infcl.ckpt8_unpack(kept).cpu().double(), act)
    ref, size = dy.double().T @ f, dy.double().abs().T @ f.abs()
    # x^ is exact, f(x^) rounded; n products accumulated in fp32 in chains of 16
    tol = (n / 16 + 20) * 2.0 ** -24 * size + EPS[grad] * ref.abs()
    if act != "none":
        tol = tol + (EPS[dtype] + 1e-6) * size + 2.0 ** -24 * dy.double().abs().sum(0)[:, None]
    assert dw.dtype == DT[grad] and ((dw.cpu().double() - ref).abs() <= tol).all()
    again = infcl.ckpt8_wgrad(dy.cuda(), kept, act, DT[grad])
    assert torch.equal(dw, again)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens_q,lens_k", [([0, 200, 0, 150], [300, 200, 129, 150]), ([10, 0, 700], [700, 900, 700])])
def test_keys_that_no_query_sweeps(lens_q, lens_k, causal):
    """Heads of 128 features whose own values are copied to LDS: sequences of keys alone,
    and parts that get no tile, copy nothing that is waited for by no one."""
    _attention(lens_q, lens_k, 4, 2, 128, "bf16", causal, (max(lens_q), max(lens_k)))
