"""Residual norms on the GPU against 64 bits: values and every gradient."""

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import block

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
F32 = 2.0 ** -24
NAMES = ("dx", "dy", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")


def _inputs(n, d, dtype, parts, wdtype, shift=0.0):
    g = torch.Generator().manual_seed(n * 31 + d)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    w = DT[wdtype]
    v = {"x": (r(n, d) + shift).to(DT[dtype])}
    if "y" in parts:
        v["y"] = (r(n, d) + shift).to(DT[dtype])
    for k in ("gate", "post_w", "post_b", "pre_w", "pre_b"):
        if k in parts:
            v[k] = r(d).to(w)
    dh = r(n, d).to(DT[dtype]) if "y" in parts else None
    dz = r(n, d).to(DT[dtype]) if "pre_w" in parts else None
    return v, dh, dz


def _near(got, want, size, dtype, steps):
    """One rounding to dtype, and `steps` of fp32 of what the result is computed from."""
    tol = HALF[dtype] * want.abs() + steps * F32 * size + 2.0 ** -25 * (dtype == "f16")
    off = (got.cpu().double() - want).abs() - tol
    return bool((off <= 0).all()), float(off.max())


ALL = ("y", "gate", "post_w", "post_b", "pre_w", "pre_b")
CASES = [  # rows, features, dtype, parts, the vectors' dtype, norm, alpha, p
    (1, 8, "f32", ALL, "f32", "layer", 1.0, 0.0),
    (3, 40, "bf16", ALL, "bf16", "layer", 0.5, 0.25),
    (5, 64, "f16", ("y", "pre_w"), "f16", "rms", 1.0, 0.0),
    (33, 72, "bf16", ("y", "post_w", "gate", "pre_w"), "f32", "rms", -1.5, 0.1),
    (9, 128, "f32", ("pre_w", "pre_b"), "f32", "layer", 1.0, 0.0),
    (17, 200, "f16", ("y", "post_w", "post_b"), "f32", "layer", 1.0, 0.5),
    (7, 512, "bf16", ("y", "gate"), "bf16", "rms", 2.0, 0.1),
    (300, 512, "bf16", ("y", "pre_w", "pre_b"), "bf16", "layer", 1.0, 0.0),
    (6, 520, "f32", ALL, "f32", "layer", 1.0, 0.2),            # rows of two waves, one nearly empty
    (11, 1160, "f16", ("y", "post_w", "gate", "pre_w"), "f16", "rms", 0.875, 0.1),
    (2, 8192, "bf16", ALL, "bf16", "layer", 1.0, 0.1),
    (4, 8184, "f32", ("y",), "f32", "rms", 0.25, 0.0),
    (5000, 24, "f32", ALL, "f32", "layer", 1.0, 0.1),          # many rows of few lanes
    (1100, 1032, "bf16", ("pre_w",), "f32", "rms", 1.0, 0.0),  # more rows than workgroups
    (3001, 1160, "bf16", ALL, "f32", "layer", 1.0, 0.1),       # ... with everything, in each form that has
    (2701, 1032, "f32", ALL, "f32", "layer", -0.5, 0.1),
    (2701, 776, "f32", ("y", "post_w", "gate", "pre_w"), "f32", "rms", 1.0, 0.25),
    (601, 8192, "f16", ALL, "f16", "layer", 1.0, 0.0),
    (601, 6008, "f16", ("y", "post_w", "gate", "pre_w", "pre_b"), "f16", "layer", 1.0, 0.1),
    (601, 4104, "bf16", ("y", "gate"), "bf16", "rms", 1.0, 0.5),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,dtype,parts,wdtype,norm,alpha,p", CASES)
def test_against_the_definition(n, d, dtype, parts, wdtype, norm, alpha, p):
    v, dh, dz = _inputs(n, d, dtype, parts, wdtype)
    mask = block.kept(n, d, p, 21, 4, 3) if p else None
    ref = block.add_norm(**v, rms=norm == "rms", alpha=alpha, mask=mask, dh=dh, dz=dz)
    dev = {k: t.cuda() for k, t in v.items()}
    h, z, kept = infcl.add_norm_fwd(**dev, norm=norm, alpha=alpha, p=p, seed=21, site=4, row0=3)
    grads = infcl.add_norm_bwd(dh.cuda() if dh is not None else None, dz.cuda() if dz is not None else None, kept)
    res = dict(zip(NAMES, grads)) | {"h": h, "z": z}
    if "y" not in parts:
        assert h is dev["x"]
        del res["h"]
    # sums over a row of up to 8192: 8 in a lane, 6 steps of lanes, up to 16 waves; three of them one after the
    # other, each with a few operations of its own: 64.  Sums over rows: up to 16 in a lane, 4 + 32 parts more.
    steps = {"h": 8, "z": 64}
    for k, got in res.items():
        if got is None:
            assert k not in ref or k[1:] not in v and k != "z", k
            continue
        want = ref[k]
        assert got.shape == want.shape
        ok, off = _near(got, want, ref[k + "_abs"], {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}[got.dtype],
                        steps.get(k, 128))
        assert ok, (k, off)
    assert all((res[k] is None) == (k[1:] not in v) for k in NAMES)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 1024])
def test_rows_far_from_zero(d):
    """Rows of mean 1000 and unit spread, in fp32: the variance is that of the centred row
    (the squares' mean less the mean's square would be off by 2^-24 10^6 = 6 percent)."""
    v, dh, dz = _inputs(20, d, "f32", ("y", "post_w", "pre_w"), "f32", shift=1000.0)
    ref = block.add_norm(**v)
    h, z, _ = infcl.add_norm_fwd(**{k: t.cuda() for k, t in v.items()})
    for k, got in (("h", h), ("z", z)):
        assert _near(got, ref[k], ref[k + "_abs"], "f32", 64)[0]
    # each row's spread comes out as it is: fp32 roundings of entries of 1000, 2^-15 each
    u = (z.cpu().double() / v["pre_w"].double()).square().mean(-1)
    assert (u - 1).abs().max() < 0.01


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,dtype,p,pre", [(3000, 64, "f32", 0.0, False), (3000, 1024, "f32", 0.0, False), (3001, 512, "f32", 0.25, True),
                                             (2999, 2048, "f32", 0.25, True), (3000, 128, "bf16", 0.25, True), (3000, 4096, "bf16", 0.0, True),
                                             (601, 8192, "f32", 0.25, True), (3000, 1024, "f16", 0.25, False)])
def test_a_gates_gradient_where_the_norm_and_its_bias_cancel(n, d, dtype, p, pre):
    """Rows whose entries are 2 or -2 have norms of 1 or -1, without a rounding, and biases of
    -post_w (1 - 2^-12) leave t = post_w 2^-12 of each such entry, again without one, whatever its
    sign of even features is; odd ones have t = 0.  dgate = sum e D t is then a sum of entries that
    each carry one rounding (and that of D's factor), added in fp32: up to 16 (n / 1280 rows and
    more) in a lane, 4 in a workgroup, 36 in the join, 64 in all, relative to what is added.
    The entries' own size, 2^12 times that, does not count."""
    g = torch.Generator().manual_seed(d)
    sign = torch.where(torch.arange(d) % 2 == 0, 1.0, -1.0)  # (of a feature: the same in all rows)
    v = {"x": torch.randn((n, d), generator=g).to(DT[dtype]), "y": (2 * sign).expand(n, d).contiguous().to(DT[dtype])}
    w = 1.0 + torch.randint(0, 8, (d,), generator=g) / 8.0
    v["post_w"], v["post_b"] = w, -sign * w * (1 - 2.0 ** -12 * (torch.arange(d) % 2 == 0))
    v["gate"] = torch.where(torch.arange(d) % 16 == 3, 0.0, 1.5)
    if pre:
        v["pre_w"], v["pre_b"] = torch.ones(d), torch.zeros(d)
    dh = (1 + torch.rand((n, d), generator=g)).to(DT[dtype])
    dz = torch.zeros((n, d), dtype=DT[dtype]) if pre else None  # (e = dh, without a rounding)
    dev = {k: t.cuda() for k, t in v.items()}
    _, _, kept = infcl.add_norm_fwd(**dev, norm="rms", eps=0.0, p=p, seed=9)
    grads = dict(zip(NAMES, infcl.add_norm_bwd(dh.cuda(), None if dz is None else dz.cuda(), kept)))
    # (the masks themselves have tests of their own)
    keep = (infcl.dropout_fwd(torch.ones((n, d), device="cuda"), p, 9).cpu() != 0) * (65536 / (65536 - round(p * 65536)))
    t = w.double() * 2.0 ** -12 * (torch.arange(d) % 2 == 0)
    want = (dh.double() * keep * t).sum(0)  # (all terms of one sign: their sizes' sum too)
    got = grads["dgate"].cpu().double()
    assert (got[1::2] == 0).all()
    assert ((got - want).abs() <= 64 * F32 * want).all(), float(((got - want).abs() / (F32 * want + 1e-30))[0::2].max())
    for k, scale in (("dpost_w", sign), ("dpost_b", torch.ones(d))):
        full = (dh.double() * keep).sum(0) * v["gate"].double() * scale.double()
        assert ((grads[k].cpu().double() - full).abs() <= 64 * F32 * full.abs()).all(), k


@pytest.mark.gpu
def test_equal_rows_and_zeros():
    """Rows without a spread: eps alone is their size; the gradient is finite."""
    x = torch.zeros((3, 64), device="cuda")
    x[1] = 5.0
    w, b = torch.ones(64, device="cuda"), torch.full((64,), 0.5, device="cuda")
    for norm in ("layer", "rms"):
        _, z, kept = infcl.add_norm_fwd(x, pre_w=w, pre_b=b, norm=norm)
        assert (z[0] == 0.5).all() and (z[1] == (0.5 if norm == "layer" else z[1, 0])).all()
        assert all(torch.isfinite(t).all() for t in infcl.add_norm_bwd(None, torch.ones_like(z), kept) if t is not None)


@pytest.mark.gpu
def test_what_is_not_finite_stays_in_its_row():
    v, dh, dz = _inputs(9, 96, "bf16", ALL, "bf16")
    v["x"][2, 5], v["y"][6, 90] = float("nan"), float("inf")
    h, z, kept = infcl.add_norm_fwd(**{k: t.cuda() for k, t in v.items()})
    dx, dy = infcl.add_norm_bwd(dh.cuda(), dz.cuda(), kept)[:2]
    for t in (z, dx, dy):
        rows = torch.isfinite(t).all(1).cpu()
        assert rows.tolist() == [i not in (2, 6) for i in range(9)]


@pytest.mark.gpu
def test_rows_of_wider_arrays_and_missing_gradients():
    v, dh, dz = _inputs(13, 72, "bf16", ALL, "f32")
    dev = {k: t.cuda() for k, t in v.items()}

    def wide(t):
        w = torch.full((t.shape[0], t.shape[1] + 40), float("nan"), dtype=t.dtype, device="cuda")
        w[:, 16:16 + t.shape[1]] = t.cuda()
        return w[:, 16:16 + t.shape[1]]

    h, z, kept = infcl.add_norm_fwd(**dev, p=0.2, seed=3)
    grads = infcl.add_norm_bwd(dh.cuda(), dz.cuda(), kept)
    h2, z2, kept2 = infcl.add_norm_fwd(**(dev | {"x": wide(v["x"]), "y": wide(v["y"])}), p=0.2, seed=3)
    grads2 = infcl.add_norm_bwd(wide(dh), wide(dz), kept2)
    assert torch.equal(h, h2) and torch.equal(z, z2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    zero = torch.zeros((13, 72), dtype=torch.bfloat16, device="cuda")
    for a, b in (((None, dz.cuda()), (zero, dz.cuda())), ((dh.cuda(), None), (dh.cuda(), zero)), ((None, None), (zero, zero))):
        assert all(torch.equal(s, t) for s, t in zip(infcl.add_norm_bwd(*a, kept), infcl.add_norm_bwd(*b, kept)))
    some = infcl.add_norm_bwd(dh.cuda(), dz.cuda(), kept, need=(False, True, False, True, False, False, True))
    assert [t is None for t in some] == [True, False, True, False, True, True, False]
    assert all(t is None or torch.equal(t, u) for t, u in zip(some, grads))
    assert infcl.add_norm_fwd(**dev, need_grad=False)[2] is None


@pytest.mark.gpu
def test_no_rows():
    v, _, _ = _inputs(0, 64, "f32", ALL, "f32")
    h, z, kept = infcl.add_norm_fwd(**{k: t.cuda() for k, t in v.items()})
    grads = infcl.add_norm_bwd(h, z, kept)
    assert h.shape == z.shape == grads[0].shape == grads[1].shape == (0, 64)
    assert all((t == 0).all() and t.shape == (64,) for t in grads[2:])


@pytest.mark.gpu
@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_autograd_gives_the_same_and_torchs_numbers(norm):
    """In fp32 against torch's own norms in fp64, with shapes of three dimensions; outputs
    that no one uses have no gradient."""
    v, dh, dz = _inputs(12, 64, "f32", ALL, "f32")
    dev = {k: (t.view(3, 4, 64) if t.dim() == 2 else t).cuda().requires_grad_() for k, t in v.items()}
    h, z = infcl.add_norm(**dev, norm=norm, alpha=0.5)
    torch.autograd.backward((h, z), (dh.view(3, 4, 64).cuda(), dz.view(3, 4, 64).cuda()))
    ref = {k: t.double().requires_grad_() for k, t in v.items()}
    f = torch.nn.functional
    unit = (lambda t, w, b: f.layer_norm(t, (64,), w, b)) if norm == "layer" else (lambda t, w, b: f.rms_norm(t, (64,), w, 1e-5) + b)
    rh = 0.5 * ref["x"] + ref["gate"] * unit(ref["y"], ref["post_w"], ref["post_b"])
    rz = unit(rh, ref["pre_w"], ref["pre_b"])
    torch.autograd.backward((rh, rz), (dh.double(), dz.double()))
    for k in v:
        # (the formulas' own bounds are in test_against_the_definition; here 2^-17 of the norm)
        a, b = dev[k].grad.cpu().double().reshape(ref[k].shape), ref[k].grad
        assert float((a - b).norm()) < 2.0 ** -17 * float(b.norm()), k
    x, y = dev["x"], dev["y"]
    h, none = infcl.add_norm(x, y, gate=dev["gate"])
    assert none is None and torch.autograd.grad(h, x, dh.view(3, 4, 64).cuda())[0].equal(dh.view(3, 4, 64).cuda())
    same, z = infcl.add_norm(x, pre_w=dev["pre_w"], norm=norm)
    assert same is x
    (dx,) = torch.autograd.grad((same * 2).sum() + z.sum(), x)
    (dzx,) = torch.autograd.grad(infcl.add_norm(x, pre_w=dev["pre_w"], norm=norm)[1].sum(), x)
    assert torch.equal(dx, dzx + 2)
    with torch.no_grad():
        assert not infcl.add_norm(x, y, pre_w=dev["pre_w"])[1].requires_grad


@pytest.mark.gpu
@pytest.mark.parametrize("kw,error", [
    (dict(y=torch.zeros((4, 8))), ValueError), (dict(y=torch.zeros((4, 16)).half()), ValueError), (dict(gate=torch.zeros(8)), ValueError),
    (dict(pre_w=torch.zeros(16).half()), ValueError), (dict(pre_w=None, y=None), ValueError), (dict(y=None, p=0.5), ValueError),
    (dict(y=None, gate=torch.zeros(16)), ValueError), (dict(y=None, alpha=2.0), ValueError), (dict(post_b=torch.zeros(16)), ValueError),
    (dict(pre_w=None, pre_b=torch.zeros(16)), ValueError), (dict(norm="batch"), ValueError), (dict(eps=-1.0), infcl.InfclError),
    (dict(p=2.0), ValueError), (dict(x=torch.zeros((4, 12)), y=None, pre_w=torch.zeros(12)), infcl.InfclError),
    (dict(x=torch.zeros((1, 8200)), y=None, pre_w=torch.zeros(8200)), infcl.InfclError), (dict(x=torch.zeros((4, 16)).double(), y=None), (TypeError, ValueError)),
])
def test_refusals(kw, error):
    a = dict(x=torch.zeros((4, 16)), y=torch.zeros((4, 16)), pre_w=torch.zeros(16)) | kw
    a = {k: t.cuda() if isinstance(t, torch.Tensor) else t for k, t in a.items()}
    with pytest.raises(error):
        infcl.add_norm_fwd(**a)
