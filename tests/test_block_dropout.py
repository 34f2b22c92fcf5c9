"""Dropout from a counter-based generator on the GPU: its masks are those of the
definition, entry by entry."""

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import block

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,dtype,p,seed,site,row0", [
    (1, 8, "f32", 0.5, 0, 0, 0), (33, 40, "bf16", 0.1, 12345, 2, 0), (7, 136, "f16", 0.3, -1, (1 << 32) - 1, 10),
    (5, 64, "f32", 0.05, 1 << 63, 1, 1 << 40), (9, 24, "bf16", 0.999, 3, 0, 0), (3, 16, "f16", 0.0, 3, 0, 0),
    (3, 16, "f32", 1.0, 3, 0, 0), (2, 2048, "bf16", 2.0 ** -16, 7, 0, 5),
])
def test_masks_and_values(n, d, dtype, p, seed, site, row0):
    x = torch.randn((n, d), generator=torch.Generator().manual_seed(n)).to(DT[dtype])
    x[x == 0] = 1
    m = block.kept(n, d, p, seed, site, row0)
    out = infcl.dropout_fwd(x.cuda(), p, seed, site, row0).cpu()
    # the factor is rounded to fp32, and so is the product, which then is rounded to dtype: one value of two at most
    want = x.double() * m
    assert torch.equal(out == 0, m == 0)
    assert ((out.double() - want).abs() <= (torch.finfo(DT[dtype]).eps / 2 + 2.0 ** -23) * want.abs()).all()
    assert torch.equal(infcl.dropout_bwd(x.cuda(), p, seed, site, row0).cpu(), out)
    on_device = torch.tensor([seed if seed < 1 << 63 else seed - (1 << 64)], device="cuda")
    assert torch.equal(infcl.dropout_fwd(x.cuda(), p, on_device, site, row0).cpu(), out)
    wide = torch.full((n, d + 24), float("nan"), dtype=DT[dtype])
    wide[:, 8:8 + d] = x
    assert torch.equal(infcl.dropout_fwd(wide.cuda()[:, 8:8 + d], p, seed, site, row0).cpu(), out)
    assert torch.equal(infcl.dropout_fwd(x.view(1, n, d).cuda(), p, seed, site, row0).cpu()[0], out)


@pytest.mark.gpu
def test_what_is_dropped_leaves_nothing():
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = infcl.dropout_fwd(x, 0.5, 11)
    m = block.kept(64, 64, 0.5, 11).cuda()
    assert (y[m == 0] == 0).all() and not torch.isfinite(y[m != 0]).any()
    assert (infcl.dropout_fwd(x, 1.0, 11) == 0).all()


@pytest.mark.gpu
def test_a_batch_in_parts_has_the_whole_ones_masks():
    x = torch.randn((70000, 16), device="cuda")
    whole = infcl.dropout_fwd(x, 0.2, 5, site=1)
    parts = [infcl.dropout_fwd(x[a:b], 0.2, 5, site=1, row0=a) for a, b in ((0, 1), (1, 40000), (40000, 70000))]
    assert torch.equal(torch.cat(parts), whole)
    assert infcl.dropout_fwd(x[:0], 0.2, 5).shape == (0, 16)


@pytest.mark.gpu
def test_gradient_and_a_seed_that_changes():
    x = torch.randn((6, 32), device="cuda", requires_grad=True)
    seed = torch.tensor([77], device="cuda")
    y = infcl.dropout(x, 0.25, seed, site=3)
    dy = torch.randn_like(y)
    y.backward(dy)
    assert torch.equal(x.grad, infcl.dropout_fwd(dy, 0.25, 77, site=3))
    y = infcl.dropout(x, 0.25, seed, site=3)
    seed += 1
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("kw,error", [
    (dict(p=-0.1), ValueError), (dict(p=1.5), ValueError), (dict(p=float("nan")), ValueError), (dict(site=1 << 32), ValueError),
    (dict(row0=-1), ValueError), (dict(seed=torch.tensor([1], dtype=torch.int32)), ValueError), (dict(x=torch.zeros((3, 16)).t()), ValueError),
    (dict(x=torch.zeros((3, 12))), infcl.InfclError), (dict(x=torch.zeros((3, 16), dtype=torch.float64)), TypeError),
])
def test_refusals(kw, error):
    a = dict(x=torch.zeros((3, 16)), p=0.1, seed=1) | kw
    a = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in a.items()}
    with pytest.raises(error):
        infcl.dropout_fwd(**a)
