"""The tower's autograd functions as the graph sees them, without a GPU: the
kernels' places are taken by torch products that leave no graph, as the kernels
leave none."""

import math

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import tower as oracle
from paper_2410_17243_amd import tower


@pytest.fixture
def plain_kernels(monkeypatch):
    """Stand-ins that compute in the inputs' type on the CPU and keep x as it is."""
    keep = lambda x: tower.Ckpt8(x.detach().clone(), torch.zeros((*x.shape[:-1], 1), dtype=torch.uint8), x.dtype)  # noqa: E731

    def wgrad(dy, kept, act="none", grad_dtype=None):
        x = oracle.act(kept.q.reshape(-1, kept.q.shape[-1]), act)
        return (dy.detach().reshape(-1, dy.shape[-1]).T @ x).to(grad_dtype or torch.float32)

    def attn_fwd(q, k, v, cu_q, max_q, *rest, **kw):
        r = oracle.attention(q.detach(), k.detach(), v.detach(), cu_q.tolist(), cu_q.tolist(), True, q.shape[2] ** -0.5)
        return r["out"].to(q.dtype), r["lse"].float()

    def attn_bwd(q, k, v, out, lse, dout, cu_q, max_q, *rest, grads=None, **kw):
        r = oracle.attention(q.detach(), k.detach(), v.detach(), cu_q.tolist(), cu_q.tolist(), True, q.shape[2] ** -0.5,
                             dout.detach())
        got = tuple(r[n].to(q.dtype) for n in ("dq", "dk", "dv"))
        for to, x in zip(grads or (), got):
            to.copy_(x)
        return got

    for name, fn in {
        "ckpt8_pack": keep, "ckpt8_act_fwd": lambda x, act: (oracle.act(x.detach(), act), keep(x)), "ckpt8_wgrad": wgrad,
        "ckpt8_act_bwd": lambda dy, kept, act: dy.detach() * oracle.act_slope(kept.q, act),
        "embed_fwd": lambda tok, table, scale=1.0: scale * table.detach()[tok],
        "embed_bwd": lambda tok, dout, vocab, scale=1.0, gdt=None: torch.zeros((vocab, dout.shape[-1]), dtype=gdt).index_add_(
            0, tok.reshape(-1), scale * dout.detach().reshape(-1, dout.shape[-1])),
        "packed_attn_fwd": attn_fwd, "packed_attn_bwd": attn_bwd,
    }.items():
        monkeypatch.setattr(tower, name, fn)


def _call(name):
    """(the function of its differentiable arguments, those arguments)."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: (torch.randn(s, generator=g) / math.sqrt(s[-1])).bfloat16().requires_grad_()  # noqa: E731
    cu = torch.tensor([0, 4, 6], dtype=torch.int32)
    return {
        "embed": (lambda w: infcl.embed(torch.tensor([1, 0, 3]), w, 2.0), [r(5, 8)]),
        "linear8": (infcl.linear8, [r(6, 8), r(16, 8), r(16)]),
        "mlp8": (lambda *a: infcl.mlp8(*a, act="gelu"), [r(6, 8), r(16, 8), r(16), r(8, 16), r(8)]),
        "packed_attn": (lambda q, k, v: infcl.packed_attn(q, k, v, cu, 4), [r(6, 2, 8), r(6, 1, 8), r(6, 1, 8)]),
        "packed_attn_qkv": (lambda x: infcl.packed_attn_qkv(x, 2, 1, cu, 4), [r(6, 4, 8)]),
    }[name]


NAMES = ["embed", "linear8", "mlp8", "packed_attn", "packed_attn_qkv"]


@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_are_refused(plain_kernels, name):
    """The kernels leave no graph: a gradient of a gradient would miss what went
    through them, so it is an error, and not a number."""
    f, args = _call(name)
    first = torch.autograd.grad(f(*args).square().sum(), args, create_graph=True)
    assert all(torch.isfinite(x).all() for x in first)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (args[0].square().sum() + sum(x.square().sum() for x in first)).backward()  # (a penalty beside a plain term)


def _layers():
    r = lambda *s: torch.randn(s, generator=torch.Generator().manual_seed(5)).bfloat16().requires_grad_()  # noqa: E731
    f32 = lambda *s: r(*s).detach().float().requires_grad_()  # noqa: E731
    mlp = lambda *a: infcl.mlp8(*a, act="gelu")  # noqa: E731
    return {
        "linear8, 12 outputs": (infcl.linear8, (r(6, 8), r(12, 8), None), ValueError),
        "linear8, fp32": (infcl.linear8, (f32(6, 8), f32(16, 8), None), TypeError),
        "mlp8, 12 outputs": (mlp, (r(6, 8), r(16, 8), None, r(12, 16), None), ValueError),
        "mlp8, 12 inside": (mlp, (r(6, 8), r(12, 8), None, r(8, 12).detach(), None), ValueError),
        "mlp8, fp32": (mlp, (f32(6, 8), f32(16, 8), f32(16), f32(8, 16), f32(8)), TypeError),
        "mlp8, fp32, one layer learns": (mlp, (f32(6, 8), f32(16, 8).detach(), None, f32(8, 16), None), TypeError),
    }


@pytest.mark.parametrize("name", list(_layers()))
def test_layers_refuse_in_the_forward_what_the_backward_cannot_do(name):
    """Widths that are no multiple of 8, and fp32 products, where a weight gradient is to come."""
    f, args, error = _layers()[name]
    with pytest.raises(error, match="layer"):
        f(*args)


@pytest.mark.parametrize("name", ["linear8", "mlp8"])
def test_layers_with_frozen_weights_need_no_weight_gradient(plain_kernels, name):
    """What only the weight gradient asks for is not asked for without one: fp32, and
    12 outputs."""
    g = torch.Generator().manual_seed(3)
    x, w1, w2 = torch.randn((6, 8), generator=g).requires_grad_(), torch.randn((16, 8), generator=g), torch.randn((12, 16), generator=g)
    y = infcl.linear8(x, w2[:, :8]) if name == "linear8" else infcl.mlp8(x, w1, None, w2, None)
    y.sum().backward()
    assert torch.isfinite(x.grad).all()
    with torch.no_grad():
        same = infcl.linear8(x, w2[:, :8].requires_grad_()) if name == "linear8" else infcl.mlp8(x, w1, None, w2.requires_grad_(), None)
    assert torch.equal(same, y)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["linear8", "mlp8"])
def test_fp32_weights_under_autocast(name):
    """fp32 weights and inputs under autocast: what the same layer gives for their
    bf16 roundings, gradients included, with the backward pass outside of autocast."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    args = [r(40, 64), r(48, 64), r(48)] + ([r(16, 48), r(16)] if name == "mlp8" else [])
    f = infcl.linear8 if name == "linear8" else (lambda *a: infcl.mlp8(*a, act="gelu"))
    dy = r(40, 48 if name == "linear8" else 16).bfloat16()
    low = [a.bfloat16().requires_grad_() for a in args]
    y = f(*low)
    y.backward(dy)
    wide = [a.bfloat16().float().requires_grad_() for a in args]
    with torch.autocast("cuda", torch.bfloat16):
        z = f(*wide)
    z.backward(dy)
    assert z.dtype == torch.bfloat16 and torch.equal(z, y)
    for a, b in zip(wide, low):
        # (a bias's gradient is an fp32 sum under autocast)
        assert a.grad.dtype == torch.float32 and torch.equal(a.grad.bfloat16(), b.grad)


def test_a_table_that_learns_takes_as_many_tokens_as_its_gradient():
    """The gradient sorts up to 2^26 tokens; more are refused before the forward's work."""
    table, n = torch.empty((100, 8), device="meta", requires_grad=True), 1 << 26
    for tokens, status in ((n + 1, infcl.INFCL_ERR_UNSUPPORTED), (n, None)):
        with pytest.raises((infcl.InfclError, ValueError)) as e:
            infcl.embed(torch.empty(tokens, dtype=torch.int32, device="meta"), table)
        assert getattr(e.value, "status", None) == status  # (n of them get as far as the device's check)
    with torch.no_grad(), pytest.raises(ValueError, match="device"):
        infcl.embed(torch.empty(n + 1, dtype=torch.int32, device="meta"), table)
