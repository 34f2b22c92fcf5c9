"""Rotary positions on the GPU against 64 bits."""

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import block

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
F32 = 2.0 ** -24


def _tol(ref, size, turns, dtype):
    """Sine and cosine are off by 1.5 roundings of the angle's rest, two of their own; two
    products and a sum add one each: 8 in all, of |u| + |v|.  The angle in turns is one
    fp64 product, off by 2^-52 of itself.  Then the rounding to dtype (steps of 2^-25 at
    the lower end of fp16)."""
    return HALF[dtype] * ref.abs() + (8 * F32 + 6.3 * turns * 2.0 ** -52) * size + 2.0 ** -25 * (dtype == "f16")


CASES = [  # tokens, heads, turned, head_dim, sections, dtype, neighbours, float positions, most position
    (1, 1, 1, 8, (1,), "f32", False, False, 10),
    (1, 3, 2, 64, (32,), "bf16", False, False, 1 << 20),
    (5, 4, 4, 64, (8, 12, 12), "f16", False, False, 100),
    (7, 2, 1, 80, (8, 14, 14), "bf16", True, False, 100),      # features and heads that are copied
    (9, 3, 3, 72, (36,), "f32", False, True, 3000),             # pairs that are no multiple of 8
    (3, 5, 4, 24, (3, 2), "f16", False, False, 1000),
    (4, 2, 2, 40, (1, 2, 3, 7), "bf16", True, True, 50),        # four axes
    (2, 1, 1, 1024, (512,), "bf16", False, False, 77),
    (3, 2, 0, 16, (8,), "f32", False, False, 9),                # none turned
    (2, 2, 2, 128, (64,), "f32", True, False, (1 << 31) - 1),   # as far out as int32 goes
    (2, 300, 200, 16, (8,), "bf16", False, False, 9),
    (4100, 2, 1, 32, (16,), "f16", False, False, 77),           # several tokens to a workgroup, an odd number of them
]


@pytest.mark.gpu
@pytest.mark.parametrize("n,heads,turned,hd,sections,dtype,nb,fl,most", CASES)
def test_against_the_definition(n, heads, turned, hd, sections, dtype, nb, fl, most):
    g = torch.Generator().manual_seed(n + hd)
    x = torch.randn((n, heads, hd), generator=g).to(DT[dtype])
    pos = torch.randint(-(most // 3), most, (n, len(sections)), generator=g, dtype=torch.int32)
    pos[0] = most
    pos = pos.float() * 0.375 if fl else pos
    freqs = infcl.rotary_freqs(sections, device="cpu")
    rest = (sections, turned, "neighbours" if nb else "halves")
    out = infcl.rotary_fwd(x.cuda(), pos.cuda(), freqs.cuda(), *rest).cpu()
    ref, size, turns = block.turned(x, pos, freqs, sections, turned, nb)
    assert out.dtype == DT[dtype] and ((out.double() - ref).abs() <= _tol(ref, size, turns, dtype)).all()
    kept = torch.ones(x.shape, dtype=torch.bool)
    kept[:, :turned, :2 * sum(sections)] = False
    assert torch.equal(out[kept], x[kept])
    back = infcl.rotary_bwd(x.cuda(), pos.cuda(), freqs.cuda(), *rest).cpu()
    ref, size, turns = block.turned(x, pos, freqs, sections, turned, nb, back=True)
    assert ((back.double() - ref).abs() <= _tol(ref, size, turns, dtype)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,pairs,nb", [(64, 32, False), (40, 15, False), (48, 20, True)])
def test_views(hd, pairs, nb, dtype):
    """Heads of a projection, heads before tokens, rows of wider positions, one position
    of several, and none: the same numbers as of copies."""
    g = torch.Generator().manual_seed(hd)
    qkv = torch.randn((6, 7, hd), generator=g).to(DT[dtype]).cuda()
    pos = torch.randint(0, 90, (6, 3), generator=g, dtype=torch.int32).cuda()
    freqs, rest = infcl.rotary_freqs(pairs), (None, None, "neighbours" if nb else "halves")
    want = infcl.rotary_fwd(qkv.clone(), pos[:, 0].contiguous(), freqs, *rest)
    assert torch.equal(infcl.rotary_fwd(qkv[:, 2:5], pos[:, :1], freqs, *rest), want[:, 2:5])
    assert torch.equal(infcl.rotary_fwd(qkv, pos[:, 0], freqs, *rest), want)
    turned = qkv.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(infcl.rotary_fwd(turned, pos[:, :1], freqs, *rest), want)
    assert torch.equal(infcl.rotary_fwd(qkv[::2], pos[::2, 0], freqs, *rest), want[::2])
    assert torch.equal(infcl.rotary_fwd(qkv[5:], pos[5:, 0], freqs, *rest), want[5:])
    one = infcl.rotary_fwd(qkv, pos[:1, 0].expand(6), freqs, *rest)
    assert torch.equal(one, infcl.rotary_fwd(qkv, pos[:1, 0].repeat(6), freqs, *rest))
    assert infcl.rotary_fwd(qkv[:0], pos[:0, 0], freqs, *rest).shape == (0, 7, hd)


@pytest.mark.gpu
def test_what_is_not_finite_stays_in_its_pair():
    x = torch.ones((2, 2, 32), device="cuda")
    x[0, 0, 3], x[1, 1, 30] = float("nan"), float("inf")
    y = infcl.rotary_fwd(x, torch.tensor([5, 6], dtype=torch.int32, device="cuda"), infcl.rotary_freqs(12))
    bad = ~torch.isfinite(y)
    assert bad.nonzero().tolist() == [[0, 0, 3], [0, 0, 15], [1, 1, 30]]


@pytest.mark.gpu
def test_gradient_and_attention_in_a_row():
    """rotary of queries and keys, then packed attention: the gradient of the projection
    against that in fp64 (bf16 roundings of the turned heads, the weights and the results,
    2^-8 each, in the root mean square)."""
    g = torch.Generator().manual_seed(3)
    lens, heads, kv, hd = [5, 1, 9], 4, 2, 32
    qkv = torch.randn((15, heads + 2 * kv, hd), generator=g).bfloat16().cuda().requires_grad_()
    cu = torch.tensor([0, 5, 6, 15], dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(m) for m in lens]).int().cuda()
    freqs = infcl.rotary_freqs(16)
    do = torch.randn((15, heads, hd), generator=g).bfloat16().cuda()
    out = infcl.packed_attn_qkv(infcl.rotary(qkv, pos, freqs, turned=heads + kv), heads, kv, cu, 9)
    out.backward(do)
    x = qkv.detach().cpu().double().requires_grad_()
    ang = pos.cpu().double()[:, None] * freqs.cpu().double()
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    r = x[:, :heads + kv]
    r = torch.cat([r[..., :16] * c - r[..., 16:] * s, r[..., 16:] * c + r[..., :16] * s], -1)
    at, outs = 0, []
    for m in lens:
        q, k, v = r[at:at + m, :heads], r[at:at + m, heads:], x[at:at + m, heads + kv:]
        k, v = k.repeat_interleave(heads // kv, 1), v.repeat_interleave(heads // kv, 1)
        w = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) * hd ** -0.5
        w = torch.softmax(w + torch.triu(torch.full((m, m), float("-inf"), dtype=torch.float64), 1), -1)
        outs.append(torch.matmul(w, v.transpose(0, 1)).transpose(0, 1))
        at += m
    ref = torch.cat(outs)
    ref.backward(do.cpu().double())
    for a, b in ((out.detach(), ref.detach()), (qkv.grad, x.grad)):
        assert float((a.cpu().double() - b).norm() / b.norm()) < 4 * 2.0 ** -8


@pytest.mark.parametrize("kw,error", [
    (dict(pos=torch.zeros(4, dtype=torch.int64)), TypeError), (dict(pos=torch.zeros(3, dtype=torch.int32)), ValueError),
    (dict(freqs=torch.zeros(4, dtype=torch.float64)), ValueError), (dict(sections=(3,)), ValueError),
    (dict(sections=(2, 2)), ValueError), (dict(paired="thirds"), ValueError), (dict(turned=3), ValueError),
    (dict(x=torch.zeros((4, 2, 16)).transpose(1, 2)), ValueError), (dict(x=torch.zeros((4, 2, 16), dtype=torch.float64)), TypeError),
    (dict(pos=torch.zeros((4, 5), dtype=torch.int32), sections=(1,) * 5), ValueError),
])
@pytest.mark.gpu
def test_refusals(kw, error):
    a = dict(x=torch.zeros((4, 2, 16)), pos=torch.zeros(4, dtype=torch.int32), freqs=torch.zeros(4)) | kw
    for k in ("x", "pos", "freqs"):
        a[k] = a[k].cuda()
    with pytest.raises(error):
        infcl.rotary_fwd(**a)


def test_tensors_of_the_host_are_refused():
    with pytest.raises(ValueError, match="device"):
        infcl.rotary_fwd(torch.zeros((4, 2, 16)), torch.zeros(4, dtype=torch.int32), torch.zeros(8))
