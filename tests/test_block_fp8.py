"""Operands in 8-bit floats on the GPU, their products and layers, against 64 bits."""

import math

import pytest
import torch

import paper_2410_17243_amd as infcl
from oracle import block
from paper_2410_17243_amd import block as binding

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def _x(n, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    spread = torch.exp2(torch.randint(-12, 3, (n, d // 8 + 1), generator=g).float()).repeat_interleave(8, 1)[:, :d]
    return (torch.randn((n, d), generator=g) * spread).to(DT[dtype])


def _value(byte):
    """What an 8-bit float stands for."""
    s, e, m = byte >> 7, (byte >> 3) & 15, byte & 7
    v = math.nan if byte & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return -v if s else v


TABLE = torch.tensor([_value(b) for b in range(256)], dtype=torch.float64)


def _held(f):
    """(values in units of the block's power of two [rows, k], exponents) of an Fp8."""
    q = TABLE[f.q.cpu().long()]
    assert (f.q.cpu()[:, f.k:(f.k + 127) // 128 * 128] == 0).all() or torch.isnan(q).any()  # (what fills up a row)
    e = f.exps.cpu().long()
    assert (e[:, (f.k + 127) // 128:] == 127).all()
    return q[:, :f.k], e[:, :(f.k + 127) // 128]


def _q(f):
    """Its bytes, without what may follow a row's last block."""
    return f.q[:, :(f.k + 127) // 128 * 128]


def _same(f, x):
    q, e = _held(f)
    rq, re = block.fp8(x)
    return torch.equal(e, re) and torch.equal(torch.nan_to_num(q, nan=999.0), torch.nan_to_num(rq, nan=999.0))


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,dtype", [(1, 8, "bf16"), (3, 136, "f16"), (130, 40, "f32"), (5, 1032, "bf16"), (257, 264, "f16"),
                                       (128, 128, "f32"), (127, 248, "bf16"), (9, 16384, "bf16")])
def test_packing_both_ways(n, d, dtype):
    x = _x(n, d, dtype)
    if n > 2:
        x[1] = 0
        x[2, :8] = torch.tensor([448.0, 449, -17, 19, 0.001953125, 0.0009765625, 3e-3, -464]).to(DT[dtype])
    a, t = infcl.fp8_pack_both(x.cuda())
    assert a.shape == (n, d) and t.shape == (d, n) and _same(a, x) and _same(t, x.t())
    only = infcl.fp8_pack(x.cuda())
    assert torch.equal(_q(only), _q(a)) and torch.equal(_held(only)[1], _held(a)[1])
    want = block.unfp8(*block.fp8(x)).to(DT[dtype])
    assert torch.equal(infcl.fp8_unpack(a).cpu(), want)
    assert torch.equal(infcl.fp8_unpack(t).cpu(), block.unfp8(*block.fp8(x.t())).to(DT[dtype]))
    wide = torch.full((n, d + 24), math.nan, dtype=DT[dtype])
    wide[:, 8:8 + d] = x
    v, w = infcl.fp8_pack_both(wide.cuda()[:, 8:8 + d])
    assert torch.equal(_q(v), _q(a)) and torch.equal(_q(w), _q(t))


@pytest.mark.gpu
def test_packing_at_the_ends():
    """Infinities and NaN take their block, subnormal and the largest numbers are kept."""
    x = torch.zeros((9, 256))
    x[0, 3], x[1, 200], x[2, 5] = math.inf, math.nan, -math.inf
    x[3, 0], x[3, 130] = 3.4028234e38, -3.4e38
    x[4, 0], x[5, 7] = 1e-45, 2.0 ** -127
    x[6, :3] = torch.tensor([65504.0, -65504.0, 1.0])
    x[7], x[8, 128] = 2.5e38, -0.0
    a, t = infcl.fp8_pack_both(x.cuda())
    assert _same(a, x) and _same(t, x.t())
    y = infcl.fp8_unpack(a).cpu()
    assert torch.isnan(y[0, :128]).all() and (y[0, 128:] == 0).all() and torch.isnan(y[1, 128:]).all() and torch.isfinite(y[3:]).all()
    assert float(infcl.fp8_unpack(infcl.fp8_pack(x[6:7].half().cuda()))[0, 0]) == 65504.0


def _whole(n, k, dtype, seed):
    """Entries whose products and sums are whole numbers that 8 bits and fp32 hold exactly,
    and whose groups of products span less than 13 bits: the product is exact."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-4, 5, (n, k), generator=g).to(DT[dtype])


SIZES = [  # n, m, k
    (1, 1, 1), (1, 3, 130), (16, 40, 512), (17, 5, 300), (33, 129, 1), (130, 257, 640), (128, 128, 4096), (300, 24, 9001),
    (520, 300, 4200), (1000, 513, 72), (256, 256, 33000), (700, 2056, 1160), (4099, 1030, 513),
    (40, 264, 16384), (9000, 1032, 200), (9000, 1031, 136), (20000, 520, 1160), (4096, 4096, 520),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,m,k", SIZES)
def test_products_of_whole_numbers_are_exact(n, m, k, dtype):
    """Every tile, part of the contraction, odd end and bias: sums that fp32 holds, rounded
    once."""
    kk = (k + 7) // 8 * 8  # (rows to pack are whole chunks: zeros)
    x, w = _whole(n, kk, dtype, 1), _whole(m, kk, dtype, 2)
    x[:, k:] = 0
    b = _whole(1, m, dtype, 3)[0] if n % 2 else None
    # powers of two for each row and block, as scales of real rows differ
    if k < 600:
        x = x * torch.exp2(torch.arange(n) % 5 - 2.0)[:, None].to(DT[dtype])
        w = w * torch.exp2(torch.arange(m) % 3 - 1.0)[:, None].to(DT[dtype])
    a, c = infcl.fp8_pack(x.cuda()), infcl.fp8_pack(w.cuda())
    out = infcl.fp8_matmul(a, c, b.cuda() if b is not None else None)
    want = x.cuda().double() @ w.cuda().double().t() + (b.cuda().double() if b is not None else 0)
    assert torch.equal(out, want.to(DT[dtype]))
    if dtype == "bf16":
        assert torch.equal(infcl.fp8_matmul(a, c, dtype=torch.float16), (x.cuda().double() @ w.cuda().double().t()).half())
    if kk * n <= 1 << 21:
        assert torch.equal(infcl.linear_fp8(x.cuda(), c, b.cuda() if b is not None else None), out)


# powers of two of a's and b's rows; the last ones' results are subnormal in fp32 and bf16
FAR = [(100, -100), (-100, 100), (60, -63), (-60, -60), (-60, 60), (110, 0), (0, -118), (-117, 117), (119, -119), (-110, 106),
       (-64, -64), (-33, -100), (-126, -10)]


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 16, 40, 300])
@pytest.mark.parametrize("ea,eb", FAR)
def test_products_of_exponents_far_apart_are_exact(ea, eb, n):
    """Whole numbers up to 4 times powers of two at both ends of bf16, in the kernel of few rows
    and that of tiles: each scale may be next to its end, and sums that fp32 holds as subnormals
    are kept.  Blocks beside them in the contraction are zeros (exponent byte 1), or
    of the other end against zeros: they add nothing."""
    k, m = 1032, 72
    x, w = _whole(n, k, "bf16", 7), _whole(m, k, "bf16", 8)
    x, w = x * torch.tensor(2.0 ** ea).bfloat16(), w * torch.tensor(2.0 ** eb).bfloat16()
    x[:, 128:256], w[:, 256:384] = 0, 0
    w[:, 128:256] = 2.0 ** 126  # against zeros
    x[:, 256:384] = -(2.0 ** 126)
    x[:, 384:512], w[:, 384:512] = 0, 0
    a, c = infcl.fp8_pack(x.cuda()), infcl.fp8_pack(w.cuda())
    e = infcl.fp8_unpack(a)
    assert torch.equal(e.cpu(), x)
    want = (x.cuda().double() @ w.cuda().double().t()).to(torch.bfloat16)
    assert torch.isfinite(want).all() and float(want.float().abs().max()) > 0
    assert torch.equal(infcl.fp8_matmul(a, c), want)
    assert torch.equal(infcl.linear_fp8(x.cuda(), c), want)


@pytest.mark.gpu
@pytest.mark.parametrize("n,m,k,dtype", [(5, 48, 264, "bf16"), (16, 100, 4096, "f16"), (40, 72, 1032, "bf16"), (300, 520, 2048, "f16"),
                                         (1025, 264, 776, "bf16")])
def test_products(n, m, k, dtype):
    """Random rows.  A group of eight products loses less than 7 of 2^-13 of its largest; the
    groups are added in fp32 (k / 8 roundings).  In the root mean square the loss is below
    2^-14 of the result's size, beside a rounding (2^-p / sqrt 3)."""
    x, w = _x(n, k, dtype, 4), _x(m, k, dtype, 5)
    b = torch.randn(m, generator=torch.Generator().manual_seed(6)).to(DT[dtype])
    a, c = block.unfp8(*block.fp8(x)), block.unfp8(*block.fp8(w))
    want, size = a @ c.t() + b.double(), a.abs() @ c.abs().t() + b.double().abs()
    packed = infcl.fp8_pack(w.cuda())
    for out in (infcl.fp8_matmul(infcl.fp8_pack(x.cuda()), packed, b.cuda()), infcl.linear_fp8(x.cuda(), packed, b.cuda())):
        off = (out.cpu().double() - want).abs()
        assert (off <= HALF[dtype] * want.abs() + (7 * 2.0 ** -13 + k / 8 * 2.0 ** -24) * size + 2.0 ** -25).all()
        assert float(off.norm() / want.norm()) < HALF[dtype] / math.sqrt(3) + 2.0 ** -14


@pytest.mark.gpu
def test_not_finite_entries_reach_their_rows_only():
    x, w = torch.randn((40, 256)).bfloat16(), torch.randn((24, 256)).bfloat16()
    x[7, 40], w[3, 200] = math.nan, math.inf
    for n in (40, 16):
        y = infcl.linear_fp8(x[:n].cuda(), infcl.fp8_pack(w.cuda())).cpu()
        bad = torch.zeros((n, 24), dtype=torch.bool)
        bad[7], bad[:, 3] = True, True
        assert torch.equal(~torch.isfinite(y), bad)


@pytest.mark.gpu
@pytest.mark.parametrize("n,k,m,dtype", [(1, 8, 8, "bf16"), (50, 136, 72, "f16"), (333, 512, 264, "bf16"), (2050, 256, 128, "f16")])
def test_a_layer_and_its_gradients(n, k, m, dtype):
    """Every product of linear_fp8 on what its operands stand for, with the bounds of
    test_products; the bias's gradient is the plain sum."""
    g = torch.Generator().manual_seed(n)
    r = lambda *s: torch.randn(s, generator=g).to(DT[dtype])  # noqa: E731
    x, w, b, dy = r(n, k), r(m, k), r(m), r(n, m)
    args = [t.cuda().requires_grad_() for t in (x.view(1, n, k), w, b)]
    y = infcl.linear_fp8(*args)
    y.backward(dy.view(1, n, m).cuda())
    held = lambda t: block.unfp8(*block.fp8(t))  # noqa: E731
    pairs = {
        "y": (y, held(x), held(w)), "dx": (args[0].grad, held(dy), held(w.t()).t().t()),
        "dw": (args[1].grad, held(dy.t()), held(x.t())),
    }
    for name, (got, a, c) in pairs.items():
        want, size = a @ c.t(), a.abs() @ c.abs().t()
        if name == "y":
            want, size = want + b.double(), size + b.double().abs()
        off = (got.detach().cpu().double().view(want.shape) - want).abs()
        assert (off <= HALF[dtype] * want.abs() + (7 * 2.0 ** -13 + a.shape[1] / 8 * 2.0 ** -24) * size + 2.0 ** -25).all(), name
    db, s = dy.double().sum(0), dy.double().abs().sum(0)
    assert ((args[2].grad.cpu().double() - db).abs() <= HALF[dtype] * db.abs() + 32 * 2.0 ** -24 * s).all()
    y2, kept = infcl.linear_fp8_fwd(x.cuda(), w.cuda(), b.cuda())
    grads = infcl.linear_fp8_bwd(dy.cuda(), kept)
    assert torch.equal(y2, y[0]) and all(torch.equal(p, a.grad.view(p.shape)) for p, a in zip(grads, args))


@pytest.mark.gpu
def test_frozen_arguments_keep_and_compute_nothing():
    x, w, b = torch.randn((20, 64)).bfloat16().cuda(), torch.randn((16, 64)).bfloat16().cuda(), torch.randn(16).bfloat16().cuda()
    full = [t.clone().requires_grad_() for t in (x, w, b)]
    infcl.linear_fp8(*full).square().sum().backward()
    for i in range(3):
        args = [t.clone().requires_grad_(j == i) for j, t in enumerate((x, w, b))]
        infcl.linear_fp8(*args).square().sum().backward()
        assert torch.equal(args[i].grad, full[i].grad)
    odd = infcl.linear_fp8(x, w[:5], b[:5])  # (no gradient: any number of outputs)
    leaf = x.clone().requires_grad_()
    assert torch.equal(infcl.linear_fp8_fwd(leaf, w[:5], b[:5], need_dx=False, need_dw=False)[0], odd)
    assert torch.equal(odd, infcl.linear_fp8(x, w, b)[:, :5])
    with pytest.raises(ValueError, match="multiple of 8"):
        infcl.linear_fp8(x, w[:5].clone().requires_grad_(), b[:5])


@pytest.mark.gpu
def test_without_gradients_nothing_is_kept(monkeypatch):
    x = torch.randn(64, 256, device="cuda").bfloat16().requires_grad_()
    w, b = (torch.randn(s, device="cuda").bfloat16().requires_grad_() for s in ((40, 256), (40,)))
    y = infcl.linear_fp8(x, w, b)
    keeps = []
    sizes = binding._layer_sizes
    monkeypatch.setattr(binding, "_layer_sizes", lambda *a: keeps.append(a[3]) or sizes(*a))
    with torch.no_grad():
        assert torch.equal(infcl.linear_fp8(x, w, b), y) and keeps == [0]
        assert torch.equal(infcl.linear_fp8(x, w[:5], b[:5]), y[:, :5])  # (any number of outputs)


@pytest.mark.gpu
def test_more_rows_than_a_weights_gradient_takes():
    """The rows are a contraction for dw alone, up to 2^23: without it there may be more, as
    with packed weights.  The last rows are what they are alone."""
    n = (1 << 23) + 40
    x = torch.randn((n, 8), device="cuda").bfloat16()
    w, b = torch.randn((8, 8), device="cuda").bfloat16(), torch.randn(8, device="cuda").bfloat16()
    y = infcl.linear_fp8(x, w, b)
    assert torch.equal(y, infcl.linear_fp8(x, infcl.fp8_pack(w), b)) and torch.equal(y[-50:], infcl.linear_fp8(x[-50:], w, b))
    del y
    tail = x[-50:].clone().requires_grad_()
    xr, br, dy = x.requires_grad_(), b.clone().requires_grad_(), torch.ones((n, 8), dtype=torch.bfloat16, device="cuda")
    dx, db = torch.autograd.grad(infcl.linear_fp8(xr, w, br), (xr, br), dy)
    assert torch.equal(dx[-50:], torch.autograd.grad(infcl.linear_fp8(tail, w), tail, dy[:50])[0])
    assert (db == float(torch.tensor(n).bfloat16())).all()  # (sums of up to 128 ones, then of 65537 of them: whole numbers)
    with pytest.raises(infcl.InfclError):  # (in the forward)
        infcl.linear_fp8(x.detach(), w.requires_grad_(), b)


@pytest.mark.gpu
def test_no_rows_and_autocast():
    w, b = torch.randn((16, 64), device="cuda"), torch.randn(16, device="cuda")
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda").requires_grad_()
    a, c = w.bfloat16().requires_grad_(), b.bfloat16().requires_grad_()
    y = infcl.linear_fp8(x, a, c)
    y.sum().backward()
    assert y.shape == (0, 16) and x.grad.shape == (0, 64) and (a.grad == 0).all() and (c.grad == 0).all()
    x = torch.randn((9, 64), device="cuda", requires_grad=True)
    w.requires_grad_()
    with torch.autocast("cuda", torch.bfloat16):
        y = infcl.linear_fp8(x, w, b)
        packed = infcl.linear_fp8(x.detach(), infcl.fp8_pack(w.detach().bfloat16()), b)
    assert y.dtype == torch.bfloat16 and torch.equal(packed, y)
    y.float().square().sum().backward()
    assert x.grad.dtype == w.grad.dtype == torch.float32 and float(w.grad.abs().sum()) > 0


@pytest.mark.gpu
def test_refusals():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    f = infcl.fp8_pack(x)
    with pytest.raises(ValueError):
        infcl.fp8_pack(x.t())
    with pytest.raises(ValueError):
        infcl.fp8_pack(x.cpu())
    with pytest.raises(TypeError):
        infcl.fp8_pack(x.double())
    with pytest.raises(infcl.InfclError):
        infcl.fp8_pack(torch.zeros((4, 12), device="cuda"))
    with pytest.raises(ValueError):
        infcl.fp8_matmul(f, infcl.fp8_pack(x[:, :56]))
    with pytest.raises(ValueError):
        infcl.fp8_matmul(f, f, torch.zeros(3, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        infcl.fp8_matmul(f, f, dtype=torch.float32)
    with pytest.raises(ValueError):
        infcl.fp8_unpack(infcl.Fp8(f.q[:, :64], f.exps, 64, x.dtype))
    with pytest.raises(ValueError):
        infcl.fp8_matmul(infcl.Fp8(f.q, f.exps[:2], 64, x.dtype), f)
    with pytest.raises(ValueError):
        infcl.linear_fp8(x, torch.zeros((8, 56), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        infcl.linear_fp8(x.float(), x.float())
    with pytest.raises(ValueError):
        infcl.linear_fp8(x.half(), x)
    with pytest.raises(ValueError, match="no backward"):
        infcl.linear_fp8(x.clone().requires_grad_(), f)
    with pytest.raises(TypeError):
        infcl.linear_fp8(x.float(), f)
