"""The text tower with rotary positions, dropout, gates, norms of what is added, and
products of 8-bit floats: chunked steps and single tokens."""

import pytest
import torch

import paper_2410_17243_amd as infcl
from paper_2410_17243_amd.gradcache import gradcache_step
from paper_2410_17243_amd.text_tower import PackedCaptions, TextTower, synthetic_captions

ALL = dict(rotary=True, gates=0.5, post_norms=True)


def _tower(kv=2, **kw):
    torch.manual_seed(1)
    return TextTower(300, 128, 2, 4, 64, 40, kv_heads=kv, act="gelu", **kw).cuda()


def test_ranges_know_their_first_token():
    c = PackedCaptions(torch.arange(10), [3, 1, 4, 2])
    assert c.first == 0 and c[1:3].first == 3 and c[1:][1:].first == 4 and c[4:].first == 10


@pytest.mark.parametrize("kw", [dict(products="int4"), dict(dropout=1.0), dict(dropout=-0.1)])
def test_choices_are_checked(kw):
    with pytest.raises(ValueError):
        TextTower(300, 128, 2, 4, 64, 40, **kw)


@pytest.mark.parametrize("products", ["16bit", "fp8"])
@pytest.mark.parametrize("act", ["silu", "none", "GELU", None])
def test_an_activation_that_is_not_there_is_refused(act, products):
    """On 8-bit products as on 16-bit ones, and before a step is taken with another."""
    with pytest.raises(ValueError, match="act must be"):
        TextTower(300, 128, 2, 4, 64, 40, act=act, products=products)


def test_frequencies_outlive_a_cast():
    """There and back, alone and inside another module, they are the same fp32 numbers; a
    tower from the meta device has those of a new one."""
    t = TextTower(300, 128, 1, 2, 64, 40, rotary=True)
    want = infcl.rotary_freqs(32, device="cpu")
    assert torch.equal(t.freqs, want)
    for cast in (lambda m: m.half(), lambda m: m.bfloat16(), lambda m: m.to("cpu", torch.float16), lambda m: m.double(), lambda m: m.float()):
        assert cast(t) is t and t.freqs.dtype == torch.float32 and torch.equal(t.freqs, want)
    torch.nn.Sequential(t).half()
    assert t.table.dtype == torch.float16 and torch.equal(t.freqs, want)
    t.to("meta")
    assert t.freqs.is_meta
    t.to_empty(device="cpu")
    assert t.freqs.dtype == torch.float32 and torch.equal(t.freqs, want)
    t.freqs = 2 * want  # (another base is kept as well)
    assert torch.equal(t.bfloat16().freqs, 2 * want) and "freqs" not in t.state_dict()
    assert TextTower(300, 128, 1, 2, 64, 40).half().freqs is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_tower_that_was_cast_is_the_one_made_so(dtype):
    """Rotary positions after .to(dtype) and .cuda(): the features of a tower of that dtype."""
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    torch.manual_seed(3)
    made = TextTower(300, 128, 2, 4, 64, 40, dtype=dt, **ALL)
    cast = TextTower(300, 128, 2, 4, 64, 40, dtype=torch.float32, **ALL)
    cast.load_state_dict({k: v.float() for k, v in made.state_dict().items()})
    c = synthetic_captions(40, 300, 40, seed=2)
    with torch.no_grad():
        assert torch.equal(cast.to(dt).cuda()(c), made.cuda()(c))


@pytest.mark.gpu
def test_gates_of_one_change_nothing():
    """The same parameters with torch's sums and norms, and with add_norm: features and
    gradients alike up to the roundings of bf16 (2^-8 each, a few of them in a row)."""
    c = synthetic_captions(40, 300, 40, seed=2)
    plain, fused = _tower(), _tower(gates=1.0)
    fused.load_state_dict(plain.state_dict(), strict=False)
    d = torch.randn((40, 64), device="cuda")
    for t in (plain, fused):
        (t(c) * d).sum().backward()
    a, b = plain(c).detach(), fused(c).detach()
    assert float((a - b).norm(dim=1).max()) < 8 * 2.0 ** -8
    grads = dict(fused.named_parameters())
    for n, p in plain.named_parameters():
        off = float((p.grad.double() - grads[n].grad.double()).norm())
        assert off <= 16 * 2.0 ** -8 * float(p.grad.double().norm()) + 1e-12, n


@pytest.mark.gpu
def test_fp32_parameters_under_autocast():
    """Residual rows in fp32 and blocks in bf16: with gates of one again alike up to the
    blocks' roundings (2^-8 each, a few in a row); on 8-bit products as far off as operands
    of 2^-5 are, through three products of two layers both ways."""
    c = synthetic_captions(40, 300, 40, seed=2)
    d = torch.randn((40, 64), device="cuda")
    plain, fused, eight = (_tower(dtype=torch.float32, **kw) for kw in ({}, {"gates": 1.0}, {"gates": 1.0, "products": "fp8"}))
    rows = []
    for t in (plain, fused, eight):
        t.load_state_dict(plain.state_dict(), strict=False)
        with torch.autocast("cuda", torch.bfloat16):
            rows.append(t(c))
        (rows[-1] * d).sum().backward()
    assert float((rows[0] - rows[1]).detach().norm(dim=1).max()) < 8 * 2.0 ** -8
    for t, bound in ((fused, 16 * 2.0 ** -8), (eight, 0.35)):
        grads = dict(t.named_parameters())
        for n, p in plain.named_parameters():
            assert grads[n].grad.dtype == torch.float32
            off = float((p.grad.double() - grads[n].grad.double()).norm())
            assert off <= bound * float(p.grad.double().norm()) + 1e-12, n


@pytest.mark.gpu
def test_chunks_have_the_whole_batchs_masks_and_gradient():
    """A step with dropout in one chunk and in four: the masks are functions of the token's
    place in the batch, so the parameters' gradients are alike up to the bf16 rounding of
    what the chunks add up (2^-8 each).  Another seed is another step."""
    c = synthetic_captions(96, 300, 40, seed=2)
    x = torch.nn.functional.normalize(torch.randn(96, 64, device="cuda"), dim=-1)
    grads, losses = [], []
    for chunk, seed in ((96, 7), (24, 7), (96, 8)):
        t = _tower(dropout=0.2, **ALL)
        t.seed = seed
        loss, _ = gradcache_step(torch.nn.Identity(), t, x.requires_grad_(), c, torch.tensor(14.29, device="cuda"), chunk)
        grads.append({n: p.grad.double() for n, p in t.named_parameters()})
        losses.append(float(loss))
    for n in grads[0]:
        a, b = grads[0][n], grads[1][n]
        assert torch.isfinite(a).all()
        assert float((a - b).norm()) <= 4 * 2.0 ** -8 * float(a.norm()) + 1e-12, n
    assert abs(losses[0] - losses[1]) < 2.0 ** -8 * losses[0] and abs(losses[0] - losses[2]) > 1e-6 * losses[0]
    t.eval()
    assert torch.equal(t(c), t(c))


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [ALL, dict(rotary=True), dict(gates=1.0, dropout=0.3), dict(products="fp8", **ALL)])
def test_extending_token_by_token_gives_the_whole_captions_features(kw):
    """Captions of one length, in one call and one token at a time, with dropout left out
    of both: the same features up to bf16 roundings.  With 8-bit operands an entry that
    differs by 2^-9 of itself is rounded to another of 2^-4 apart once in 32 times: 2^-6.5 in
    the root mean square for each operand, of four products a layer and two layers."""
    t = _tower(**kw).eval()
    tokens = torch.randint(0, 300, (5, 9), generator=torch.Generator().manual_seed(5)).cuda()
    with torch.no_grad():
        whole = t(PackedCaptions(tokens.reshape(-1), [9] * 5))
    t.train()  # (single tokens have no dropout either way)
    cache = t.new_cache(5)
    for i in range(9):
        last = t.extend(tokens[:, i].contiguous(), cache)
    bound = 16 ** 0.5 * 2.0 ** -6.5 if "products" in kw else 8 * 2.0 ** -8
    assert float((whole - last).norm(dim=1).max()) < bound


def _extended(t, tokens):
    cache = t.new_cache(tokens.shape[0])
    for i in range(tokens.shape[1]):
        last = t.extend(tokens[:, i].contiguous(), cache)
    return last, cache


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(), dict(rotary=True, gates=1.0), dict(products="fp8", **ALL)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_extending_under_autocast(kw, dtype):
    """A tower of fp32 parameters over a cache made under the same autocast: the weights are
    packed from what forward packs, byte for byte, and the features are those of whole
    captions, with the bounds of bf16 parameters (above).  A cache of another dtype is
    refused before anything of it changes."""
    t = _tower(dtype=torch.float32, **kw).eval()
    tokens = torch.randint(0, 300, (5, 9), generator=torch.Generator().manual_seed(5)).cuda()
    with torch.no_grad(), torch.autocast("cuda", dtype):
        whole = t(PackedCaptions(tokens.reshape(-1), [9] * 5))
        last, cache = _extended(t, tokens)
    bound = 16 ** 0.5 * 2.0 ** -6.5 if "products" in kw else 8 * 2.0 ** -8
    assert float((whole - last).norm(dim=1).max()) < bound
    for b, packed in zip(t.blocks, cache["packed"]):
        for name, f in packed.items():
            want = infcl.fp8_pack(getattr(b, name).detach().to(dtype))
            assert torch.equal(f.q, want.q) and torch.equal(f.exps, want.exps) and f.dtype == dtype
    taken = cache["len"].clone()
    other = torch.float16 if dtype == torch.bfloat16 else torch.bfloat16
    for context in (torch.autocast("cuda", enabled=False), torch.autocast("cuda", other)):
        with context, pytest.raises(ValueError, match="cache"):
            t.extend(tokens[:, 0].contiguous(), cache)
    assert torch.equal(cache["len"], taken) and cache["taken"] == 9


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(), dict(products="fp8", **ALL)])
def test_extending_a_tower_that_was_cast(kw):
    """The cache has the dtype that the parameters have now."""
    t = _tower(dtype=torch.float32, **kw).half().eval()
    tokens = torch.randint(0, 300, (5, 9), generator=torch.Generator().manual_seed(5)).cuda()
    with torch.no_grad():
        whole = t(PackedCaptions(tokens.reshape(-1), [9] * 5))
    last = _extended(t, tokens)[0]
    assert float((whole - last).norm(dim=1).max()) < (16 ** 0.5 * 2.0 ** -6.5 if "products" in kw else 8 * 2.0 ** -8)


@pytest.mark.gpu
def test_a_step_on_8_bit_products():
    """Every parameter has a gradient, near that of 16-bit products: each operand is off by
    2^-4 / sqrt(12) to 2^-4 / sqrt(3) of itself in the root mean square, about 2^-5, and a
    gradient passes up to three products in each of two layers both ways."""
    c = synthetic_captions(64, 300, 40, seed=4)
    d = torch.randn((64, 64), device="cuda")
    grads = []
    for products in ("16bit", "fp8"):
        t = _tower(products=products, **ALL)
        (t(c) * d).sum().backward()
        grads.append({n: p.grad.double() for n, p in t.named_parameters()})
    for n, a in grads[0].items():
        assert torch.isfinite(grads[1][n]).all()
        assert float((grads[1][n] - a).norm()) < 0.35 * float(a.norm()), n
