"""The text tower as it is used: chunked training steps under the tiled loss,
and captions extended token by token."""

import numpy as np
import pytest
import torch

from paper_2410_17243_amd.gradcache import gradcache_step
from paper_2410_17243_amd.text_tower import PackedCaptions, TextTower, synthetic_captions


def test_captions_are_taken_by_ranges():
    c = PackedCaptions(torch.arange(10), [3, 1, 4, 2])
    assert c.shape == (4,) and c.max_len == 4
    d = c[1:3]
    assert d.tokens.tolist() == [3, 4, 5, 6, 7] and d.cu.tolist() == [0, 1, 5] and d.positions().tolist() == [0, 0, 1, 2, 3]
    assert c[2:2].shape == (0,)
    with pytest.raises(ValueError):
        PackedCaptions(torch.arange(3), [3, 0])
    with pytest.raises(TypeError):
        c[0]


def _tower(dtype=torch.bfloat16, kv=2):
    torch.manual_seed(1)
    return TextTower(300, 128, 2, 4, 64, 40, kv_heads=kv, act="gelu", dtype=dtype).cuda()


@pytest.mark.gpu
def test_chunks_give_the_whole_batch_gradient():
    """A step in one chunk and in four: the loss's gradients reach the parameters
    alike, up to the bf16 rounding of what the chunks add up (2^-8 each)."""
    c = synthetic_captions(96, 300, 40, seed=2)
    x = torch.nn.functional.normalize(torch.randn(96, 64, device="cuda"), dim=-1)
    grads = []
    for chunk in (96, 24):
        t = _tower()
        loss, _ = gradcache_step(torch.nn.Identity(), t, x.requires_grad_(), c, torch.tensor(14.29, device="cuda"), chunk)
        assert torch.isfinite(loss)
        grads.append({n: p.grad.double() for n, p in t.named_parameters()})
    for n in grads[0]:
        a, b = grads[0][n], grads[1][n]
        assert float((a - b).norm()) <= 4 * 2.0 ** -8 * float(a.norm()) + 1e-12, n


@pytest.mark.gpu
def test_steps_lower_the_loss():
    c = synthetic_captions(64, 300, 40, seed=3)
    x = torch.nn.functional.normalize(torch.randn(64, 64, device="cuda"), dim=-1)
    t = _tower()
    opt = torch.optim.Adam(t.parameters(), lr=1e-3, eps=1e-6)
    seen = []
    for _ in range(12):
        opt.zero_grad(set_to_none=True)
        loss, _ = gradcache_step(torch.nn.Identity(), t, x.requires_grad_(), c, torch.tensor(14.29, device="cuda"), 32)
        opt.step()
        seen.append(float(loss))
    assert np.isfinite(seen).all() and seen[-1] < 0.7 * seen[0], seen


@pytest.mark.gpu
@pytest.mark.parametrize("kv", [1, 4])
def test_extending_token_by_token_gives_the_whole_captions_features(kv):
    """Captions of one length, in one call and one token at a time: the same
    features up to bf16 roundings (unit rows of 64 entries; a few of 2^-8 in the
    layers' sums)."""
    t = _tower(kv=kv)
    tokens = torch.randint(0, 300, (5, 9), generator=torch.Generator().manual_seed(5)).cuda()
    whole = t(PackedCaptions(tokens.reshape(-1), [9] * 5))
    cache = t.new_cache(5)
    for i in range(9):
        last = t.extend(tokens[:, i].contiguous(), cache)
    assert cache["len"].tolist() == [9] * 5
    assert float((whole - last).detach().norm(dim=1).max()) < 8 * 2.0 ** -8
    with pytest.raises(ValueError):
        t.extend(tokens[:2, 0].contiguous(), cache)


@pytest.mark.gpu
def test_too_long_captions_are_refused():
    with pytest.raises(ValueError):
        _tower()(PackedCaptions(torch.zeros(41, dtype=torch.int64, device="cuda"), [41]))
